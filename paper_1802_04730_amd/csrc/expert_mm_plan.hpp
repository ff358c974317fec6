// Which tile a product grouped by expert takes: host side, from extents and the device (tests compile it by itself).
#pragma once
#include "tc355_host.hpp"

namespace tc355 {

// Row tiles that R rows of E experts can need, whatever their shares, those of no expert among them.
inline int64_t most_row_tiles(int64_t R, int64_t E, int64_t bm) {
  const int64_t n = (R + (E + 1) * (bm - 1)) / bm;
  return R < n ? R : n;
}

// Shares of the experts are not known here: R/E rows each with half a tile lost is what a router's make of it.
inline double expected_row_tiles(int64_t R, int64_t E, int64_t bm) { return (double)R / bm + 0.5 * (double)(E < R ? E : R); }

// Side of the (square) tile, `most` or less, for `tiles(side)` tiles: the estimate is a compute unit's number of tiles times a
// tile's products, over the rate that the side reaches on large extents (relative to 256; 16-bit storage, 8192^3: 1268, 1092 TFLOP/s
// and about 780).  Larger tiles read less per product; smaller ones lose less to the last row tile of an expert and to compute units
// without a tile.  Measured, us, sides 256 / 128 / 64: (E,R,N,K) = (8,16384,4096,4096) 492 / 617 / -, (16,8192,4096,2048) 195 / 192 / 266,
// (16,2048,2048,2048) 51 / 36 / 41, (4,2000,512,512) 21 / 12 / 8.  fp32 takes 64 always: at a rate of the matrix core that is a sixteenth, no tile is
// short of operands ((16,2048,2048,2048) 497 / 259 / 223, (64,16384,1024,2048) 1023 / 777 / 692); products with an operand across its rows
// take 128 at most, since 256 has too few registers left for them (dX and dW of (8,16384,4096,4096): 557 and 856 / 613 and 618).
template <typename F>
int expert_tile_side(int most, int cus, F tiles) {
  const struct {
    int side;
    double rate;
  } sides[] = {{256, 1.0}, {128, 0.87}, {64, 0.62}};
  int best = 0;
  double least = 0;
  for (const auto& s : sides) {
    if (s.side > most) continue;
    const double load = tiles(s.side) / cus, t = (load < 1 ? 1 : load) * s.side * s.side / s.rate;
    if (!best || t < least) {
      best = s.side;
      least = t;
    }
  }
  return best;
}

}  // namespace tc355
