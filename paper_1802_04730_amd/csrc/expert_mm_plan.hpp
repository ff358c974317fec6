// Which tile a product grouped by expert takes: host side, from extents and the device (tests compile it by itself).
#pragma once
#include <cmath>

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
// tile's products, over the rate that the side reaches relative to 256.  Larger tiles read less per product; smaller ones lose less to the last row tile of an
// expert and to compute units without a tile.  Measured, bfloat16, us, sides 256 / 128 / 64: 8192^3 774 / 975 / 1468; uneven shares, (E,R,N,K) = (8,16384,4096,4096) 508 / 603 / 910,
// (16,8192,4096,2048) 181 / 175 / 249, (32,16384,2048,4096) 349 / 352 / 493, (16,2048,2048,2048) 46 / 31 / 40, (4,2000,512,512) 15.6 / 7.5 / 6.2.  Over 70 drawn shapes the choice is
// 2.0 % off the best side forward, 0.6 % for dX, 1.1 % for dW (geometric means; at worst 1.35, 1.13, 1.64 times).  fp32 takes 64 always: at a rate of the matrix core that is a
// sixteenth, no tile is short of operands ((16,2048,2048,2048) 497 / 259 / 223, (64,16384,1024,2048) 1023 / 777 / 692).  Products with an operand across its rows
// take 128 at most, since there is no tile of 256 for them: one that was tried took 557 us for dX of (8,16384,4096,4096) where 128 took 613, and 856 for dW where
// 128 took 618 (too few registers).
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

// Whether a product whose experts have fewer than 64 rows on average goes to the kernel for few rows (expert_rows.hpp: 16 rows by 32 columns, no
// LDS) rather than to tiles.  Either one's time grows with its workgroups per compute unit beyond a half; a lone tile takes 4.5 times (rows of no
// whole 16-byte pieces: twice, fp32: 5 and 4.5 times) as long as a lone workgroup of the few rows.  Measured, us, few rows / tiles, weights from memory: bfloat16, 8 experts, N = 4096,
// K = 2048, with 4 rows each 30 / 35, 8: 32 / 35, 16: 42 / 35, 32: 61 / 35, 63: 103 / 40 (64 rows of one expert, in a kernel of that shape that was here: 67);
// 32 experts, 2048, 1024: 4 rows 30 / 26; small products always: 12 experts of 58 rows, 130, 1000: 7.4 / 10.2; fp32, 8 experts, 2048, 1024: 16 rows 19 / 25, 32: 29 / 25;
// width 4099 x 2047: 4 rows 70 / 58.  Over 2417 shapes of up to 63 rows an expert the choice is 1.5 % off the better one (geometric mean; at worst 1.54 times).
// Where one expert has all rows, which no average tells: 64 x 32 rows, 1024 x 2048 88 / 20 (tiles are taken), 8 x 8 rows, 4096 x 2048 14 / 17 (few rows).
inline bool expert_few_rows(bool f32, bool whole, int cus, int64_t R, int64_t E, int64_t N) {
  if (R / E >= 64) return false;
  const double few = expected_row_tiles(R, E, 16) * ceil_div(N, 32) / cus, tile = expected_row_tiles(R, E, 64) * ceil_div(N, 64) / cus;
  const double lone = f32 ? (whole ? 5 : 4.5) : whole ? 4.5 : 2, each = f32 ? 6 : whole ? 1 : 3;
  return 1 + 1.5 * (few > 0.5 ? few - 0.5 : 0) <= lone + each * (tile > 0.5 ? tile - 0.5 : 0);
}

// Parts into which the gradient of the weights cuts each expert's rows: tiles of the weights alone may be too few for the device, and
// the longest expert's rows take their time however many compute units wait.  Estimated, us: rounds of workgroups (four on a compute unit) times
// the rows of a part of a longer expert, taken as 1.5 times the average, plus, with parts, a launch and the way of the partial sums
// to the workspace and back; more parts where they save 15 %.  Measured, us, 1 / 2 / 4 / 8 / 16 parts: bfloat16 (E,R,N,K) = (4,65536,256,256)
// 161 / 91 / 51 / 37 / 42, (1,8192,512,512) 59 / 36 / 22 / 18 / 22, (4,131072,1024,1024) 634 / 449 / 403 / 397 / 425, (16,16384,256,512) 23 / 25 / 28 / 37 / 54; fp32
// (4,65536,256,256) 512 / 261 / 136 / 114 / 113, (2,3000,64,64) 41 / 25 / 15 / 10 / 9, (8,8192,1024,512) 93 / 103 / 102 / 114 / 168.  Over 380 shapes the choice is 1.0 % off the best number
// (geometric mean; at worst 1.28 times).
constexpr int EMM_MOST_PARTS = 16;
inline int expert_weights_parts(bool f32, int cus, int64_t R, int64_t E, int64_t N, int64_t K, int side) {
  const double tiles = (double)E * ceil_div(N, side) * ceil_div(K, side), rows = (double)R / E * (E > 1 ? 1.5 : 1);
  const double row = side == 128 ? 0.5 / 64 : f32 ? 1.0 / 32 : 0.85 / 64;  // of a tile, us
  int best = 1;
  double least = 0;
  for (int s = 1; s <= EMM_MOST_PARTS; s *= 2) {
    const double t = std::ceil(tiles * s / (4 * cus)) * (rows / s * row + 2) + (s > 1 ? 3.5 + 12.0 * s * E * N * K / 4e6 : 0);
    if (s == 1 || t < 0.85 * least) {
      best = s;
      least = t;
    }
  }
  return best;
}

}  // namespace tc355
