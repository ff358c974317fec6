// Which kernel and tile a product with 8-bit weights takes: host side, from extents and the device (tests compile it by itself).
#pragma once
#include "expert_mm_plan.hpp"

namespace tc355 {

// Side of the (square) tile: the estimate is a compute unit's number of tiles times a tile's products, over the rate that the side reaches relative to the others, and as
// many stages more as a tile's start and end take.  float outputs (by the half instruction) take 128 at most.  The rates are those of operands that come from memory, not from the
// caches that the product before left them in: tiles of 128, two a compute unit, ask for a third more of them at a time and lose most.  Measured so (sets of operands in turn),
// bfloat16, us, sides 64 / 128 / 256: (E,R,N,K) = (1,4096,8192,4096) 241 / 166 / 131, 8192^3 839 / 580 / 456, of (1,4096,8192,1024) 66 / 47 / 49, uneven shares (32,16384,2048,4096)
// 276 / 195 / 180, even ones 264 / 178 / 136, uneven (32,16384,4096,2048) 293 / 211 / 183, (8,16384,2048,4096) 240 / 173 / 159, (16,16384,2048,4096) 256 / 191 / 168, (64,16384,2048,2048)
// 173 / 133 / 113, (128,32768,1024,2048) 186 / 134 / 116, (128,16384,2048,1024) 133 / 103 / 106, (8,4096,4096,4096) 152 / 115 / 106, (16,2048,2048,2048) 35 / 26 / 37, (64,2048,1024,2048) 41 / 34 / 39,
// (256,16384,1024,2048) 151 / 136 / 153, (1,512,4096,4096) 21 / 27 / 54, (4,2000,512,512) 6.1 / 8.0 / 16.  Over 41 shapes the choice is 2.2 % off the best side; at worst 15 %, where an expert's few rows
// make short tiles of 256, which the estimate counts as half lost: (16,4096,2048,2048) 51 / 43 / 38, (32,8192,1024,2048) 51 / 44 / 38, taken 128.  float, sides 64 / 128, from the caches: (1,4096,4096,4096) 216 / 183, (32,8192,2048,2048) 146 / 128, (16,2048,2048,2048) 39 / 47,
// (12,2100,1001,517) 12 / 17.
inline int q8_tile_side(bool f32, int cus, int64_t R, int64_t E, int64_t NO, int64_t stages) {
  const struct {
    int side;
    double rate, more;
  } sides[] = {{256, f32 ? 0 : 1.0, 2}, {128, f32 ? 1.0 : 0.7, 1}, {64, f32 ? 0.85 : 0.45, 0.5}};
  int best = 0;
  double least = 0;
  for (const auto& s : sides) {
    if (s.rate == 0) continue;
    const double load = expected_row_tiles(R, E, s.side) * (double)ceil_div(NO, s.side) / cus;
    const double t = (load < 1 ? 1 : load) * s.side * s.side / s.rate * (1 + s.more / (double)stages);
    if (!best || t < least) {
      best = s.side;
      least = t;
    }
  }
  return best;
}

// Whether a product goes to the kernel for few rows (16 rows by 32 columns a workgroup, the reduction shared by its wavefronts) rather than to tiles of 64: while it has up to two
// workgroups a compute unit (three for float).  Beyond, tiles read the rows' share of the operands less often.  Measured, us, few / tiles: (1,1,8192,4096) 7.5 / 18, 16 rows 9.9 / 19, 33 rows 20 / 19,
// 63 rows 27 / 20; (1,32,2048,8192) 16 / 23; (1,100,512,4096) 9.0 / 13; (8,8,1024,4096) 8.0 / 13; (8,32,4096,2048) 14.3 / 14.0, float 16 / 21; (8,128,4096,2048) 22 / 14;
// (32,128,2048,1024) 24 / 13; (1,16,4096,1024) 5.5 / 5.2.
inline bool q8_few_rows(bool f32, int cus, int64_t R, int64_t E, int64_t NO) {
  return expected_row_tiles(R, E, 16) * (double)ceil_div(NO, 32) <= (f32 ? 3.0 : 2.0) * cus;
}

}  // namespace tc355
