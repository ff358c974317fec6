// Which kernel and tile a product with 8-bit weights takes: host side, from extents and the device (tests compile it by itself).
#pragma once
#include "expert_mm_plan.hpp"

namespace tc355 {

// Side of the (square) tile.  Products of float outputs, which go by the half instruction, take 128 at most.
inline int q8_tile_side(bool f32, int cus, int64_t R, int64_t E, int64_t NO) {
  return expert_tile_side(f32 ? 128 : 256, cus, [&](int b) { return expected_row_tiles(R, E, b) * (double)ceil_div(NO, b); });
}

// Whether a product goes to the kernel for few rows rather than to tiles.
inline bool q8_few_rows(int cus, int64_t R, int64_t E, int64_t NO) {
  if (R / E >= 64) return false;
  const double few = expected_row_tiles(R, E, 16) * ceil_div(NO, 32) / cus, tile = expected_row_tiles(R, E, 64) * ceil_div(NO, 64) / cus;
  return 1 + 1.5 * (few > 0.5 ? few - 0.5 : 0) <= 4.5 + (tile > 0.5 ? tile - 0.5 : 0);
}

}  // namespace tc355
