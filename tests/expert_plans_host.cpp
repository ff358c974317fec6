// The host's choice of a tile for the products grouped by expert, for tests that ask which one their shapes take.
#include "expert_mm_plan.hpp"

using namespace tc355;

// A product with R rows of E experts and `out` columns.
extern "C" int rows_side(int most, int cus, int64_t R, int64_t E, int64_t out) {
  return expert_tile_side(most, cus, [&](int b) { return expected_row_tiles(R, E, b) * (double)ceil_div(out, b); });
}
extern "C" int weights_side(int most, int cus, int64_t E, int64_t N, int64_t K) {
  return expert_tile_side(most, cus, [&](int b) { return (double)E * (double)ceil_div(N, b) * (double)ceil_div(K, b); });
}
extern "C" int weights_parts(int f32, int cus, int64_t R, int64_t E, int64_t N, int64_t K, int side) {
  return expert_weights_parts(f32 != 0, cus, R, E, N, K, side);
}
extern "C" int64_t row_tiles(int64_t R, int64_t E, int64_t bm) { return most_row_tiles(R, E, bm); }
