// The host's choices between kernels of the products grouped by expert, for tests that hold them against what was measured.
#include "expert_mm_plan.hpp"

using namespace tc355;

extern "C" int few_rows(int f32, int whole, int cus, int64_t R, int64_t E, int64_t N) { return expert_few_rows(f32 != 0, whole != 0, cus, R, E, N); }

extern "C" int weights_parts(int f32, int cus, int64_t R, int64_t E, int64_t N, int64_t K, int side) { return expert_weights_parts(f32 != 0, cus, R, E, N, K, side); }
extern "C" int weights_side(int most, int cus, int64_t E, int64_t N, int64_t K) {
  return expert_tile_side(most, cus, [&](int b) { return (double)E * (double)ceil_div(N, b) * (double)ceil_div(K, b); });
}
extern "C" int rows_side(int most, int cus, int64_t R, int64_t E, int64_t out) {
  return expert_tile_side(most, cus, [&](int b) { return expected_row_tiles(R, E, b) * (double)ceil_div(out, b); });
}
