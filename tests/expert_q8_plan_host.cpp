// The host's choice of a kernel and tile for products with 8-bit weights, for tests that ask which one their shapes take.
#include "expert_mm_q8_plan.hpp"

extern "C" int q8_side(int f32, int cus, int64_t R, int64_t E, int64_t NO, int64_t stages) { return tc355::q8_tile_side(f32 != 0, cus, R, E, NO, stages); }
extern "C" int q8_few(int f32, int cus, int64_t R, int64_t E, int64_t NO) { return tc355::q8_few_rows(f32 != 0, cus, R, E, NO); }
