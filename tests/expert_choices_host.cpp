// The host's choices between kernels of the products grouped by expert, for tests that hold them against what was measured.
#include "expert_mm_plan.hpp"

using namespace tc355;

extern "C" int few_rows(int f32, int whole, int cus, int64_t R, int64_t E, int64_t N) { return expert_few_rows(f32 != 0, whole != 0, cus, R, E, N); }
