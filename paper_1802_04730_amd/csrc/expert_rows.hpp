// Products grouped by expert where an expert has few rows (a decoding step): Y(r,n) = act(sum_k X(src(r),k) * W(e(r),n,k)).
// What bounds it: the weights' bytes, each read for a handful of rows.  32 rows of 8 experts, 4096 x 2048 bfloat16: 26-29 us a call (4.6-5.2 TB/s of weights), the kernel 23.5 (5.7).
//
// A workgroup computes 16 rows by 16 CT columns of one expert; its wavefronts share the reduction, in steps of 64 bytes of a row.
// Operands go from memory to registers in the matrix instruction's layout -- nothing is used twice, so LDS would only be a
// detour -- with EROWS_AHEAD steps requested together, and the partial tiles meet once, in LDS, in the wavefronts' order.
// expert_few_rows (expert_mm_plan.hpp) says which products it takes.
#pragma once
#include "expert_mm.hpp"

namespace tc355 {

constexpr int EROWS_AHEAD = 4;  // steps in flight of a wavefront

template <typename T, int CT, int WK>
__global__ __launch_bounds__(64 * WK) void expert_few_rows_kernel(ExpertRowsArgs p) {
  constexpr int PER = Elem<T>::PER16, STEP = 4 * PER, U = EROWS_AHEAD;
  __shared__ __align__(16) f4 part[WK][CT][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15, q = lane >> 4;
  ExpertTile t;
  if (!expert_tile(p.off, p.E, p.R, 16, p.nt, blockIdx.x, &t)) return;
  const int hi = __builtin_amdgcn_readfirstlane(t.hi), e = __builtin_amdgcn_readfirstlane(t.e);
  const int m0 = __builtin_amdgcn_readfirstlane(t.lo) + __builtin_amdgcn_readfirstlane(t.m) * 16, n0 = __builtin_amdgcn_readfirstlane(t.n) * (16 * CT);
  const bool owned = e < p.E && p.T > 0;
  f4 acc[CT];
#pragma unroll
  for (int n = 0; n < CT; n++) acc[n] = f4{0, 0, 0, 0};
  if (owned) {
    const int steps = (p.Q + STEP - 1) / STEP, whole = p.Q / STEP;
    const int first = (int)((int64_t)steps * wave / WK), last = (int)((int64_t)steps * (wave + 1) / WK);
    const int row = min(m0 + i, hi - 1);
    const T* a = static_cast<const T*>(p.A) + (int64_t)(p.row ? min(max(p.row[row], 0), p.T - 1) : row) * p.Q + (int64_t)first * STEP + q * PER;
    const T* b[CT];
#pragma unroll
    for (int n = 0; n < CT; n++)
      b[n] = static_cast<const T*>(p.W) + ((int64_t)e * p.NO + min(n0 + 16 * n + i, p.NO - 1)) * p.Q + (int64_t)first * STEP + q * PER;
    int s = first;
    const int end = min(last, whole);
    for (; s + U <= end; s += U) {
      Pack<T, PER> fb[U][CT], fa[U];
#pragma unroll
      for (int u = 0; u < U; u++) {
#pragma unroll
        for (int n = 0; n < CT; n++) fb[u][n] = load_pack<T, PER>(b[n] + u * STEP);
        fa[u] = load_pack<T, PER>(a + u * STEP);
      }
#pragma unroll
      for (int u = 0; u < U; u++)
#pragma unroll
        for (int n = 0; n < CT; n++) acc[n] = emm_mfma<T>(__builtin_bit_cast(u4, fb[u][n]), __builtin_bit_cast(u4, fa[u]), acc[n]);
#pragma unroll
      for (int n = 0; n < CT; n++) b[n] += U * STEP;
      a += U * STEP;
    }
    for (; s < last; s++) {
      const int at = s * STEP + q * PER;  // (of a pointer that has come this far)
      u4 fb[CT];
#pragma unroll
      for (int n = 0; n < CT; n++) fb[n] = emm_load_any(b[n] - at, at, p.Q);
      const u4 fa = emm_load_any(a - at, at, p.Q);
#pragma unroll
      for (int n = 0; n < CT; n++) acc[n] = emm_mfma<T>(fb[n], fa, acc[n]);
#pragma unroll
      for (int n = 0; n < CT; n++) b[n] += STEP;
      a += STEP;
    }
  }
#pragma unroll
  for (int n = 0; n < CT; n++) part[wave][n][lane] = acc[n];
  __syncthreads();
  const bool by4 = (p.NO & 3) == 0;
  for (int n = wave; n < CT; n += WK) {
    const int r = m0 + i, c = n0 + 16 * n + 4 * q;
    f4 v = part[0][n][lane];
#pragma unroll
    for (int w = 1; w < WK; w++) v += part[w][n][lane];
    if (r >= hi || c >= p.NO) continue;
    if (p.row && owned && (p.row[r] < 0 || p.row[r] >= p.T)) v = f4{0, 0, 0, 0};  // (a row of zeros)
    if (p.relu) {
#pragma unroll
      for (int x = 0; x < 4; x++) v[x] = v[x] > 0.0f ? v[x] : 0.0f;  // (NaN and -0 give +0)
    }
    emm_store(static_cast<T*>(p.C) + (int64_t)r * p.NO + c, p.NO - c, by4, v);
  }
}

}  // namespace tc355
