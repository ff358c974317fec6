// Exchange between the lanes of a wavefront: reductions over groups of 16 or 64 lanes.
#pragma once
#include "tc355_device.hpp"

namespace tc355 {

// f(x, y) over the G lanes of a group, in all of them, f the same both ways round: y of another lane.  Rows of 16 lanes by moves between lanes, beyond by swaps of rows and of
// halves: a wavefront's two copies of x become its even rows (halves) and its odd ones.
template <int CTRL, typename X>
__device__ __forceinline__ X from_lane(X x) {
  if constexpr (sizeof(X) == 8) {
    typedef int two __attribute__((ext_vector_type(2)));
    const two v = __builtin_bit_cast(two, x);
    const two o = {__builtin_amdgcn_update_dpp(0, v[0], CTRL, 0xf, 0xf, true), __builtin_amdgcn_update_dpp(0, v[1], CTRL, 0xf, 0xf, true)};
    return __builtin_bit_cast(X, o);
  } else {
    return __builtin_bit_cast(X, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
  }
}
template <bool HALVES, typename X>
__device__ __forceinline__ void swap_rows(X x, X& even, X& odd) {
  constexpr int W = sizeof(X) / 4;
  typedef unsigned words __attribute__((ext_vector_type(W)));
  const words v = __builtin_bit_cast(words, x);
  words a, b;
#pragma unroll
  for (int i = 0; i < W; i++) {
    const auto r = HALVES ? __builtin_amdgcn_permlane32_swap(v[i], v[i], false, false) : __builtin_amdgcn_permlane16_swap(v[i], v[i], false, false);
    a[i] = r[0];
    b[i] = r[1];
  }
  even = __builtin_bit_cast(X, a);
  odd = __builtin_bit_cast(X, b);
}
template <int G, typename X, typename F>
__device__ __forceinline__ X group_all(X x, F f) {
  x = f(x, from_lane<0xB1>(x));   // lane ^ 1
  x = f(x, from_lane<0x4E>(x));   // lane ^ 2
  x = f(x, from_lane<0x141>(x));  // 7 - lane of 8: the other four
  x = f(x, from_lane<0x140>(x));  // 15 - lane: the other eight
  if constexpr (G > 16) {
    X even, odd;
    swap_rows<false>(x, even, odd);
    x = f(even, odd);
    if constexpr (G > 32) {
      swap_rows<true>(x, even, odd);
      x = f(even, odd);
    }
  }
  return x;
}
__device__ __forceinline__ float most_of(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ float sum_of(float a, float b) { return a + b; }
__device__ __forceinline__ unsigned larger(unsigned a, unsigned b) { return a > b ? a : b; }
__device__ __forceinline__ int smaller(int a, int b) { return a < b ? a : b; }

}  // namespace tc355
