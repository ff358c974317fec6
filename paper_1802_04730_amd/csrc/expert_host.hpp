// What the host sides of the operators around experts share: limits, checks of arguments, launches.
#pragma once
#include "../../include/tc355.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "expert_types.hpp"
#include "tc355_host.hpp"

namespace tc355 {

constexpr int64_t kMostRows = (int64_t)1 << 30;   // rows, widths: 32-bit indices with room for a tile
constexpr int64_t kMostWidth = (int64_t)1 << 22;  // of the products: a tile's 256 rows of fp32 within 32-bit offsets
constexpr int64_t kMostIndex = ((int64_t)1 << 31) - 1;

inline bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }
inline tc_status launched() { return hipGetLastError() == hipSuccess ? TC_OK : TC_ERR_LAUNCH; }
inline tc_status took(const char* path, tc_status st) {
  note_path(path);
  return st;
}
inline bool known(tc_type t) { return t == TC_F32 || t == TC_BF16 || t == TC_F16; }
inline int bits_of(int64_t v) {  // of a number up to v
  int b = 1;
  while (b < 62 && (v >> b)) b++;
  return b;
}
inline int64_t round256(int64_t n) { return (n + 255) / 256 * 256; }

// f(T{}) with the storage type
template <typename F>
tc_status by_type(tc_type t, F f) {
  if (t == TC_F32) return f(float{});
  if (t == TC_BF16) return f(bf16{});
  return f(f16{});
}

// launch(workgroups, first): one after the other until all `n` workgroups of WG_THREADS have run.
template <typename F>
tc_status in_launches(int64_t n, F launch) {
  for (int64_t at = 0; at < n;) {
    const int64_t some = next_launch(n - at, WG_THREADS);
    launch(dim3((unsigned)some), at);
    at += some;
  }
  return launched();
}

}  // namespace tc355
