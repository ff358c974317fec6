// Storage types of the operators around experts (float, bfloat16, IEEE half) and what their kernels share.
//
// Values are widened to 32 bits (float storage: to 64 where a kernel only streams) as they are read, summed there, and rounded to the
// storage type once, to nearest even, when an output is written.
#pragma once
#include "tc355_device.hpp"

namespace tc355 {

typedef __bf16 bf16;
typedef _Float16 f16;
typedef short s4v __attribute__((ext_vector_type(4)));
typedef unsigned u4 __attribute__((ext_vector_type(4)));

template <typename T> struct Elem;
template <> struct Elem<float> {
  typedef float v4 __attribute__((ext_vector_type(4)));
  typedef v4 v16;  // 16 bytes
  static constexpr int PER16 = 4;
};
template <> struct Elem<bf16> {
  typedef bf16 v4 __attribute__((ext_vector_type(4)));
  typedef bf16 v8 __attribute__((ext_vector_type(8)));
  typedef v8 v16;
  static constexpr int PER16 = 8;
};
template <> struct Elem<f16> {
  typedef f16 v4 __attribute__((ext_vector_type(4)));
  typedef f16 v8 __attribute__((ext_vector_type(8)));
  typedef v8 v16;
  static constexpr int PER16 = 8;
};

// V neighbours whose elements alone are aligned: one load or store of up to 16 bytes all the same (global memory).
template <typename T, int V>
struct __attribute__((packed, aligned(sizeof(T)))) Pack {
  T e[V];
};
template <typename T, int V>
__device__ __forceinline__ Pack<T, V> load_pack(const T* p) {
  return *reinterpret_cast<const Pack<T, V>*>(p);
}
// Stores pass the caches by: outputs are far larger than those, or read by a later launch (16384 rows of 4096 bfloat16 out of a table: 73 us,
// so 46; with a launch behind it that reads them back 62 us either way).
template <typename T, int V>
__device__ __forceinline__ void store_pack(T* p, const Pack<T, V>& v) {
  constexpr int BYTES = sizeof(T) * V;
  if constexpr (BYTES == 16 || BYTES == 8) {
    typedef unsigned words __attribute__((ext_vector_type(BYTES / 4)));
    typedef unsigned words_any __attribute__((ext_vector_type(BYTES / 4), aligned(sizeof(T))));
    __builtin_nontemporal_store(static_cast<words_any>(__builtin_bit_cast(words, v)), reinterpret_cast<words_any*>(p));
  } else {
#pragma unroll
    for (int i = 0; i < V; i++) __builtin_nontemporal_store(v.e[i], p + i);
  }
}

// The columns of a row of `width` (at least V) that unit `u` of V handles.  The last unit of a width that is no multiple of V begins V
// before the end: what it loads is whole, without a branch -- which would make each load wait for the one before --, and it owns the
// elements from `skip` on.  (Rows narrower than 16 bytes go by units of one element.)
template <int V>
struct RowUnit {
  int c, skip;
  bool on;
  __device__ __forceinline__ RowUnit(int64_t u, int width) {
    const int64_t at = u * V;
    on = at < width;
    c = (int)(on ? at : 0);
    skip = max(0, c + V - width);
    c -= skip;
  }
};
template <typename T, int V>
__device__ __forceinline__ Pack<T, V> load_unit(const T* row, const RowUnit<V>& u) {
  return load_pack<T, V>(row + u.c);
}
template <typename T, int V>
__device__ __forceinline__ void store_unit(T* row, const RowUnit<V>& u, const Pack<T, V>& v) {
  if (u.skip == 0) {
    store_pack<T, V>(row + u.c, v);
  } else {
#pragma unroll
    for (int i = 1; i < V; i++)
      if (i >= u.skip) __builtin_nontemporal_store(v.e[i], row + u.c + i);
  }
}

// What a kernel that only streams sums in: float storage in 64 bits, as everywhere in the library; 16-bit storage in 32.
template <typename T> struct Wide { typedef float type; };
template <> struct Wide<float> { typedef double type; };

// Rounded once from the wide type.
template <typename T, typename S>
__device__ __forceinline__ T narrow(S v) {
  return static_cast<T>(v);
}

}  // namespace tc355
