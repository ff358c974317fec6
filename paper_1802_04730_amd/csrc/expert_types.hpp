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
  typedef float v4 __attribute__((ext_vector_type(4)));  // 16 bytes
  static constexpr int PER16 = 4;
};
template <> struct Elem<bf16> {
  typedef bf16 v4 __attribute__((ext_vector_type(4)));
  typedef bf16 v8 __attribute__((ext_vector_type(8)));
  static constexpr int PER16 = 8;
};
template <> struct Elem<f16> {
  typedef f16 v4 __attribute__((ext_vector_type(4)));
  typedef f16 v8 __attribute__((ext_vector_type(8)));
  static constexpr int PER16 = 8;
};

// 16 bytes whose elements alone are aligned: one load or store all the same (global memory).
template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) Any16 {
  T e[16 / sizeof(T)];
};

template <typename T>
__device__ __forceinline__ Any16<T> load16(const T* p) {
  return *reinterpret_cast<const Any16<T>*>(p);
}
template <typename T>
__device__ __forceinline__ void store16(T* p, const Any16<T>& v) {
  *reinterpret_cast<Any16<T>*>(p) = v;
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
