// Rows and weights in 8 bits (e4m3: 3 bits of mantissa, largest value 448) with a scale for each block of 128 elements of a row, or of 128 x 128 of a matrix.
//   S = the smallest power of two with max |block| / S <= 448, at least 2^-126;   Q = X / S, to the nearest, ties to even
// S is kept as a byte, S = 2^(byte - 127) (e8m0).  A block that holds an Inf or a NaN has the byte 255 and values of NaN: it stands for NaN.
//
// A power of two, since dividing by it rounds nothing: e4m3 has an exponent of its own, so that a finer scale would gain no bits, only up to one binade at the lower end
// of its 18; what an element stands for does not hang on how a scale was rounded; and the matrix core applies such bytes by itself.
// The byte from the bits of the largest magnitude: 448 = 1.75 * 2^8, so exponent - 8, and one more where the mantissa is above 1.75 -- which adding 0x1fffff carries.
//
// Bounded by memory: each element is read once and written once as a byte (twice with the transposed form, whose values and scales are the same, since
// a block's are: a block goes through LDS once, and leaves by whole lines both ways).  Measured, bfloat16: weights of 32 x 2048 x 4096 both ways 190 us (5.6 TB/s), 16384 rows of 4096
// 37.5 (5.4), 16 rows 3.5.
#pragma once
#include "expert_types.hpp"
#include "lanes.hpp"

namespace tc355 {

constexpr int Q8_BLOCK = 128;
constexpr unsigned Q8_NAN = 255;  // scale of a block that stands for NaN

// The scale's byte from the bits of the largest magnitude.
__device__ __forceinline__ unsigned q8_scale(unsigned most) {
  if (most >= 0x7f800000u) return Q8_NAN;
  const int byte = (int)((most + 0x1fffffu) >> 23) - 8;
  return byte < 1 ? 1u : (unsigned)byte;
}
template <typename T>
__device__ __forceinline__ unsigned q8_magnitude(T x) {
  return __builtin_bit_cast(unsigned, static_cast<float>(x)) & 0x7fffffffu;
}
// Four values over the scale, as bytes.
__device__ __forceinline__ unsigned q8_bytes(float a, float b, float c, float d, unsigned scale) {
  if (scale == Q8_NAN) return 0x7f7f7f7fu;
  const float s = __builtin_bit_cast(float, (254u - scale) << 23);
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a * s, b * s, 0, false);
  return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c * s, d * s, r, true);
}
typedef unsigned u2 __attribute__((ext_vector_type(2)));
template <typename T>
__device__ __forceinline__ u2 q8_bytes8(const Pack<T, 8>& x, unsigned scale) {
  const auto f = [&](int i) { return static_cast<float>(x.e[i]); };
  return u2{q8_bytes(f(0), f(1), f(2), f(3), scale), q8_bytes(f(4), f(5), f(6), f(7), scale)};
}

// Eight neighbours of a row of `width` elements from column c on, zeros past its end.
template <typename T>
__device__ __forceinline__ Pack<T, 8> q8_load(const T* row, int c, int width) {
  if (c + 8 <= width) return load_pack<T, 8>(row + c);
  Pack<T, 8> x;
#pragma unroll
  for (int i = 0; i < 8; i++) x.e[i] = c + i < width ? row[c + i] : static_cast<T>(0.0f);
  return x;
}

struct QuantizeRowsArgs {
  const void* X;           // [R][K]
  unsigned char* Q;        // [R][blocks * 128]
  unsigned char* S;        // [R][blocks]
  long long all;           // R * blocks
  int K, blocks;
};

// 16 lanes a block; U blocks of a thread requested together.
template <typename T, int U>
__global__ __launch_bounds__(WG_THREADS) void quantize_rows_kernel(QuantizeRowsArgs p, int64_t first) {
  const int lane = threadIdx.x & 15;
  const int64_t b0 = (first + blockIdx.x) * (WG_THREADS / 16 * U) + threadIdx.x / 16;
  Pack<T, 8> x[U];
#pragma unroll
  for (int u = 0; u < U; u++) {
    const int64_t b = min(b0 + u * (WG_THREADS / 16), p.all - 1), r = b / p.blocks;
    x[u] = q8_load(static_cast<const T*>(p.X) + r * p.K, (int)(b - r * p.blocks) * Q8_BLOCK + 8 * lane, p.K);
  }
#pragma unroll
  for (int u = 0; u < U; u++) {
    const int64_t b = b0 + u * (WG_THREADS / 16);
    if (b >= p.all) return;  // (all 16 lanes)
    unsigned most = 0;
#pragma unroll
    for (int i = 0; i < 8; i++) most = larger(most, q8_magnitude(x[u].e[i]));
    const unsigned s = q8_scale(group_all<16>(most, larger));
    *reinterpret_cast<u2*>(p.Q + b * Q8_BLOCK + 8 * lane) = q8_bytes8(x[u], s);
    if (lane == 0) p.S[b] = (unsigned char)s;
  }
}

struct QuantizeWeightsArgs {
  const void* W;      // [E][N][K]
  unsigned char* Q;   // [E][N][kb * 128]
  unsigned char* S;   // [E][nb][kb]
  unsigned char* Qt;  // [E][K][nb * 128] or nullptr
  unsigned char* St;  // [E][kb][nb]
  long long E;
  int N, K, nb, kb;
};

// A block of 128 x 128 a workgroup: 16 lanes a row, 16 rows at a time.
template <typename T>
__global__ __launch_bounds__(WG_THREADS) void quantize_weights_kernel(QuantizeWeightsArgs p, int64_t first) {
  __shared__ __align__(16) unsigned bytes[Q8_BLOCK * Q8_BLOCK / 4 + 7 * 8];  // row r at 32 r + 8 (r / 16): the 16 rows of a thread's column miss the others' banks
  __shared__ unsigned part[WAVES_PER_WG];
  const int64_t at = first + blockIdx.x;
  const int64_t e = at / ((int64_t)p.nb * p.kb);
  const int in = (int)(at - e * p.nb * p.kb), n0 = in / p.kb * Q8_BLOCK, k0 = in % p.kb * Q8_BLOCK;
  const int tid = threadIdx.x, lane = tid & 15, row = tid >> 4;
  const T* W = static_cast<const T*>(p.W) + (e * p.N + n0) * p.K;
  Pack<T, 8> x[8];
  unsigned most = 0;
#pragma unroll
  for (int j = 0; j < 8; j++) {
    const int r = 16 * j + row;
    x[j] = Pack<T, 8>{};
    if (n0 + r < p.N) x[j] = q8_load(W + (int64_t)r * p.K, k0 + 8 * lane, p.K);
  }
#pragma unroll
  for (int j = 0; j < 8; j++)
#pragma unroll
    for (int i = 0; i < 8; i++) most = larger(most, q8_magnitude(x[j].e[i]));
  most = group_all<64>(most, larger);
  if ((tid & 63) == 0) part[tid >> 6] = most;
  __syncthreads();
  const unsigned s = q8_scale(larger(larger(part[0], part[1]), larger(part[2], part[3])));
  if (tid == 0) {
    p.S[at] = (unsigned char)s;
    if (p.Qt) p.St[(e * p.kb + k0 / Q8_BLOCK) * p.nb + n0 / Q8_BLOCK] = (unsigned char)s;
  }
  unsigned char* const Q = p.Q + (e * p.N + n0) * ((int64_t)p.kb * Q8_BLOCK) + k0 + 8 * lane;
#pragma unroll
  for (int j = 0; j < 8; j++) {
    const int r = 16 * j + row;
    const u2 v = q8_bytes8(x[j], s);
    if (n0 + r < p.N) __builtin_nontemporal_store(v, reinterpret_cast<u2*>(Q + (int64_t)r * p.kb * Q8_BLOCK));
    if (p.Qt) *reinterpret_cast<u2*>(bytes + 32 * r + 8 * j + 2 * lane) = v;
  }
  if (!p.Qt) return;
  __syncthreads();
  // 16 rows by 4 columns a thread: eight threads write 128 bytes of a row of the transposed form
  const int rows = tid & 7, cols = tid >> 3;
  unsigned d[16];
#pragma unroll
  for (int j = 0; j < 16; j++) d[j] = bytes[32 * (16 * rows + j) + 8 * rows + cols];
  unsigned char* const Qt = p.Qt + (e * p.K + k0 + 4 * cols) * ((int64_t)p.nb * Q8_BLOCK) + n0 + 16 * rows;
#pragma unroll
  for (int c = 0; c < 4; c++) {
    u4 o;
#pragma unroll
    for (int w = 0; w < 4; w++) {  // byte c of four rows
      const unsigned lo = __builtin_amdgcn_perm(d[4 * w + 1], d[4 * w], (unsigned)((4 + c) << 8 | c)), hi = __builtin_amdgcn_perm(d[4 * w + 3], d[4 * w + 2], (unsigned)((4 + c) << 8 | c));
      o[w] = (lo & 0xffffu) | hi << 16;
    }
    if (k0 + 4 * cols + c < p.K) __builtin_nontemporal_store(o, reinterpret_cast<u4*>(Qt + (int64_t)c * p.nb * Q8_BLOCK));
  }
}

}  // namespace tc355
