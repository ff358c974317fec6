// The weighted sum of a token's k expert rows, and its gradient.
//   O(t,n)               = sum_i w(t,i) * Y(Place(t,i), n)
//   dY(Place(t,i), n)    = w(t,i) * dO(t,n)
//   dw(t,i)              = sum_n dO(t,n) * Y(Place(t,i), n)
// Both only move bytes: every row of Y is read once, 16 bytes a lane, all k of a token in flight together.  A slot without a place (-1) takes
// no part.  The gradient gives a token to one wavefront, which reads its row of dO once for all slots (for 8 of them at
// a time) and sums dw over its lanes in a fixed order.  Measured at 8192 tokens, 4 rows of 2048 bfloat16: 30 us (5.6 TB/s) and,
// behind it, 54 us (5.6 TB/s; by itself, with nothing of Y in the caches, 71); with a branch around each slot's load 60 and 52, with stores through the caches 42 and 52.
#pragma once
#include <type_traits>

#include "expert_types.hpp"

namespace tc355 {

struct ExpertSumArgs {
  const void* Y;     // [R][N]
  const float* Wt;   // [T][k] or nullptr: ones
  const int* Place;  // [T][k]
  void* O;           // [T][N]
  long long T, R;
  int N, k, lpr, cols;
};

template <typename T, int V, int SLOTS>
__global__ __launch_bounds__(WG_THREADS) void expert_sum_kernel(ExpertSumArgs p, int64_t first) {
  typedef typename Wide<T>::type S;
  const int64_t g = ((first + blockIdx.x) * WG_THREADS + threadIdx.x) / p.lpr;
  const int64_t t = g / p.cols;
  const RowUnit<V> u((g % p.cols) * p.lpr + (threadIdx.x & (p.lpr - 1)), p.N);
  if (t >= p.T || !u.on) return;
  S acc[V];
#pragma unroll
  for (int i = 0; i < V; i++) acc[i] = 0;
  for (int i0 = 0; i0 < p.k && p.R; i0 += SLOTS) {
    int64_t at[SLOTS];
    float w[SLOTS];
    bool on[SLOTS];
#pragma unroll
    for (int j = 0; j < SLOTS; j++) {
      const int i = min(i0 + j, p.k - 1), r = p.Place[t * p.k + i];
      w[j] = p.Wt ? p.Wt[t * p.k + i] : 1.0f;
      on[j] = i0 + j < p.k && r >= 0 && r < p.R;
      at[j] = on[j] ? (int64_t)r * p.N : 0;
    }
    Pack<T, V> v[SLOTS];  // (a slot that takes no part reads the first row: branches would make each load wait for the one before)
#pragma unroll
    for (int j = 0; j < SLOTS; j++) v[j] = load_unit<T, V>(static_cast<const T*>(p.Y) + at[j], u);
#pragma unroll
    for (int j = 0; j < SLOTS; j++)
#pragma unroll
      for (int i = 0; i < V; i++) acc[i] = on[j] ? acc[i] + (S)w[j] * (S)v[j].e[i] : acc[i];
  }
  Pack<T, V> o;
#pragma unroll
  for (int i = 0; i < V; i++) o.e[i] = narrow<T>(acc[i]);
  store_unit<T, V>(static_cast<T*>(p.O) + t * p.N, u, o);
}

struct ExpertSumGradArgs {
  const void* dO;    // [T][N]
  const void* Y;     // [R][N]
  const float* Wt;   // [T][k]
  const int* Place;  // [T][k]
  void* dY;          // [R][N]
  float* dWt;        // [T][k]
  long long T, R;
  int N, k;
};

template <typename T, int V, int SLOTS>
__global__ __launch_bounds__(WG_THREADS) void expert_sum_grad_kernel(ExpertSumGradArgs p, int64_t first) {
  typedef typename Wide<T>::type S;
  const int lane = threadIdx.x & 63;
  const int64_t t = (first + blockIdx.x) * WAVES_PER_WG + (threadIdx.x >> 6);
  if (t >= p.T) return;
  const T* dO = static_cast<const T*>(p.dO) + t * p.N;
  if (p.R == 0) {
    for (int i = lane; i < p.k; i += 64) p.dWt[t * p.k + i] = 0.0f;
    return;
  }
  for (int i0 = 0; i0 < p.k; i0 += SLOTS) {
    long long at[SLOTS];
    float w[SLOTS];
    S dw[SLOTS];
#pragma unroll
    for (int j = 0; j < SLOTS; j++) {
      at[j] = i0 + j < p.k ? p.Place[t * p.k + i0 + j] : -1;
      if (at[j] >= p.R) at[j] = -1;
      w[j] = i0 + j < p.k ? p.Wt[t * p.k + i0 + j] : 0.0f;
      dw[j] = 0;
    }
    const auto columns = [&](const RowUnit<V>& u, auto whole) {
      const Pack<T, V> d = load_unit<T, V>(dO, u);
      Pack<T, V> y[SLOTS];
#pragma unroll
      for (int j = 0; j < SLOTS; j++)
        if (at[j] >= 0) y[j] = load_unit<T, V>(static_cast<const T*>(p.Y) + at[j] * p.N, u);
#pragma unroll
      for (int j = 0; j < SLOTS; j++)
        if (at[j] >= 0) {
          Pack<T, V> o;
#pragma unroll
          for (int i = 0; i < V; i++) {
            if (whole.value || i >= u.skip) dw[j] += (S)d.e[i] * (S)y[j].e[i];
            o.e[i] = narrow<T>((S)w[j] * (S)d.e[i]);
          }
          T* out = static_cast<T*>(p.dY) + at[j] * p.N;
          if constexpr (whole.value) store_pack<T, V>(out + u.c, o);
          else store_unit<T, V>(out, u, o);
        }
    };
    for (int64_t x = lane; x * V < p.N; x += 64) {
      const RowUnit<V> u(x, p.N);
      if (u.skip == 0) columns(u, std::true_type{});
      else columns(u, std::false_type{});
    }
#pragma unroll
    for (int j = 0; j < SLOTS; j++)
#pragma unroll
      for (int d = 32; d; d /= 2) dw[j] += __shfl_xor(dw[j], d);
#pragma unroll
    for (int j = 0; j < SLOTS; j++)
      if (lane == j && i0 + j < p.k) p.dWt[t * p.k + i0 + j] = (float)dw[j];
  }
}

}  // namespace tc355
