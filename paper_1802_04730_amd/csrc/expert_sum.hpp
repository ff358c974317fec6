// The weighted sum of a token's k expert rows, and its gradient.
//   O(t,n)               = sum_i w(t,i) * Y(Place(t,i), n)
//   dY(Place(t,i), n)    = w(t,i) * dO(t,n)
//   dw(t,i)              = sum_n dO(t,n) * Y(Place(t,i), n)
// Both only move bytes: every row of Y is read once, 16 bytes a lane, all k of a token in flight together.  A slot without a place (-1) takes
// no part.  The gradient gives a token to one wavefront, which reads its row of dO once for all slots (for 8 of them at
// a time) and sums dw over its lanes in a fixed order.
#pragma once
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

constexpr int ESUM_SLOTS = 8;

template <typename T>
__global__ __launch_bounds__(WG_THREADS) void expert_sum_kernel(ExpertSumArgs p) {
  constexpr int V = Elem<T>::PER16;
  typedef typename Wide<T>::type S;
  const int64_t g = ((int64_t)blockIdx.x * WG_THREADS + threadIdx.x) / p.lpr;
  const int64_t t = g / p.cols;
  if (t >= p.T) return;
  const int c = ((int)(g % p.cols) * p.lpr + (threadIdx.x & (p.lpr - 1))) * V;
  if (c >= p.N) return;
  const bool whole = c + V <= p.N;
  const T* Y = static_cast<const T*>(p.Y) + c;
  S acc[V];
#pragma unroll
  for (int i = 0; i < V; i++) acc[i] = 0;
  for (int i0 = 0; i0 < p.k; i0 += ESUM_SLOTS) {
    long long at[ESUM_SLOTS];
    float w[ESUM_SLOTS];
#pragma unroll
    for (int j = 0; j < ESUM_SLOTS; j++) {
      at[j] = i0 + j < p.k ? p.Place[t * p.k + i0 + j] : -1;
      w[j] = i0 + j < p.k && p.Wt ? p.Wt[t * p.k + i0 + j] : 1.0f;
    }
    Any16<T> v[ESUM_SLOTS];
    if (whole) {
#pragma unroll
      for (int j = 0; j < ESUM_SLOTS; j++)
        if (at[j] >= 0 && at[j] < p.R) v[j] = load16(Y + at[j] * p.N);
    }
#pragma unroll
    for (int j = 0; j < ESUM_SLOTS; j++)
      if (at[j] >= 0 && at[j] < p.R) {
#pragma unroll
        for (int i = 0; i < V; i++)
          if (whole || c + i < p.N) acc[i] += (S)w[j] * (S)(whole ? v[j].e[i] : Y[at[j] * p.N + i]);
      }
  }
  T* out = static_cast<T*>(p.O) + t * p.N + c;
  if (whole) {
    Any16<T> o;
#pragma unroll
    for (int i = 0; i < V; i++) o.e[i] = narrow<T>(acc[i]);
    store16(out, o);
  } else {
    for (int i = 0; c + i < p.N; i++) out[i] = narrow<T>(acc[i]);
  }
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

template <typename T, int SLOTS>
__global__ __launch_bounds__(WG_THREADS) void expert_sum_grad_kernel(ExpertSumGradArgs p) {
  constexpr int V = Elem<T>::PER16;
  typedef typename Wide<T>::type S;
  const int lane = threadIdx.x & 63;
  const int64_t t = (int64_t)blockIdx.x * WAVES_PER_WG + (threadIdx.x >> 6);
  if (t >= p.T) return;
  const T* dO = static_cast<const T*>(p.dO) + t * p.N;
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
    for (int c = lane * V; c < p.N; c += 64 * V) {
      if (c + V <= p.N) {
        const Any16<T> d = load16(dO + c);
        Any16<T> y[SLOTS];
#pragma unroll
        for (int j = 0; j < SLOTS; j++)
          if (at[j] >= 0) y[j] = load16(static_cast<const T*>(p.Y) + at[j] * p.N + c);
#pragma unroll
        for (int j = 0; j < SLOTS; j++)
          if (at[j] >= 0) {
            Any16<T> o;
#pragma unroll
            for (int i = 0; i < V; i++) {
              dw[j] += (S)d.e[i] * (S)y[j].e[i];
              o.e[i] = narrow<T>((S)w[j] * (S)d.e[i]);
            }
            store16(static_cast<T*>(p.dY) + at[j] * p.N + c, o);
          }
      } else {
        for (int i = 0; c + i < p.N; i++) {
          const S d = (S)dO[c + i];
#pragma unroll
          for (int j = 0; j < SLOTS; j++)
            if (at[j] >= 0) {
              dw[j] += d * (S)static_cast<const T*>(p.Y)[at[j] * p.N + c + i];
              static_cast<T*>(p.dY)[at[j] * p.N + c + i] = narrow<T>((S)w[j] * d);
            }
        }
      }
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
