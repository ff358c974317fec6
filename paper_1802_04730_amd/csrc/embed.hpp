// Rows of a token table and their gradient.
//   O(t,j)    = s * LUT(Idx(t), j)
//   dLUT(e,j) (+)= s * sum over the t with Idx(t) = e of dO(t,j)
// Both only move bytes.  A group of lanes takes 16 bytes each of a row; rows of any width start at any multiple of an element.
//
// The gradient walks the tokens sorted by number (key_sort.hpp): a row's tokens are a run of the sorted list, found by bisection, and
// are added in their own order, by one lane per element: no atomics, the same sum each time.  Language has words that make up a
// large part of a batch, so a run is cut at the multiples of EMBED_RUN: a kernel of its own sums every whole stretch of
// EMBED_RUN places that belongs to one number, and a row adds its ends and those sums.  Rows of numbers that do not occur are written with zeros, or left
// alone where the gradient is added to what is there.
#pragma once
#include "expert_types.hpp"

namespace tc355 {

constexpr int EMBED_RUN = 32;

struct EmbedArgs {
  const void* LUT;
  const int* Idx;
  void* O;
  long long E, T;
  int D, lpr, cols;  // lanes of a row's group: a power of two <= 64; groups of a row
  float scale;
};

template <typename T>
__global__ __launch_bounds__(WG_THREADS) void embed_kernel(EmbedArgs p, int64_t first) {
  constexpr int V = Elem<T>::PER16;
  const int64_t g = ((first + blockIdx.x) * WG_THREADS + threadIdx.x) / p.lpr;
  const int64_t t = g / p.cols;
  if (t >= p.T) return;
  const int c = ((int)(g % p.cols) * p.lpr + (threadIdx.x & (p.lpr - 1))) * V;
  if (c >= p.D) return;
  const long long e = p.Idx[t];
  const bool ok = e >= 0 && e < p.E;
  const T* src = static_cast<const T*>(p.LUT) + (ok ? e : 0) * p.D + c;
  T* out = static_cast<T*>(p.O) + t * p.D + c;
  typedef typename Wide<T>::type S;
  if (c + V <= p.D) {
    const Any16<T> v = load16(src);
    Any16<T> o;
#pragma unroll
    for (int i = 0; i < V; i++) o.e[i] = narrow<T>(ok ? (S)v.e[i] * (S)p.scale : (S)__builtin_nanf(""));
    store16(out, o);
  } else {
    for (int i = 0; c + i < p.D; i++) out[i] = narrow<T>(ok ? (S)src[i] * (S)p.scale : (S)__builtin_nanf(""));
  }
}

struct EmbedGradArgs {
  const void* dO;
  void* dLUT;
  void* part;        // [stretches][D], of the wide type
  const int* key;    // sorted numbers; E: of no row
  const int* order;  // the tokens in that order
  int T, E, D, lpr, cols, rows;  // rows of a workgroup
  float scale;
  int add;
};

// acc += the V columns from c on of the rows `order[lo .. hi)`, of which `left` are there
template <typename T, typename S, int V>
__device__ __forceinline__ void embed_add_rows(const EmbedGradArgs& p, int lo, int hi, int c, bool whole, S (&acc)[V]) {
  constexpr int NB = 8;  // rows in flight
  const T* dO = static_cast<const T*>(p.dO) + c;
  for (int r = lo; r < hi; r += NB) {
    int t[NB];
#pragma unroll
    for (int j = 0; j < NB; j++) t[j] = r + j < hi ? p.order[r + j] : 0;
    if (whole) {
      Any16<T> v[NB];
#pragma unroll
      for (int j = 0; j < NB; j++)
        if (r + j < hi) v[j] = load16(dO + (int64_t)t[j] * p.D);
#pragma unroll
      for (int j = 0; j < NB; j++)
        if (r + j < hi) {
#pragma unroll
          for (int i = 0; i < V; i++) acc[i] += (S)v[j].e[i];
        }
    } else {
#pragma unroll
      for (int j = 0; j < NB; j++)
        if (r + j < hi) {
#pragma unroll
          for (int i = 0; i < V; i++)
            if (c + i < p.D) acc[i] += (S)dO[(int64_t)t[j] * p.D + i];
        }
    }
  }
}

// Sums of the whole stretches of EMBED_RUN places that belong to one number.
template <typename T>
__global__ __launch_bounds__(WG_THREADS) void embed_stretch_kernel(EmbedGradArgs p, int stretches) {
  constexpr int V = Elem<T>::PER16;
  typedef typename Wide<T>::type S;
  const int64_t g = ((int64_t)blockIdx.x * WG_THREADS + threadIdx.x) / p.lpr;
  const int64_t s = g / p.cols;
  if (s >= stretches) return;
  const int lo = (int)s * EMBED_RUN, k = p.key[lo];
  if (k != p.key[lo + EMBED_RUN - 1] || k >= p.E) return;
  const int c = ((int)(g % p.cols) * p.lpr + (threadIdx.x & (p.lpr - 1))) * V;
  if (c >= p.D) return;
  const bool whole = c + V <= p.D;
  S acc[V];
#pragma unroll
  for (int i = 0; i < V; i++) acc[i] = 0;
  embed_add_rows<T, S, V>(p, lo, lo + EMBED_RUN, c, whole, acc);
  S* out = static_cast<S*>(p.part) + s * p.D + c;
#pragma unroll
  for (int i = 0; i < V; i++)
    if (whole || c + i < p.D) out[i] = acc[i];
}

template <typename T, typename TO>
__global__ __launch_bounds__(WG_THREADS) void embed_grad_kernel(EmbedGradArgs p) {
  constexpr int V = Elem<T>::PER16, MOST = 64;
  typedef typename Wide<T>::type S;
  __shared__ int begin[MOST + 1];
  const int64_t e0 = (int64_t)blockIdx.x * p.rows;
  if ((int)threadIdx.x <= p.rows) {  // the first place of a number >= e
    const int64_t e = e0 + threadIdx.x;
    int lo = 0, hi = p.T;
    while (lo < hi) {
      const int mid = (int)(((unsigned)lo + (unsigned)hi) >> 1);
      if (p.key[mid] < e) lo = mid + 1;
      else hi = mid;
    }
    begin[threadIdx.x] = lo;
  }
  __syncthreads();
  const int groups = WG_THREADS / p.lpr, lane = threadIdx.x & (p.lpr - 1);
  for (int u = threadIdx.x / p.lpr; u < p.rows * p.cols; u += groups) {
    const int x = u / p.cols;
    const int64_t e = e0 + x;
    const int c = ((u % p.cols) * p.lpr + lane) * V;
    if (e >= p.E || c >= p.D) continue;
    const int lo = begin[x], hi = begin[x + 1];
    if (p.add && lo == hi) continue;
    const bool whole = c + V <= p.D;
    S acc[V];
#pragma unroll
    for (int i = 0; i < V; i++) acc[i] = 0;
    const int s0 = (lo + EMBED_RUN - 1) / EMBED_RUN, s1 = hi / EMBED_RUN;  // whole stretches
    if (s0 < s1) {
      embed_add_rows<T, S, V>(p, lo, s0 * EMBED_RUN, c, whole, acc);
      const S* part = static_cast<const S*>(p.part) + c;
#pragma unroll 4
      for (int s = s0; s < s1; s++)
#pragma unroll
        for (int i = 0; i < V; i++)
          if (whole || c + i < p.D) acc[i] += part[(int64_t)s * p.D + i];
      embed_add_rows<T, S, V>(p, s1 * EMBED_RUN, hi, c, whole, acc);
    } else {
      embed_add_rows<T, S, V>(p, lo, hi, c, whole, acc);
    }
    TO* out = static_cast<TO*>(p.dLUT) + e * p.D + c;
    constexpr int W = Elem<TO>::PER16;
    if (whole && V % W == 0) {
#pragma unroll
      for (int h = 0; h < V / W; h++) {
        Any16<TO> o;
        if (p.add) o = load16(out + h * W);
#pragma unroll
        for (int i = 0; i < W; i++) o.e[i] = narrow<TO>(p.add ? acc[h * W + i] * (S)p.scale + (S)o.e[i] : acc[h * W + i] * (S)p.scale);
        store16(out + h * W, o);
      }
    } else {
#pragma unroll
      for (int i = 0; i < V; i++)
        if (c + i < p.D) out[i] = narrow<TO>(p.add ? acc[i] * (S)p.scale + (S)out[i] : acc[i] * (S)p.scale);
    }
  }
}

}  // namespace tc355
