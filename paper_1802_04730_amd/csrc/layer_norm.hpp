// Layer norm of the rows of a matrix, and its gradient.
//   m = sum_n X(t,n) / N,  s = sqrt(sum_n (X(t,n) - m)^2 / N + eps),  y = (X - m) / s
//   O(t,n)  = y(t,n) W(n) + B(n)
//   dX(t,n) = (h - sum_n h / N - y sum_n (h y) / N) / s,  h = dO W
//   dW(n) (+)= sum_t dO(t,n) y(t,n),  dB(n) (+)= sum_t dO(t,n)
// What bounds them: the rows' bytes, each read once and written once; for a handful of rows the launch and one chain of a load and three sums over lanes.
//
// G lanes (16, 64 or a whole workgroup) hold a row in registers, so that the mean is known before the squares of the differences to it are
// summed: no cancellation, whatever the mean.  Groups of lanes go through the rows at a stride, with W and B, or the sums for dW and dB, in
// registers all the while and the next row requested before this one is summed.  The gradient takes m and s from X again: it has to
// read X anyway.  Sums over the rows: each workgroup's own, in its order of the rows, are joined in the workgroups' order by a second launch; no
// atomics.  Rows too long for registers (norm_long_*) are read once for each sum; their dW and dB come from a pass down the columns.
//
// Sums are in 32 bits for 16-bit storage and in 64 for float storage, as everywhere where rows are only streamed; along rows too long for registers in 64, since a lane adds up to
// 2^18 elements of one: in 32 bits, squares of one size would be off by parts in 2^8.
//
// Measured: 16384 rows of 4096 bfloat16, weights in float, 51-53 us (5.1-5.2 TB/s) forward, 87-92 for the gradient (4.6) and 6.5 for its join; 8 rows of 2048 4.2; 1500 rows of 333 floats
// 3.8, 7.9 and 4.5 (16 rows a part, four a group of lanes: 10.5 and 3).  Widths of four units a lane, 16384 rows of bfloat16: 2048 30 forward and 77 for gradient and join (2.6 TB/s), 5120 65 and 166 (3.0), 8192 97 and 193 (4.2): the
// gradient's sums take 270 registers there, one wavefront a SIMD.  Beyond registers: 8192 rows of 8192 floats 158 (3.4 TB/s, each row read three times, mostly from cache) and 399 (2.0), of 12288 bfloat16 161 and 409.
#pragma once
#include "expert_types.hpp"
#include "lanes.hpp"

namespace tc355 {

struct NormArgs {
  const void* X;   // [T][N]
  const void* W;   // [N]
  const void* B;   // [N] or nullptr
  void* O;         // [T][N]
  const void* dO;  // [T][N]
  void* dX;        // [T][N]
  void* part;      // [parts][2][N]: sums for dW and dB; nullptr: none are asked for
  void* stat;      // [T][2] of long rows: m and 1/s; nullptr: not kept
  long long T;
  int N;
  float eps;
};

__device__ __forceinline__ float norm_inverse(float v) { return 1.0f / sqrtf(v); }
__device__ __forceinline__ double norm_inverse(double v) { return 1.0 / sqrt(v); }

// Sum over the G lanes of a row, in all of them.  lds: 2 x 4 values that a whole workgroup's sums go through, `turn` which four.
template <int G, typename S>
__device__ __forceinline__ S norm_sum(S x, S* lds, int& turn) {
  x = group_all<(G < 64 ? G : 64)>(x, [](S a, S b) { return a + b; });
  if constexpr (G > 64) {
    S* at = lds + 4 * turn;
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = x;
    __syncthreads();
    x = (at[0] + at[1]) + (at[2] + at[3]);
  }
  return x;
}

template <typename S, typename T, int V>
__device__ __forceinline__ void norm_widen(const Pack<T, V>& p, S (&x)[V]) {
#pragma unroll
  for (int i = 0; i < V; i++) x[i] = (S)p.e[i];
}

// A row's mean and 1/s from its columns in registers; x becomes x - m.  Columns that the unit does not own count for nothing.
template <int G, int V, int C, typename S>
__device__ __forceinline__ S norm_centre(S (&x)[C][V], const RowUnit<V> (&u)[C], int N, S eps, S* lds, int& turn) {
  S sum = 0;
#pragma unroll
  for (int c = 0; c < C; c++)
#pragma unroll
    for (int i = 0; i < V; i++) sum += u[c].on && i >= u[c].skip ? x[c][i] : (S)0;
  const S m = norm_sum<G>(sum, lds, turn) / (S)N;
  S square = 0;
#pragma unroll
  for (int c = 0; c < C; c++)
#pragma unroll
    for (int i = 0; i < V; i++) {
      x[c][i] -= m;
      square += u[c].on && i >= u[c].skip ? x[c][i] * x[c][i] : (S)0;
    }
  return norm_inverse(norm_sum<G>(square, lds, turn) / (S)N + eps);
}

template <typename T, typename TW, int V, int G, int C>
__global__ __launch_bounds__(WG_THREADS) void norm_rows_kernel(NormArgs p) {
  typedef typename Wide<T>::type S;
  __shared__ S lds[8];
  int turn = 0;
  const int lane = threadIdx.x % G;
  const int64_t step = (int64_t)gridDim.x * (WG_THREADS / G);
  int64_t t = (int64_t)blockIdx.x * (WG_THREADS / G) + threadIdx.x / G;
  if (G < WG_THREADS && t >= p.T) return;
  RowUnit<V> u[C];
  float w[C][V], b[C][V];
  Pack<T, V> next[C];
#pragma unroll
  for (int c = 0; c < C; c++) {
    u[c] = RowUnit<V>(c * G + lane, p.N);
    next[c] = load_unit<T, V>(static_cast<const T*>(p.X) + t * p.N, u[c]);
  }
#pragma unroll
  for (int c = 0; c < C; c++) {
    norm_widen(load_unit<TW, V>(static_cast<const TW*>(p.W), u[c]), w[c]);
#pragma unroll
    for (int i = 0; i < V; i++) b[c][i] = 0.0f;
    if (p.B) norm_widen(load_unit<TW, V>(static_cast<const TW*>(p.B), u[c]), b[c]);
  }
  for (; t < p.T; t += step) {
    S x[C][V];
    const int64_t then = t + step < p.T ? t + step : t;
#pragma unroll
    for (int c = 0; c < C; c++) {
      norm_widen(next[c], x[c]);
      next[c] = load_unit<T, V>(static_cast<const T*>(p.X) + then * p.N, u[c]);
    }
    const S r = norm_centre<G>(x, u, p.N, (S)p.eps, lds, turn);
#pragma unroll
    for (int c = 0; c < C; c++) {
      Pack<T, V> o;
#pragma unroll
      for (int i = 0; i < V; i++) o.e[i] = narrow<T>(x[c][i] * r * (S)w[c][i] + (S)b[c][i]);
      if (u[c].on) store_unit<T, V>(static_cast<T*>(p.O) + t * p.N, u[c], o);
    }
  }
}

template <typename T, typename TW, int V, int G, int C>
__global__ __launch_bounds__(WG_THREADS) void norm_rows_grad_kernel(NormArgs p) {
  typedef typename Wide<T>::type S;
  constexpr int SLOTS = WG_THREADS / G;  // rows of a workgroup at a time
  __shared__ S lds[8];
  extern __shared__ __align__(16) char more[];  // [2][N] of S where several rows share a workgroup
  int turn = 0;
  const int lane = threadIdx.x % G, slot = threadIdx.x / G;
  const int64_t step = (int64_t)gridDim.x * SLOTS;
  RowUnit<V> u[C];
  float w[C][V];
  S dw[C][V], db[C][V];
  Pack<T, V> nx[C], nd[C];
  int64_t t = (int64_t)blockIdx.x * SLOTS + slot;
  const auto request = [&](int64_t row) {
#pragma unroll
    for (int c = 0; c < C; c++) {
      nx[c] = load_unit<T, V>(static_cast<const T*>(p.X) + row * p.N, u[c]);
      nd[c] = load_unit<T, V>(static_cast<const T*>(p.dO) + row * p.N, u[c]);
    }
  };
#pragma unroll
  for (int c = 0; c < C; c++) u[c] = RowUnit<V>(c * G + lane, p.N);
  request(t < p.T ? t : p.T - 1);
#pragma unroll
  for (int c = 0; c < C; c++) {
    norm_widen(load_unit<TW, V>(static_cast<const TW*>(p.W), u[c]), w[c]);
#pragma unroll
    for (int i = 0; i < V; i++) dw[c][i] = db[c][i] = 0;
  }
  for (; t < p.T; t += step) {
    S x[C][V];
    Pack<T, V> d[C];
#pragma unroll
    for (int c = 0; c < C; c++) {
      norm_widen(nx[c], x[c]);
      d[c] = nd[c];
    }
    request(t + step < p.T ? t + step : t);
    const S r = norm_centre<G>(x, u, p.N, (S)p.eps, lds, turn);
    S first = 0, second = 0;
#pragma unroll
    for (int c = 0; c < C; c++)
#pragma unroll
      for (int i = 0; i < V; i++) {
        x[c][i] *= r;  // (y)
        const S g = (S)d[c].e[i], h = g * (S)w[c][i];
        const bool mine = u[c].on && i >= u[c].skip;
        first += mine ? h : (S)0;
        second += mine ? h * x[c][i] : (S)0;
        dw[c][i] += g * x[c][i];
        db[c][i] += g;
      }
    first = norm_sum<G>(first, lds, turn) / (S)p.N;
    second = norm_sum<G>(second, lds, turn) / (S)p.N;
#pragma unroll
    for (int c = 0; c < C; c++) {
      Pack<T, V> o;
#pragma unroll
      for (int i = 0; i < V; i++) o.e[i] = narrow<T>(((S)d[c].e[i] * (S)w[c][i] - first - x[c][i] * second) * r);
      if (u[c].on) store_unit<T, V>(static_cast<T*>(p.dX) + t * p.N, u[c], o);
    }
  }
  if (!p.part) return;
  S* const part = static_cast<S*>(p.part) + (int64_t)blockIdx.x * 2 * p.N;
  if constexpr (SLOTS == 1) {
#pragma unroll
    for (int c = 0; c < C; c++)
#pragma unroll
      for (int i = 0; i < V; i++)
        if (u[c].on && i >= u[c].skip) {
          part[u[c].c + i] = dw[c][i];
          part[p.N + u[c].c + i] = db[c][i];
        }
  } else {  // the workgroup's rows, one slot after the other
    S* const sum = reinterpret_cast<S*>(more);
    for (int s = 0; s < SLOTS; s++) {
      if (slot == s) {
#pragma unroll
        for (int c = 0; c < C; c++)
#pragma unroll
          for (int i = 0; i < V; i++)
            if (u[c].on && i >= u[c].skip) {
              S* const a = sum + u[c].c + i;
              a[0] = s ? a[0] + dw[c][i] : dw[c][i];
              a[p.N] = s ? a[p.N] + db[c][i] : db[c][i];
            }
      }
      __syncthreads();
    }
    for (int j = threadIdx.x; j < 2 * p.N; j += WG_THREADS) part[j] = sum[j];
  }
}

// ---- rows that do not fit into registers ----------------------------------------------------------------------------------

// f(unit) for this thread's units of a row.
template <int V, typename F>
__device__ __forceinline__ void norm_units(int N, F f) {
  for (int64_t x = threadIdx.x; x * V < N; x += WG_THREADS) f(RowUnit<V>(x, N));
}
// (the neighbours of a unit are added in S, units in 64 bits)
template <typename T, int V, typename S>
__device__ __forceinline__ void norm_long_stats(const T* row, int N, S eps, double* lds, int& turn, S* mean, S* inverse) {
  double sum = 0;
  norm_units<V>(N, [&](const RowUnit<V>& u) {
    const Pack<T, V> x = load_unit<T, V>(row, u);
    S of = 0;
#pragma unroll
    for (int i = 0; i < V; i++) of += i >= u.skip ? (S)x.e[i] : (S)0;
    sum += of;
  });
  const S m = (S)(norm_sum<WG_THREADS>(sum, lds, turn) / N);
  double square = 0;
  norm_units<V>(N, [&](const RowUnit<V>& u) {
    const Pack<T, V> x = load_unit<T, V>(row, u);
    S of = 0;
#pragma unroll
    for (int i = 0; i < V; i++) of += i >= u.skip ? ((S)x.e[i] - m) * ((S)x.e[i] - m) : (S)0;
    square += of;
  });
  *mean = m;
  *inverse = norm_inverse((S)(norm_sum<WG_THREADS>(square, lds, turn) / N) + eps);
}

template <typename T, typename TW, int V>
__global__ __launch_bounds__(WG_THREADS) void norm_long_kernel(NormArgs p) {
  typedef typename Wide<T>::type S;
  __shared__ double lds[8];
  int turn = 0;
  for (int64_t t = blockIdx.x; t < p.T; t += gridDim.x) {
    const T* row = static_cast<const T*>(p.X) + t * p.N;
    S m, r;
    norm_long_stats<T, V>(row, p.N, (S)p.eps, lds, turn, &m, &r);
    norm_units<V>(p.N, [&](const RowUnit<V>& u) {
      const Pack<T, V> x = load_unit<T, V>(row, u);
      const Pack<TW, V> w = load_unit<TW, V>(static_cast<const TW*>(p.W), u);
      Pack<TW, V> b{};
      if (p.B) b = load_unit<TW, V>(static_cast<const TW*>(p.B), u);
      Pack<T, V> o;
#pragma unroll
      for (int i = 0; i < V; i++) o.e[i] = narrow<T>(((S)x.e[i] - m) * r * (S)(float)w.e[i] + (S)(float)b.e[i]);
      store_unit<T, V>(static_cast<T*>(p.O) + t * p.N, u, o);
    });
  }
}

template <typename T, typename TW, int V>
__global__ __launch_bounds__(WG_THREADS) void norm_long_grad_kernel(NormArgs p) {
  typedef typename Wide<T>::type S;
  __shared__ double lds[8];
  int turn = 0;
  for (int64_t t = blockIdx.x; t < p.T; t += gridDim.x) {
    const T *row = static_cast<const T*>(p.X) + t * p.N, *grad = static_cast<const T*>(p.dO) + t * p.N;
    S m, r;
    norm_long_stats<T, V>(row, p.N, (S)p.eps, lds, turn, &m, &r);
    if (p.stat && threadIdx.x == 0) {
      static_cast<S*>(p.stat)[2 * t] = m;
      static_cast<S*>(p.stat)[2 * t + 1] = r;
    }
    double firsts = 0, seconds = 0;
    norm_units<V>(p.N, [&](const RowUnit<V>& u) {
      const Pack<T, V> x = load_unit<T, V>(row, u), d = load_unit<T, V>(grad, u);
      const Pack<TW, V> w = load_unit<TW, V>(static_cast<const TW*>(p.W), u);
      S of = 0, with = 0;
#pragma unroll
      for (int i = 0; i < V; i++) {
        const S h = (S)d.e[i] * (S)(float)w.e[i];
        of += i >= u.skip ? h : (S)0;
        with += i >= u.skip ? h * (((S)x.e[i] - m) * r) : (S)0;
      }
      firsts += of;
      seconds += with;
    });
    const S first = (S)(norm_sum<WG_THREADS>(firsts, lds, turn) / p.N), second = (S)(norm_sum<WG_THREADS>(seconds, lds, turn) / p.N);
    norm_units<V>(p.N, [&](const RowUnit<V>& u) {
      const Pack<T, V> x = load_unit<T, V>(row, u), d = load_unit<T, V>(grad, u);
      const Pack<TW, V> w = load_unit<TW, V>(static_cast<const TW*>(p.W), u);
      Pack<T, V> o;
#pragma unroll
      for (int i = 0; i < V; i++) o.e[i] = narrow<T>(((S)d.e[i] * (S)(float)w.e[i] - first - ((S)x.e[i] - m) * r * second) * r);
      store_unit<T, V>(static_cast<T*>(p.dX) + t * p.N, u, o);
    });
  }
}

// The sums of long rows for dW and dB, down the columns: workgroup (x, y) takes 256 V columns of every gridDim.y-th row.
template <typename T, int V>
__global__ __launch_bounds__(WG_THREADS) void norm_columns_kernel(NormArgs p) {
  typedef typename Wide<T>::type S;
  const RowUnit<V> u((int64_t)blockIdx.x * WG_THREADS + threadIdx.x, p.N);
  if (!u.on) return;
  S dw[V], db[V];
#pragma unroll
  for (int i = 0; i < V; i++) dw[i] = db[i] = 0;
  for (int64_t t = blockIdx.y; t < p.T; t += gridDim.y) {
    const S m = static_cast<const S*>(p.stat)[2 * t], r = static_cast<const S*>(p.stat)[2 * t + 1];
    const Pack<T, V> x = load_unit<T, V>(static_cast<const T*>(p.X) + t * p.N, u), d = load_unit<T, V>(static_cast<const T*>(p.dO) + t * p.N, u);
#pragma unroll
    for (int i = 0; i < V; i++) {
      dw[i] += (S)d.e[i] * (((S)x.e[i] - m) * r);
      db[i] += (S)d.e[i];
    }
  }
  S* const part = static_cast<S*>(p.part) + (int64_t)blockIdx.y * 2 * p.N;
#pragma unroll
  for (int i = 0; i < V; i++)
    if (i >= u.skip) {
      part[u.c + i] = dw[i];
      part[p.N + u.c + i] = db[i];
    }
}

// dW and dB (+)= the sums of the parts: 16 columns a workgroup, 16 lanes beside each other in a row, 16 shares of the parts, joined in their order.
template <typename S, typename TW>
__global__ __launch_bounds__(WG_THREADS) void norm_join_kernel(const S* part, int parts, int N, void* dW, void* dB, int add) {
  __shared__ S sum[16][17];
  const int lane = threadIdx.x & 15, share = threadIdx.x >> 4;
  const int64_t j = (int64_t)blockIdx.x * 16 + lane, all = dB ? 2 * (int64_t)N : N;
  S v = 0;
  if (j < all) {
    int q = share;
    for (; q + 16 * 7 < parts; q += 16 * 8) {  // eight loads in flight
      S x[8];
#pragma unroll
      for (int i = 0; i < 8; i++) x[i] = part[(q + 16 * i) * 2 * (int64_t)N + j];
#pragma unroll
      for (int i = 0; i < 8; i++) v += x[i];
    }
    for (; q < parts; q += 16) v += part[q * 2 * (int64_t)N + j];
  }
  sum[share][lane] = v;
  __syncthreads();
  if (share || j >= all) return;
#pragma unroll
  for (int s = 1; s < 16; s++) v += sum[s][lane];
  TW* const o = j < N ? static_cast<TW*>(dW) + j : static_cast<TW*>(dB) + (j - N);
  if (add) v += (S)(float)*o;
  *o = narrow<TW>(v);
}

}  // namespace tc355
