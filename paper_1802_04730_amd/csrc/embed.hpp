// Rows of a token table and their gradient.
//   O(t,j)    = s * LUT(Idx(t), j)
//   dLUT(e,j) (+)= s * sum over the t with Idx(t) = e of dO(t,j)
// Both only move bytes.  A group of lanes takes up to 16 bytes each of a row, as many elements as make 16 bytes of the wider of input and
// output; rows of any width start at any multiple of an element.  A call with 16384 rows of 4096 bfloat16 takes 43 us (6.3 TB/s: words that come again are read
// from cache, 78 MB of 134 from memory), with 8 rows 3.3-3.7 (the kernel 2.5).
//
// The gradient walks the tokens sorted by number (key_sort.hpp) in chunks of EMBED_CHUNK places: a group of lanes adds up its chunk's rows of dO
// in order, whose addresses are all known beforehand, and hands on a sum where the number changes.  Runs of one number
// inside a chunk go to the table; the ends that a chunk shares with its neighbours go to a workspace, and a second launch joins them, chunk by
// chunk: language has words that make up a large part of a batch.  No atomics, one order for every sum.  Rows of numbers that do not occur are
// written with zeros by workgroups of their own in the same launch, or left alone where the gradient is added to what is there.
// (A group of lanes per row of the table, empty or not: 402 us against 233 and 10 at 32768 tokens of 2048 bfloat16, a table of 131072 rows in fp32: three
// dependent trips to memory a row.)
#pragma once
#include "expert_types.hpp"

namespace tc355 {

// Places of a chunk.  Small ones spread few tokens over the device; long ones hand fewer partial sums on, which counts sooner where a few numbers make up
// much of the batch, as words do, and where a wide table's zeros keep the device busy anyway.  us, 8 / 32 places, numbers by Zipf's law (in brackets: all
// equally often).  Table written, 8192, 14336 and 20000 tokens: 5000 x 256 bfloat16 37 / 40 (30 / 39), 45 / 44 (34 / 41), 50 / 45 (35 / 41); 32000 x 1024 46 / 44 (39 / 44), 58 / 51 (45 / 50),
// 64 / 54 (48 / 52); 32000 x 2048 in fp32 of bfloat16 86 / 81 (78 / 80), 99 / 86 (90 / 89), 107 / 87 (90 / 88); the same of fp32 94 / 81 (83 / 82), 110 / 88 (99 / 91), 119 / 93 (104 / 96).
// Added to: 5000 x 256 38 / 43 (31 / 42), 46 / 47 (34 / 44), 52 / 47 (36 / 43); 32000 x 2048 49 / 61 (50 / 65), 64 / 70 (70 / 76), 77 / 72 (87 / 89).
constexpr int EMBED_CHUNK = 32;
constexpr int EMBED_SMALL_CHUNK = 8;
constexpr int EMBED_FEW = 14336;         // from so many tokens on chunks are long,
constexpr int EMBED_FEW_WRITTEN = 8192;  // or from so many where a table of EMBED_WIDE columns or more is written
constexpr int EMBED_WIDE = 512;

struct EmbedArgs {
  const void* LUT;
  const int* Idx;
  void* O;
  long long E, T;
  int D, lpr, cols;  // lanes of a row's group: a power of two <= 64; groups of a row
  float scale;
};

template <typename T, int V>
__global__ __launch_bounds__(WG_THREADS) void embed_kernel(EmbedArgs p, int64_t first) {
  typedef typename Wide<T>::type S;
  const int64_t g = ((first + blockIdx.x) * WG_THREADS + threadIdx.x) / p.lpr;
  const int64_t t = g / p.cols;
  const RowUnit<V> u((g % p.cols) * p.lpr + (threadIdx.x & (p.lpr - 1)), p.D);
  if (t >= p.T || !u.on) return;
  const long long e = p.Idx[t];
  const bool ok = e >= 0 && e < p.E;
  Pack<T, V> v = load_unit<T, V>(static_cast<const T*>(p.LUT) + (ok ? e : 0) * p.D, u);
#pragma unroll
  for (int i = 0; i < V; i++) v.e[i] = narrow<T>(ok ? (S)v.e[i] * (S)p.scale : (S)__builtin_nanf(""));
  store_unit<T, V>(static_cast<T*>(p.O) + t * p.D, u, v);
}

struct EmbedGradArgs {
  const void* dO;
  void* dLUT;
  void* part;        // [chunks][2][D], of the wide type: the sums of the run that a chunk begins with, and ends with
  const int* key;    // sorted numbers; E: of no row
  const int* order;  // the tokens in that order
  int T, E, D, lpr;  // lanes of a group: a power of two <= 256
  int chunk;         // EMBED_CHUNK or EMBED_SMALL_CHUNK
  unsigned token_wgs;  // workgroups that take chunks; the others take `rows` rows each
  int rows;
  float scale;
  int add;
};

// The first place of a number >= e, by all lanes of a wavefront.
__device__ __forceinline__ int first_place(const int* key, int T, int64_t e) {
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = T;  // the answer is in [lo, hi]
  while (lo < hi) {
    const int step = (hi - lo + 63) / 64;
    const int64_t at = lo + (int64_t)(lane + 1) * step - 1;
    const int below = __popcll(__ballot(at < hi && key[at < hi ? at : lo] < e));
    lo += below * step;
    hi = min(hi, lo + step - 1);
    if (lo > hi) lo = hi;
  }
  return lo;
}

// The table's row, or what is added to it.
template <typename TO, int V, typename S>
__device__ __forceinline__ void embed_give(const EmbedGradArgs& p, int64_t e, const RowUnit<V>& u, const S (&acc)[V]) {
  TO* out = static_cast<TO*>(p.dLUT) + e * p.D;
  Pack<TO, V> o;
  if (p.add) o = load_unit<TO, V>(out, u);
#pragma unroll
  for (int i = 0; i < V; i++) o.e[i] = narrow<TO>(p.add ? acc[i] * (S)p.scale + (S)o.e[i] : acc[i] * (S)p.scale);
  store_unit<TO, V>(out, u, o);
}

constexpr int EMBED_FILL_ROWS = 32;

template <typename T, typename TO, int V>
__global__ __launch_bounds__(WG_THREADS) void embed_grad_kernel(EmbedGradArgs p) {
  typedef typename Wide<T>::type S;
  const int lane = threadIdx.x & (p.lpr - 1), group = threadIdx.x / p.lpr, groups = WG_THREADS / p.lpr;
  if (blockIdx.x >= p.token_wgs) {  // zeros for the rows of no token
    __shared__ int bounds[2], used[EMBED_FILL_ROWS];
    for (int64_t e0 = (int64_t)(blockIdx.x - p.token_wgs) * p.rows, end = min(e0 + p.rows, (int64_t)p.E); e0 < end; e0 += EMBED_FILL_ROWS) {
      const int n = (int)min((int64_t)EMBED_FILL_ROWS, end - e0), wave = threadIdx.x >> 6;
      if (wave < 2) {
        const int at = first_place(p.key, p.T, e0 + wave * n);
        if ((threadIdx.x & 63) == 0) bounds[wave] = at;
      } else if (wave == 2 && (threadIdx.x & 63) < EMBED_FILL_ROWS) {
        used[threadIdx.x & 63] = 0;
      }
      __syncthreads();
      for (int j = bounds[0] + threadIdx.x; j < bounds[1]; j += WG_THREADS) used[p.key[j] - e0] = 1;
      __syncthreads();
      for (int x = group; x < n; x += groups) {
        if (used[x]) continue;
        for (int64_t c = lane; c * V < p.D; c += p.lpr) {
          const RowUnit<V> u(c, p.D);
          Pack<TO, V> o;
#pragma unroll
          for (int i = 0; i < V; i++) o.e[i] = static_cast<TO>(0.0f);
          store_unit<TO, V>(static_cast<TO*>(p.dLUT) + (e0 + x) * p.D, u, o);
        }
      }
      __syncthreads();
    }
    return;
  }
  // a chunk for each group of lanes: its numbers (with the neighbours') and tokens
  extern __shared__ int mem[];  // groups of chunk + 3 numbers, then of chunk + 1 tokens (odd rows: groups in different banks)
  int *const keys = mem + group * (p.chunk + 3), *const tokens = mem + groups * (p.chunk + 3) + group * (p.chunk + 1);
  const int64_t chunk = (int64_t)blockIdx.x * groups + group;
  const int64_t lo = chunk * p.chunk;
  const int n = (int)max((int64_t)0, min((int64_t)p.chunk, p.T - lo));
  for (int j = lane; j < n + 2 && n; j += p.lpr) {
    const int64_t at = lo - 1 + j;
    keys[j] = at >= 0 && at < p.T ? p.key[at] : -1;  // (-1: nobody's)
    if (j < n) tokens[j] = p.order[lo + j];
  }
  __syncthreads();
  if (n == 0) return;
  const int* const key = keys + 1;
  constexpr int NB = 8;  // rows in flight
  for (int64_t c = lane; c * V < p.D; c += p.lpr) {
    const RowUnit<V> u(c, p.D);
    S acc[V];
#pragma unroll
    for (int i = 0; i < V; i++) acc[i] = 0;
    bool from_before = key[0] == key[-1];
    for (int r0 = 0; r0 < n; r0 += NB) {
      if (key[r0] >= p.E) break;  // (tokens of no row come last)
      Pack<T, V> v[NB];
#pragma unroll
      for (int j = 0; j < NB; j++) v[j] = load_unit<T, V>(static_cast<const T*>(p.dO) + (int64_t)tokens[min(r0 + j, n - 1)] * p.D, u);
#pragma unroll
      for (int j = 0; j < NB; j++) {
        const int r = r0 + j;
        if (r >= n || key[r] >= p.E) break;
#pragma unroll
        for (int i = 0; i < V; i++) acc[i] += (S)v[j].e[i];
        const bool goes_on = key[r + 1] == key[r];
        if (goes_on && r + 1 < n) continue;
        if (!goes_on && !from_before) {
          embed_give<TO, V>(p, key[r], u, acc);
        } else {  // what comes from the chunk before goes in front, whether it ends here or not
          S* out = static_cast<S*>(p.part) + (chunk * 2 + (from_before ? 0 : 1)) * p.D + u.c;
#pragma unroll
          for (int i = 0; i < V; i++)
            if (i >= u.skip) out[i] = acc[i];
        }
        from_before = false;
#pragma unroll
        for (int i = 0; i < V; i++) acc[i] = 0;
      }
    }
  }
}

// Runs that begin in a chunk and end in a later one: the chunk's last sum, then the first sums of those behind it.
template <typename T, typename TO, int V>
__global__ __launch_bounds__(WG_THREADS) void embed_join_kernel(EmbedGradArgs p) {
  typedef typename Wide<T>::type S;
  // a wavefront for each chunk, wherever its columns are
  const int64_t chunk = (int64_t)blockIdx.x * WAVES_PER_WG + (threadIdx.x >> 6);
  const int64_t end = (chunk + 1) * p.chunk;
  if (end >= p.T) return;
  const int first = p.key[end - p.chunk], before = chunk ? p.key[end - p.chunk - 1] : -1, last = p.key[end - 1], next = p.key[end];
  if (last != next || last >= p.E || (first == last && before == last)) return;
  const int64_t past = first_place(p.key + end, (int)(p.T - end), (int64_t)last + 1) + end;
  const int64_t chunks = (past - 1) / p.chunk;  // the last chunk of the run
  const int lane = threadIdx.x & 63;
  for (int64_t c = (int64_t)blockIdx.y * 64 + lane; c * V < p.D; c += 64 * gridDim.y) {
    const RowUnit<V> u(c, p.D);
    const S* part = static_cast<const S*>(p.part);
    S acc[V];
    const Pack<S, V> tail = load_unit<S, V>(part + (chunk * 2 + 1) * p.D, u);
#pragma unroll
    for (int i = 0; i < V; i++) acc[i] = tail.e[i];
    constexpr int NB = 8;
    for (int64_t x = chunk + 1; x <= chunks; x += NB) {
      Pack<S, V> v[NB];
#pragma unroll
      for (int j = 0; j < NB; j++) v[j] = load_unit<S, V>(part + min(x + j, chunks) * 2 * p.D, u);
#pragma unroll
      for (int j = 0; j < NB; j++)
#pragma unroll
        for (int i = 0; i < V; i++) acc[i] = x + j <= chunks ? acc[i] + v[j].e[i] : acc[i];
    }
    embed_give<TO, V>(p, last, u, acc);
  }
}

}  // namespace tc355
