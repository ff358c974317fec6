// The router of a layer of experts.
//   p = softmax(L(t,:));  the k largest logits of a token, equal ones by the lower number;  w = p there, or (norm) p over their sum
//   Off, Row, Place: the slots (t,i) sorted by expert, stable; Off(e): the first place of expert e; Row(r): the token of place r;
//   Place(t,i): the place of a slot
//   dL(t,e) = [e chosen as i] w_i g_i - share_e * sum_i g_i w_i,  share = p, or (norm) w for the chosen and 0 for the others
//
// Logits of -inf are experts that a token may not choose: a slot that finds no other is left empty (number -1, weight 0, no place).
// NaN ranks above every number, as does nothing else; a row with a NaN or a +inf has weights of NaN, as the formula has.
// The selection compares the logits themselves, as integers that order as they do (-0 as +0), so that rounding never decides.
//
// A group of 16 lanes (64 for more than 128 experts) takes a token, each lane a few neighbouring logits: k rounds find the
// largest of what is left by exchange inside the group (moves between lanes of a row of 16, without LDS).  What bounds it is those
// rounds' latency, not the logits' bytes.  A workgroup takes ROUTE_TOKENS tokens and counts its slots per expert; the counts are
// summed over the workgroups, and a last launch places the slots (key_sort.hpp's ranks by ballot).  Up to ROUTE_ALONE tokens
// all of it is one workgroup's, in one launch.  No atomics on memory; integer ones in LDS.  Measured: 16 tokens of 64 experts, 4
// chosen, 4.8 us; 16384 of 128, 8 chosen, 12.5 for the selection (29 by exchange through LDS), 4.2 for the sums, 6.0 for the places (63 where every
// workgroup added the earlier ones' counts up), 8.4-10.6 for the gradient.
// The lines between the forms, us a call: one workgroup / two launches, 64 experts of which 4: 32 tokens 6.3 / 7.9, 48: 7.8 / 8.0, 64: 9.1 / 8.1; 128 of which 8:
// 9.8 / 11.4, 14.2 / 11.6, 17.2 / 11.8; 256 of which 8: 37 / 39, 55 / 40, 71 / 40; 8 of which 2: 4.8 / 6.4, 5.5 / 6.5, 6.2 / 6.7.
// Counts added up by every workgroup / by a launch of its own, 512, 1024 and 2048 tokens: 64 experts 9.4 / 11.4, 10.0 / 11.4, 12.2 / 11.7; 128: 13.4 / 15.0,
// 14.7 / 15.3, 17.5 / 15.6; 256: 42.7 / 43.7, 45.0 / 44.0, 50.9 / 44.6; 8: 7.5 / 9.5, 8.1 / 9.6, 9.5 / 9.6.
#pragma once
#include "expert_types.hpp"
#include "key_sort.hpp"
#include "lanes.hpp"

namespace tc355 {

constexpr int ROUTE_TOKENS = 32;      // of a workgroup
constexpr int ROUTE_ALONE = 32;       // tokens that one workgroup routes by itself
constexpr int ROUTE_MOST_ALONE = 64;  // the same without a workspace
constexpr int ROUTE_MOST_E = 1023;    // (with the empty slots' bin: 10 bits)
constexpr int ROUTE_MOST_K = 64;
constexpr int ROUTE_DIRECT_TILES = 32;  // up to so many workgroups add the earlier ones' counts up themselves

struct RouteArgs {
  const void* L;  // [T][E]
  float* Wt;      // [T][k]
  int* Id;        // [T][k]
  int* Off;       // [E+1]
  int* Row;       // [T*k]
  int* Place;     // [T][k]
  int* count;     // [bins][tiles + 1]; nullptr: one workgroup does it all
  int T, E, k, norm, bits, tiles, summed;
  int tokens;     // of a workgroup
};

__device__ __forceinline__ unsigned route_order(float x) {  // orders as the logits do; 0: -inf
  if (x != x) return 0xffffffffu;
  const unsigned b = __builtin_bit_cast(unsigned, x + 0.0f);
  const unsigned o = b & 0x80000000u ? ~b : b | 0x80000000u;
  return o - 0x007fffffu;  // (-inf is the lowest: 0x007fffff)
}

// A lane's logits: V neighbours from column c on, in as few loads as they fit; -inf past the end.
template <typename T, int V>
__device__ __forceinline__ void load_logits(const T* row, int c, int E, float (&x)[V]) {
  constexpr int P = V < Elem<T>::PER16 ? V : Elem<T>::PER16;
  if (c + V <= E) {
#pragma unroll
    for (int h = 0; h < V; h += P) {
      const Pack<T, P> v = load_pack<T, P>(row + c + h);
#pragma unroll
      for (int i = 0; i < P; i++) x[h + i] = (float)v.e[i];
    }
  } else {
#pragma unroll
    for (int v = 0; v < V; v++) x[v] = c + v < E ? (float)row[c + v] : -__builtin_inff();
  }
}

// The places of a workgroup's slots: Id of the tokens of workgroup `tile`, all threads.
__device__ __forceinline__ void route_place(const RouteArgs& p, int tile, const int* start, int* count) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, bins = 1 << p.bits;
  for (int b = lane; b < bins; b += 64) count[wave * bins + b] = 0;
  const int64_t first = (int64_t)tile * p.tokens * p.k, all = (int64_t)p.T * p.k;
  const int64_t last = min(first + (int64_t)p.tokens * p.k, all);
  // a quarter of the slots for each wavefront, counted first, then placed
  const int share = ((int)(last - first) + WAVES_PER_WG - 1) / WAVES_PER_WG;
  const int64_t lo = min(first + (int64_t)wave * share, last), hi = min(lo + share, last);
  for (int64_t s0 = lo; s0 < hi; s0 += 64) {
    const bool on = s0 + lane < hi;
    const int e = on ? p.Id[s0 + lane] : 0;
    rank_and_count(count + wave * bins, e < 0 ? p.E : e, p.bits, on, lane);
  }
  __syncthreads();
  for (int b = threadIdx.x; b < bins; b += WG_THREADS) {
    int at = start[b];
#pragma unroll
    for (int w = 0; w < WAVES_PER_WG; w++) {
      const int c = count[w * bins + b];
      count[w * bins + b] = at;
      at += c;
    }
  }
  __syncthreads();
  for (int64_t s0 = lo; s0 < hi; s0 += 64) {
    const int64_t s = s0 + lane;
    const bool on = s < hi;
    const int e = on ? p.Id[s] : 0;
    const int r = rank_and_count(count + wave * bins, e < 0 ? p.E : e, p.bits, on, lane);
    if (on) {
      p.Place[s] = e < 0 ? -1 : r;
      p.Row[r] = e < 0 ? -1 : (int)(s / p.k);
    }
  }
}

// What follows the selection: mem holds the workgroup's slots of each expert.  They go to memory, or, where one workgroup does it all, turn into starts,
// and the slots are placed.
__device__ __forceinline__ void route_counted(const RouteArgs& p, int* mem, int* part) {
  const int bins = 1 << p.bits;
  __syncthreads();
  if (p.count) {
    for (int b = threadIdx.x; b < bins; b += WG_THREADS) p.count[(int64_t)b * (p.tiles + 1) + blockIdx.x] = mem[b];
    return;
  }
  // one workgroup: counts to starts, then the places
  __threadfence_block();
  int run = 0;
  for (int b0 = 0; b0 < bins; b0 += WG_THREADS) {
    const int b = b0 + threadIdx.x, c = b < bins ? mem[b] : 0;
    int total;
    const int lower = block_prefix<WAVES_PER_WG>(c, part, &total);
    if (b < bins) mem[b] = run + lower;
    run += total;
    if (b <= p.E) p.Off[b] = mem[b];
  }
  __syncthreads();
  route_place(p, 0, mem, mem + bins);
}

template <typename T, int G, int V>
__global__ __launch_bounds__(WG_THREADS) void route_kernel(RouteArgs p) {
  extern __shared__ int mem[];  // [bins] counts; one workgroup: starts in their place, [waves][bins] counters behind
  __shared__ int part[WAVES_PER_WG];
  const int bins = 1 << p.bits;
  for (int b = threadIdx.x; b < bins; b += WG_THREADS) mem[b] = 0;
  __syncthreads();
  const int lane = threadIdx.x & (G - 1), group = threadIdx.x / G;
  const T* L = static_cast<const T*>(p.L);
  for (int r = group; r < p.tokens; r += WG_THREADS / G) {
    const int64_t t = (int64_t)blockIdx.x * p.tokens + r;
    if (t >= p.T) break;  // (the whole group, and all groups behind it)
    float x[V];
    unsigned key[V];
    float most = -__builtin_inff();
    load_logits<T, V>(L + t * p.E, lane * V, p.E, x);
#pragma unroll
    for (int v = 0; v < V; v++) {
      key[v] = route_order(x[v]);
      most = fmaxf(most, x[v]);
    }
    most = group_all<G>(most, most_of);
    if (most == -__builtin_inff()) most = 0.0f;  // (nothing to choose: every exp is 0, or NaN)
    float sum = 0.0f;
    if (!p.norm) {
#pragma unroll
      for (int v = 0; v < V; v++) sum += expf(x[v] - most);
      sum = group_all<G>(sum, sum_of);
    }
    float val = 0.0f;
    int id = -1;
    const int slot_lane = lane;
    for (int i = 0; i < p.k; i++) {
      unsigned best = 0;
#pragma unroll
      for (int v = 0; v < V; v++) best = larger(best, key[v]);
      best = group_all<G>(best, larger);
      int at = 0x7fffffff;
#pragma unroll
      for (int v = V - 1; v >= 0; v--)
        if (key[v] == best) at = lane * V + v;
      at = group_all<G>(at, smaller);
      float mine = 0.0f;
#pragma unroll
      for (int v = 0; v < V; v++)
        if (best && at == lane * V + v) {
          key[v] = 0;
          mine = x[v];
        }
      const float chosen = group_all<G>(mine, [](float a, float b) { return a != 0.0f ? a : b; });  // (the others have 0; so may it)
      const float w = best ? expf(chosen - most) : 0.0f;
      if (p.norm) sum += w;
      if ((i & (G - 1)) == slot_lane) {
        val = w;
        id = best ? at : -1;
      }
      if ((i & (G - 1)) == G - 1 || i == p.k - 1) {  // (k <= G, by the host's choice of G)
        const int s = (i & ~(G - 1)) + slot_lane;
        if (s <= i) {
          p.Wt[t * p.k + s] = id < 0 ? 0.0f : val / sum;
          p.Id[t * p.k + s] = id;
          atomicAdd(&mem[id < 0 ? p.E : id], 1);
        }
      }
    }
  }
  route_counted(p, mem, part);
}

static __global__ __launch_bounds__(WG_THREADS) void route_place_kernel(RouteArgs p) {
  extern __shared__ int mem[];
  __shared__ int part[WAVES_PER_WG];
  const int bins = 1 << p.bits;
  tile_starts<WG_THREADS>(p.count, p.tiles, bins, blockIdx.x, p.summed, mem, part);
  if (blockIdx.x == 0)  // (before the first tile nothing counts: its starts are the experts')
    for (int b = threadIdx.x; b <= p.E; b += WG_THREADS) p.Off[b] = mem[b];
  route_place(p, blockIdx.x, mem, mem + bins);
}

struct RouteGradArgs {
  const void* L;    // [T][E]
  const int* Id;    // [T][k]
  const float* dWt; // [T][k]
  void* dL;         // [T][E]
  int T, E, k, norm;
};

template <typename T, int G, int V>
__global__ __launch_bounds__(WG_THREADS) void route_grad_kernel(RouteGradArgs p, int64_t first) {
  const int lane = threadIdx.x & (G - 1);
  const int64_t t = (first + blockIdx.x) * (WG_THREADS / G) + threadIdx.x / G;
  if (t >= p.T) return;
  const T* L = static_cast<const T*>(p.L) + t * p.E;
  float x[V], g[V];
  bool chosen[V];
  float most = -__builtin_inff();
  load_logits<T, V>(L, lane * V, p.E, x);
#pragma unroll
  for (int v = 0; v < V; v++) {
    most = fmaxf(most, x[v]);
    g[v] = 0.0f;
    chosen[v] = false;
  }
  most = group_all<G>(most, most_of);
  if (most == -__builtin_inff()) most = 0.0f;
  for (int i0 = 0; i0 < p.k; i0 += G) {  // a slot a lane, handed round
    const int i = min(i0 + lane, p.k - 1);
    const int ids = p.Id[t * p.k + i];
    const float ds = p.dWt[t * p.k + i];
    const int n = min(G, p.k - i0);
    for (int j = 0; j < n; j++) {
      const int id = __shfl(ids, j, G);
      const float d = __shfl(ds, j, G);
#pragma unroll
      for (int v = 0; v < V; v++)
        if (id == lane * V + v) {
          g[v] = d;
          chosen[v] = true;
        }
    }
  }
  float sum = 0.0f, inner = 0.0f;
#pragma unroll
  for (int v = 0; v < V; v++) {
    x[v] = expf(x[v] - most);
    if (!p.norm || chosen[v]) sum += x[v];
    if (chosen[v]) inner += g[v] * x[v];
  }
  sum = group_all<G>(sum, sum_of);
  inner = group_all<G>(inner, sum_of);
  if (sum == 0.0f) sum = 1.0f;  // (a row of nothing, or without slots)
  const float share = 1.0f / sum;
  inner *= share;
  T* const out = static_cast<T*>(p.dL) + t * p.E;
  T o[V];
#pragma unroll
  for (int v = 0; v < V; v++) o[v] = narrow<T>((!p.norm || chosen[v] ? x[v] * share : 0.0f) * (g[v] - inner));  // (g: 0 where not chosen)
  const int c = lane * V;
  if (c + V <= p.E) {
    constexpr int P = V < Elem<T>::PER16 ? V : Elem<T>::PER16;
#pragma unroll
    for (int h = 0; h < V; h += P) {
      Pack<T, P> v;
#pragma unroll
      for (int i = 0; i < P; i++) v.e[i] = o[h + i];
      *reinterpret_cast<Pack<T, P>*>(out + c + h) = v;
    }
  } else {
#pragma unroll
    for (int v = 0; v < V; v++)
      if (c + v < p.E) out[c + v] = o[v];
  }
}

}  // namespace tc355
