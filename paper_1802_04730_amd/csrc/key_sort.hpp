// Stable counting sort of small keys: the token numbers of an embedding's gradient.
//   order = the indices 0 .. n-1 by (key, index)
// A pass sorts by one digit: every workgroup counts its keys per digit, then finds where each of them goes -- keys of lower digits
// anywhere, of the same digit in earlier workgroups, in earlier wavefronts of its own, in earlier lanes -- and writes them there.
// No atomics on memory: the order, and with it every sum taken along it, is the same each time.
//
// Lanes of one digit find each other by a ballot per bit of the digit.  Bounded by the latency of a pass's launches at the sizes of a
// training step (32768 keys of 18 bits: two passes of two launches, SORT_TIME_LARGE); up to SORT_SMALL keys everything stays in one workgroup's LDS, in
// one launch (1500 keys of 14 bits: SORT_TIME_SMALL).
#pragma once
#include "tc355_device.hpp"

namespace tc355 {

constexpr int SORT_MOST_BITS = 10;          // of a digit
constexpr int SORT_MOST_BINS = 1 << SORT_MOST_BITS;
constexpr int SORT_THREADS = 512;
constexpr int SORT_TILE = 2048;             // keys of a workgroup
constexpr int SORT_ROUNDS = 4;              // keys of a thread
constexpr int SORT_SMALL = 4096;            // keys that one workgroup sorts by itself
constexpr int SORT_DIRECT_TILES = 32;       // up to so many workgroups add the earlier ones' counts up themselves
static_assert(SORT_TILE == SORT_ROUNDS * SORT_THREADS && SORT_SMALL == SORT_ROUNDS * 1024, "keys of a workgroup");

// Lanes of the wavefront that have the same digit (of `bits` bits) as this one, among `on`.
__device__ __forceinline__ unsigned long long same_digit(int d, int bits, bool on) {
  unsigned long long peers = __ballot(on);
  for (int b = 0; b < bits; b++) {
    const bool one = (d >> b) & 1;
    const unsigned long long m = __ballot(one);
    peers &= one ? m : ~m;
  }
  return peers;
}

// Rank of this lane's key among the wavefront's earlier keys of its digit; count: the wavefront's own counters in LDS, which go on.
__device__ __forceinline__ int rank_and_count(int* count, int d, int bits, bool on, int lane) {
  const unsigned long long peers = same_digit(d, bits, on);
  const int leader = peers ? __ffsll((long long)peers) - 1 : lane;
  int before = 0;
  if (on && lane == leader) {
    before = count[d];
    count[d] = before + __popcll(peers);
  }
  before = __shfl(before, leader);
  __builtin_amdgcn_wave_barrier();
  return before + __popcll(peers & ((1ull << lane) - 1));
}

// Exclusive prefix sums of v over the workgroup's threads (thread order); *total: the sum.  part: WAVES ints in LDS.
template <int WAVES>
__device__ __forceinline__ int block_prefix(int v, int* part, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int incl = v;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int o = __shfl_up(incl, d);
    if (lane >= d) incl += o;
  }
  if (lane == 63) part[wave] = incl;
  __syncthreads();
  int before = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < WAVES; w++) {
    const int x = part[w];
    before += w < wave ? x : 0;
    sum += x;
  }
  __syncthreads();
  *total = sum;
  return before + incl - v;
}

struct SortPass {
  const int* key;   // [n]; first pass: the caller's, of which those outside [0, E) and `pad` count as E
  const int* order; // [n]; nullptr in the first pass: 0 .. n-1
  int* key_out;     // [n]
  int* order_out;   // [n]
  int* count;       // [bins][tiles + 1]
  int n, E, shift, bits, tiles;
  long long pad;
  int summed;       // count holds sums over the earlier tiles; behind the last one, all tiles' sum
};

__device__ __forceinline__ int sort_key(const SortPass& p, int i) {
  const int k = p.key[i];
  if (p.order) return k;
  return k < 0 || k >= p.E || k == p.pad ? p.E : k;
}

static __global__ __launch_bounds__(SORT_THREADS) void sort_count_kernel(SortPass p) {
  __shared__ int count[SORT_MOST_BINS];
  const int bins = 1 << p.bits;
  for (int b = threadIdx.x; b < bins; b += SORT_THREADS) count[b] = 0;
  __syncthreads();
  const int64_t first = (int64_t)blockIdx.x * SORT_TILE;
  for (int j = threadIdx.x; j < SORT_TILE; j += SORT_THREADS)
    if (first + j < p.n) atomicAdd(&count[(sort_key(p, (int)(first + j)) >> p.shift) & (bins - 1)], 1);
  __syncthreads();
  for (int b = threadIdx.x; b < bins; b += SORT_THREADS) p.count[(int64_t)b * (p.tiles + 1) + blockIdx.x] = count[b];
}

// count[b][t] of tile t becomes the sum over the tiles before it; count[b][tiles] the sum of all.  A workgroup per bin.
static __global__ __launch_bounds__(WG_THREADS) void sort_sum_kernel(int* count, int tiles) {
  __shared__ int part[WAVES_PER_WG];
  int* c = count + (int64_t)blockIdx.x * (tiles + 1);
  int run = 0;
  for (int t0 = 0; t0 < tiles; t0 += 4 * WG_THREADS) {
    const int t = t0 + 4 * (int)threadIdx.x;
    int v[4], all = 0, sum;
#pragma unroll
    for (int j = 0; j < 4; j++) {
      v[j] = t + j < tiles ? c[t + j] : 0;
      all += v[j];
    }
    int before = run + block_prefix<WAVES_PER_WG>(all, part, &sum);
#pragma unroll
    for (int j = 0; j < 4; j++) {
      if (t + j < tiles) c[t + j] = before;
      before += v[j];
    }
    run += sum;
  }
  if (threadIdx.x == 0) c[tiles] = run;
}

// start[b], b < bins: where the first key of tile `tile` with digit b goes.
template <int THREADS>
__device__ __forceinline__ void tile_starts(const int* count, int tiles, int bins, int tile, int summed, int* start, int* part) {
  int run = 0;
  for (int b0 = 0; b0 < bins; b0 += THREADS) {
    const int b = b0 + threadIdx.x;
    int all = 0, before = 0;
    if (b < bins) {
      const int* c = count + (int64_t)b * (tiles + 1);
      if (summed) {
        before = c[tile];
        all = c[tiles];
      } else {
        for (int t0 = 0; t0 < tiles; t0 += 8) {
          int v[8];
#pragma unroll
          for (int j = 0; j < 8; j++) v[j] = t0 + j < tiles ? c[t0 + j] : 0;
#pragma unroll
          for (int j = 0; j < 8; j++) {
            all += v[j];
            before += t0 + j < tile ? v[j] : 0;
          }
        }
      }
    }
    int sum;
    const int lower = block_prefix<THREADS / 64>(all, part, &sum);
    if (b < bins) start[b] = run + lower + before;
    run += sum;
  }
  __syncthreads();
}

static __global__ __launch_bounds__(SORT_THREADS) void sort_scatter_kernel(SortPass p) {
  constexpr int WAVES = SORT_THREADS / 64, ROUNDS = SORT_ROUNDS;
  __shared__ int start[SORT_MOST_BINS], count[WAVES][SORT_MOST_BINS], part[WAVES];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, bins = 1 << p.bits;
  for (int b = lane; b < bins; b += 64) count[wave][b] = 0;
  tile_starts<SORT_THREADS>(p.count, p.tiles, bins, blockIdx.x, p.summed, start, part);
  const int64_t first = (int64_t)blockIdx.x * SORT_TILE + wave * (SORT_TILE / WAVES) + lane;
  int key[ROUNDS], rank[ROUNDS];
#pragma unroll
  for (int j = 0; j < ROUNDS; j++) key[j] = first + 64 * j < p.n ? sort_key(p, (int)(first + 64 * j)) : 0;
#pragma unroll
  for (int j = 0; j < ROUNDS; j++) rank[j] = rank_and_count(count[wave], (key[j] >> p.shift) & (bins - 1), p.bits, first + 64 * j < p.n, lane);
  __syncthreads();
#pragma unroll
  for (int j = 0; j < ROUNDS; j++) {
    if (first + 64 * j >= p.n) break;
    const int d = (key[j] >> p.shift) & (bins - 1);
    int to = start[d] + rank[j];
    for (int w = 0; w < wave; w++) to += count[w][d];
    p.key_out[to] = key[j];
    p.order_out[to] = p.order ? p.order[first + 64 * j] : (int)(first + 64 * j);
  }
}

// All digits in one workgroup, n <= SORT_ROUNDS * THREADS.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void sort_small_kernel(SortPass p, int key_bits) {
  constexpr int WAVES = THREADS / 64, ROUNDS = SORT_ROUNDS, MOST = ROUNDS * THREADS;
  extern __shared__ int mem[];  // keys, indices: MOST each; counters: WAVES * bins; starts: bins
  __shared__ int part[WAVES];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, bins = 1 << p.bits;
  int *keys = mem, *idx = mem + MOST, *count = mem + 2 * MOST, *start = count + WAVES * bins;
  const int first = wave * (MOST / WAVES) + lane;
  int key[ROUNDS], at[ROUNDS];
#pragma unroll
  for (int j = 0; j < ROUNDS; j++) {
    at[j] = first + 64 * j;
    key[j] = at[j] < p.n ? sort_key(p, at[j]) : 0;
  }
  for (int shift = 0; shift < key_bits; shift += p.bits) {
    for (int b = threadIdx.x; b < WAVES * bins; b += THREADS) count[b] = 0;
    __syncthreads();
    int rank[ROUNDS];
#pragma unroll
    for (int j = 0; j < ROUNDS; j++) rank[j] = rank_and_count(count + wave * bins, (key[j] >> shift) & (bins - 1), p.bits, first + 64 * j < p.n, lane);
    __syncthreads();
    int run = 0;
    for (int b0 = 0; b0 < bins; b0 += THREADS) {
      const int b = b0 + (int)threadIdx.x;
      int c[WAVES], all = 0, sum;
#pragma unroll
      for (int w = 0; w < WAVES; w++) c[w] = b < bins ? count[w * bins + b] : 0;
#pragma unroll
      for (int w = 0; w < WAVES; w++) {
        if (b < bins) count[w * bins + b] = all;
        all += c[w];
      }
      const int lower = block_prefix<WAVES>(all, part, &sum);
      if (b < bins) start[b] = run + lower;
      run += sum;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < ROUNDS; j++) {
      if (first + 64 * j >= p.n) break;
      const int d = (key[j] >> shift) & (bins - 1), to = start[d] + count[wave * bins + d] + rank[j];
      keys[to] = key[j];
      idx[to] = at[j];
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < ROUNDS; j++) {
      if (first + 64 * j >= p.n) break;
      key[j] = keys[first + 64 * j];
      at[j] = idx[first + 64 * j];
    }
  }
#pragma unroll
  for (int j = 0; j < ROUNDS; j++) {
    if (first + 64 * j >= p.n) break;
    p.key_out[first + 64 * j] = key[j];
    p.order_out[first + 64 * j] = at[j];
  }
}

}  // namespace tc355
