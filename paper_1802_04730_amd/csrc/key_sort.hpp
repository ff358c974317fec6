// Stable counting sort of small keys: the token numbers of an embedding's gradient.
//   order = the indices 0 .. n-1 by (key, index)
// A pass sorts by one digit: every workgroup counts its keys per digit, then finds where each of them goes -- keys of lower digits
// anywhere, of the same digit in earlier workgroups, in earlier wavefronts of its own, in earlier lanes -- and writes them there.
// No atomics on memory: the order, and with it every sum taken along it, is the same each time.
//
// Lanes of one digit find each other by a ballot per bit of the digit.  Bounded by the latency of a pass's launches at the sizes of a
// training step (32768 keys of 18 bits: two passes of a count of 4.7 us and a placement of 9.4).  Up to SORT_SMALL keys are ranked by counting instead.
#pragma once
#include "tc355_device.hpp"

namespace tc355 {

constexpr int SORT_MOST_BITS = 10;          // of a digit
constexpr int SORT_MOST_BINS = 1 << SORT_MOST_BITS;
constexpr int SORT_THREADS = 512;
constexpr int SORT_TILE = 2048;             // keys of a workgroup
constexpr int SORT_ROUNDS = 4;              // keys of a thread
constexpr int SORT_SMALL = 8192;            // keys that are ranked by counting
// Up to so many workgroups add the earlier ones' counts up themselves; beyond, a launch of its own does.  us, a whole gradient, without / with that
// launch: 20000 tokens 74 / 78, 50 / 54, 50000: 130 / 133, 61 / 64, 100000: 235 / 233, 87 / 87 (32000 x 2048, 10007 x 333).
constexpr int SORT_DIRECT_TILES = 32;
static_assert(SORT_TILE == SORT_ROUNDS * SORT_THREADS, "keys of a workgroup");

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

__device__ __forceinline__ int row_key(const SortPass& p, int k) { return k < 0 || k >= p.E || k == p.pad ? p.E : k; }
__device__ __forceinline__ int sort_key(const SortPass& p, int i) {
  const int k = p.key[i];
  return p.order ? k : row_key(p, k);
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

// Few keys, n <= SORT_SMALL: every key's rank is counted among all of them, from LDS; a workgroup ranks 32, eight groups of 32 lanes
// sharing the list.  n^2 comparisons, but one launch of one round trip to memory: 1500 keys in 5.8 us (all passes in one workgroup's LDS:
// 8.5), and at 8192 the time of the passes (the whole gradient of 333 columns, 31.9 us at 8192, 33.8 at 8193).
static __global__ __launch_bounds__(WG_THREADS) void sort_rank_kernel(SortPass p) {
  constexpr int KEYS = 32, SHARES = WG_THREADS / KEYS;
  extern __shared__ __align__(16) int keys[];  // n, rounded up to a multiple of 32
  __shared__ int part[SHARES][KEYS];
  const int all = (p.n + 31) / 32 * 32, share = all / SHARES;  // (a multiple of 4)
  for (int j0 = threadIdx.x; j0 < all; j0 += 8 * WG_THREADS) {  // eight loads in flight
    int k[8];
#pragma unroll
    for (int x = 0; x < 8; x++) k[x] = p.key[min(j0 + x * WG_THREADS, p.n - 1)];
#pragma unroll
    for (int x = 0; x < 8; x++) {
      const int j = j0 + x * WG_THREADS;
      if (j < all) keys[j] = j < p.n ? row_key(p, k[x]) : 0x7fffffff;  // (above every key)
    }
  }
  __syncthreads();
  const int i = blockIdx.x * KEYS + (threadIdx.x & (KEYS - 1)), s = threadIdx.x / KEYS;
  const int key = keys[i];
  int rank = 0;
  typedef int i4 __attribute__((ext_vector_type(4)));
  for (int j0 = s * share; j0 < (s + 1) * share; j0 += 32) {  // eight reads in flight
    i4 k[8];
#pragma unroll
    for (int y = 0; y < 8; y++) k[y] = *reinterpret_cast<const i4*>(keys + min(j0 + 4 * y, all - 4));
#pragma unroll
    for (int y = 0; y < 8; y++) {
      const int j = j0 + 4 * y;
      int more = 0;
#pragma unroll
      for (int x = 0; x < 4; x++) more += k[y][x] < key + (j + x < i) ? 1 : 0;  // (an equal one counts if it comes before)
      rank += j < (s + 1) * share ? more : 0;
    }
  }
  part[s][threadIdx.x & (KEYS - 1)] = rank;
  __syncthreads();
  if (s || i >= p.n) return;
  for (int w = 1; w < SHARES; w++) rank += part[w][threadIdx.x];
  p.key_out[rank] = key;
  p.order_out[rank] = i;
}

}  // namespace tc355
