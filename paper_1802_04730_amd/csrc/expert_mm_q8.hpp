// Products grouped by expert of rows and weights in 8 bits (quantize8.hpp):
//   Y(r,n) = act(sum_b 2^(SX(s,b) + SW(e,n/128,b) - 254) sum_{k of block b} X(s,k) W(e,n,k)),  s = src(r)
// With the transposed form of the weights it is the gradient of the rows too.  What bounds it: 2 R N K operations on the 8-bit matrix core; the weights' bytes where an
// expert has few rows.
//
// Tiles, stages of 128 bytes, their way to LDS and the swizzle are expert_mm.hpp's.  A stage is a block of 128 elements: one matrix instruction of 16 x 16 x 128
// takes a whole stage, with the scales' bytes as operands, so that scaling costs nothing.  A lane's 32 bytes of a row are the chunks q and 4 + q: which elements those are is
// all the same, as long as both operands agree.
//
// The 8-bit matrix instruction adds the products of 8 neighbours with the bits down to 2^-13 of the largest one's exponent and cuts the rest; beyond these
// groups its sums keep 24 bits (measured with products that cancel).  So up to 2^-10 of a group's largest product is lost -- operands in e4m3 are
// off by 2^-4 of their own --, a choice for 16-bit outputs: its rate is over three times the 16-bit instruction's (3.8 PFLOP/s against 1.2, both from registers).  The cut is
// 2^-16 of the outputs' norm with normally distributed operands and 2^-14.4 where columns stand out by 20 times, of which half rounds away 2^-12.2 and bfloat16 2^-9.2: 1 in 80 and 1 in 35 bfloat16 outputs are rounded to another
// neighbour (half: 1 in 15 and 1 in 7), and the error against 64 bits is that of sums in 32 bits for bfloat16 and 0.3 and 2.3 % above it for half.  Outputs whose terms cancel lose more of themselves.
// float outputs go by the half instruction instead, which takes the same values, widened, and sums them in 32 bits.
//
// Measured, rows and weights in 8 bits, bfloat16: (R,N,K) = (4096,8192,4096) 125-131 us (2.1-2.2 PFLOP/s; the library's product without blocks 95), 8192^3 460 (2.4), (4096,4096,8192) 109
// (2.5); 32 experts, 16384 rows, uneven shares, 2048 x 4096 180-206, the gradient of the rows with a gate 213-230; eight experts with 4 rows each, 4096 x 2048, 14 (4.8 TB/s of weights).  A stage of a tile
// of 256 takes 1.4 us where few tiles run and 1.5-1.7 where all do; its products alone 0.87, or 1.2 at the power that 256 compute units may draw.  What is left are the loads: 0.3 us a stage,
// as four wavefronts ask the address path at once, whether LDS is read or not, and 0.1 for two barriers.  Tried and left: a branch behind each matrix instruction that gives every wavefront slots of its
// own for its loads (2.6 us a stage), a copy of the loop for each wavefront instead (1.6), eight wavefronts (1.4 / 1.7), loads spread over the next stage's first steps too (1.5 / 1.7), buffer
// loads (the same); rows put in 8 bits by the kernel for few rows itself (22 us where the launch before it and the product take 18).
#pragma once
#include "expert_mm.hpp"
#include "quantize8.hpp"

#include <type_traits>

namespace tc355 {

typedef int i8v __attribute__((ext_vector_type(8)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));

struct Q8Args {
  const unsigned char* A;   // [T][stages * 128]
  const unsigned char* SA;  // [T][stages]
  const unsigned char* W;   // [E][NO][stages * 128]
  const unsigned char* SW;  // [E][nb][stages]
  void* C;                  // [R][NO]
  const void* gate;         // [R][NO] or nullptr
  const int* off;           // [E+1]; nullptr: one expert has all rows
  const int* row;           // [R] or nullptr
  int R, T, E, stages, NO;
  int nt;                   // column tiles
  int relu;
};

// expert_tile, also without offsets.
__device__ __forceinline__ bool q8_tile(const Q8Args& p, int bm, ExpertTile* t) {
  if (p.off) return expert_tile(p.off, p.E, p.R, bm, p.nt, blockIdx.x, t);
  const unsigned mt = (unsigned)((p.R + bm - 1) / bm), total = mt * p.nt, run = (total + 7) / 8;
  const unsigned at = (blockIdx.x & 7) * run + blockIdx.x / 8;
  if (blockIdx.x / 8 >= run || at >= total) return false;
  const int block = (int)(at / (unsigned)(8 * p.nt)), in = (int)(at % (unsigned)(8 * p.nt)), rows = min(8, (int)mt - 8 * block);
  *t = ExpertTile{0, 0, p.R, 8 * block + in % rows, in / rows};
  return true;
}

// Up to four scale bytes of a row from stage `s` on, the first one lowest.
__device__ __forceinline__ unsigned q8_scales(const unsigned char* row, int s, int stages) {
  typedef unsigned any __attribute__((aligned(1)));
  if (s + 4 <= stages) return *reinterpret_cast<const any*>(row + s);
  unsigned v = 0;
  for (int i = 0; i < 3; i++)
    if (s + i < stages) v |= (unsigned)row[s + i] << (8 * i);
  return v;
}

// acc += the products of a stage: w and x 32 bytes of a row each, their scales bytes SW of sw and SX of sx.
template <typename T, int SW, int SX>
__device__ __forceinline__ f4 q8_mfma(const i8v& w, const i8v& x, f4 acc, unsigned sw, unsigned sx) {
  if constexpr (sizeof(T) == 2) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, acc, 0, 0, SW, (int)sw, SX, (int)sx);
  } else {
    f4 sum = {0, 0, 0, 0};
    typedef Elem<f16>::v8 v8;
#pragma unroll
    for (int s = 0; s < 4; s++) {
      v8 a, b;
#pragma unroll
      for (int h = 0; h < 2; h++) {
        const h2 a0 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[2 * s + h], 1.0f, false), a1 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[2 * s + h], 1.0f, true);
        const h2 b0 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x[2 * s + h], 1.0f, false), b1 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x[2 * s + h], 1.0f, true);
        a[4 * h] = a0[0]; a[4 * h + 1] = a0[1]; a[4 * h + 2] = a1[0]; a[4 * h + 3] = a1[1];
        b[4 * h] = b0[0]; b[4 * h + 1] = b0[1]; b[4 * h + 2] = b1[0]; b[4 * h + 3] = b1[1];
      }
      sum = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, sum, 0, 0, 0);
    }
    const int a = (int)(sw >> (8 * SW) & 255), b = (int)(sx >> (8 * SX) & 255);
    const bool nan = a == (int)Q8_NAN || b == (int)Q8_NAN;
#pragma unroll
    for (int v = 0; v < 4; v++) acc[v] += nan ? __builtin_nanf("") : __builtin_amdgcn_ldexpf(sum[v], a + b - 254);
    return acc;
  }
}

template <int I>
using Q8Int = std::integral_constant<int, I>;
// f(integral constants 0 .. N-1), in turn.
template <int N, int I = 0, typename F>
__device__ __forceinline__ void q8_for(F f) {
  if constexpr (I < N) {
    f(Q8Int<I>{});
    q8_for<N, I + 1>(f);
  }
}

// 16 bytes a lane straight to LDS, lane l's to `lds` + 16 l (both uniform).  In asm, so that the compiler does not take every later LDS read for one of these bytes and
// wait for them: who reads them waits by emm_wait<0> and a barrier.
__device__ __forceinline__ void q8_to_lds(const char* p, unsigned lds) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(p), "s"(lds) : "memory", "m0");
}
__device__ __forceinline__ void q8_to_lds(const char* base, unsigned off, unsigned lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "s"(lds) : "memory", "m0");
}

constexpr int Q8_CHUNK = 64;  // stages whose scales are in LDS

// Each wavefront multiplies MI x NI blocks of 16 x 16, a stage in MI steps: a step multiplies one block of 16 rows with all columns.  The first half of the steps reads the other rows'
// fragments; then a barrier: nobody reads this buffer any more, and the second half requests the stage after the next into it, a few loads a step, since the wavefront
// stands still where the address path has more than it takes.  Before the last step another barrier: the next stage, requested a stage and a half before, is in LDS, and the
// last step replaces each column's fragment by the next stage's as soon as it is used.  Four wavefronts: 128 x 128 of a tile of 256 each read a third less from LDS (128 KB a
// stage) than eight, whose reads and the loads' writes would take as long as the products; a wavefront has all 512 registers of its SIMD's lanes, half of them sums (and 4 values in scratch
// memory beside them).
// LDS of a tile: two stages and the scales, or the results on their way out.
template <typename T, int BM, int BN>
constexpr int q8_tile_lds() {
  constexpr int in = 2 * (BM + BN) * EMM_STAGE + Q8_CHUNK * (BM + (BN + Q8_BLOCK - 1) / Q8_BLOCK), out = BM * BN * sizeof(T);
  return in > out ? in : out;
}
// Rows from m0 on (BM of them, or up to `hi`), BN columns from n0 on.
template <typename T, int BM, int BN, int WM, int WN>
__device__ __forceinline__ void q8_tile_product(const Q8Args& p, char* lds, int e, int m0, int hi, int n0) {
  constexpr int NW = WM * WN, MI = BM / WM / 16, NI = BN / WN / 16;
  constexpr int PA = BM / 8 / NW, PB = BN / 8 / NW, LOADS = PA + PB;  // loads of a wavefront a stage, 8 rows each
  constexpr int EACH = LOADS / (MI / 2);                              // of them in each of the steps of a stage's second half
  constexpr int BLOCKS = (BN + Q8_BLOCK - 1) / Q8_BLOCK;
  static_assert(MI % 2 == 0 && EACH * (MI / 2) == LOADS && PA * 8 * NW == BM && PB * 8 * NW == BN && BN / WN <= Q8_BLOCK, "whole steps, loads and blocks");
  constexpr int BYTES_A = BM * EMM_STAGE, STAGE = (BM + BN) * EMM_STAGE;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 15, q = lane >> 4;
  const int rm = (wave / WN) * (BM / WM), cn = (wave % WN) * (BN / WN);
  const bool owned = e < p.E && p.T > 0;
  f4 acc[MI][NI];
#pragma unroll
  for (int m = 0; m < MI; m++)
#pragma unroll
    for (int n = 0; n < NI; n++) acc[m][n] = f4{0, 0, 0, 0};
  if (owned) {
    const int64_t ld = (int64_t)p.stages * EMM_STAGE;
    const auto source = [&](int j) -> int64_t {
      const int r = min(m0 + j, hi - 1);  // (rows past the expert's: any will do)
      return p.row ? min(max(p.row[r], 0), p.T - 1) : r;
    };
    const int most = p.NO - 1 - n0, nb = (p.NO + Q8_BLOCK - 1) / Q8_BLOCK;
    const lds_char* const mem = (lds_char*)lds;
    const unsigned base = (unsigned)(uintptr_t)mem;
    lds_char* const scales = (lds_char*)lds + 2 * STAGE;
    // this lane's rows of the loads, at its chunk of the stage
    const char* a[PA];
    unsigned b[PB];
    const char* w = reinterpret_cast<const char*>(p.W) + ((int64_t)e * p.NO + n0) * ld;
    const int chunk = ((lane & 7) ^ (lane >> 3)) * 16;
#pragma unroll
    for (int j = 0; j < PA; j++) a[j] = reinterpret_cast<const char*>(p.A) + source((wave * PA + j) * 8 + (lane >> 3)) * ld + chunk;
#pragma unroll
    for (int j = 0; j < PB; j++) b[j] = (unsigned)(min((wave * PB + j) * 8 + (lane >> 3), most) * ld) + chunk;
    const auto load = [&](auto j, unsigned to) {  // one of the wavefront's loads
      constexpr int J = decltype(j)::value;
      if constexpr (J < PA) {
        q8_to_lds(a[J], base + to + (wave * PA + J) * 1024);
        a[J] += EMM_STAGE;
      } else {
        q8_to_lds(w, b[J - PA], base + to + BYTES_A + (wave * PB + J - PA) * 1024);
      }
    };
    // The scales of a chunk of stages from s0 on: A's as [stage][wavefront's rows][16][MI], so that a lane reads those of its rows at once, B's as [block][stage].
    const auto fill = [&](int s0) {
      const int n = min(Q8_CHUNK, p.stages - s0);
      for (int r = tid; r < BM; r += 64 * NW) {
        const unsigned char* from = p.SA + source(r) * p.stages + s0;
        lds_char* const to = scales + r / (16 * MI) * (16 * MI) + r % 16 * MI + r / 16 % MI;
        for (int s = 0; s < n; s += 16) {
          unsigned v[4];
#pragma unroll
          for (int x = 0; x < 4; x++) v[x] = s + 4 * x < n ? q8_scales(from, s + 4 * x, n) : 0;
#pragma unroll
          for (int x = 0; x < 16; x++) to[(s + x) * BM] = (char)(v[x / 4] >> (8 * (x & 3)));
        }
      }
      for (int x = tid; x < BLOCKS * Q8_CHUNK; x += 64 * NW) {
        const int block = min(n0 / Q8_BLOCK + x / Q8_CHUNK, nb - 1), s = min(x % Q8_CHUNK, n - 1);
        scales[Q8_CHUNK * BM + x] = (char)p.SW[((int64_t)e * nb + block) * p.stages + s0 + s];
      }
    };
    typedef unsigned words __attribute__((ext_vector_type((MI + 3) / 4)));
    const auto row_scales = [&](int s) -> words {
      const lds_char* at = scales + (s % Q8_CHUNK) * BM + rm + i * MI;
      if constexpr (MI == 8) return *(const __attribute__((address_space(3))) words*)at;
      else if constexpr (MI == 4) return words{*(const __attribute__((address_space(3))) unsigned*)at};
      else return words{*(const __attribute__((address_space(3))) unsigned short*)at};
    };
    const auto col_scale = [&](int s) -> unsigned {
      return *(const __attribute__((address_space(3))) unsigned char*)(scales + Q8_CHUNK * BM + (n0 % Q8_BLOCK + cn) / Q8_BLOCK * Q8_CHUNK + s % Q8_CHUNK);
    };
    const auto fragment = [&](unsigned from, int r0) -> i8v {
      const lds_char* row = mem + from + (r0 + i) * EMM_STAGE;
      const u4 lo = *(const __attribute__((address_space(3))) u4*)(row + ((q ^ (i & 7)) * 16)), hi = *(const __attribute__((address_space(3))) u4*)(row + (((4 + q) ^ (i & 7)) * 16));
      return i8v{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
    };
    q8_for<LOADS>([&](auto j) { load(j, 0); });
    w += EMM_STAGE;
    if (p.stages > 1) {
      q8_for<LOADS>([&](auto j) { load(j, STAGE); });
      w += EMM_STAGE;
    }
    fill(0);
    // All but the last `left_` loads are in LDS, for all wavefronts, and what any of them has asked LDS for is there.
    const auto meet = [](auto left_) {
      emm_wait<decltype(left_)::value>();
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
    };
    meet(Q8Int<0>{});
    i8v fa[MI], fb[NI];
    fa[0] = fragment(0, rm);
#pragma unroll
    for (int n = 0; n < NI; n++) fb[n] = fragment(BYTES_A, cn + 16 * n);
    words sx = row_scales(0);
    unsigned sw = col_scale(0);
    // stage s, in the buffer at `now`; NEXT: there is another one; MORE: and one behind that
    const auto stage = [&](int s, unsigned now, auto next_, auto more_) {
      constexpr bool NEXT = decltype(next_)::value, MORE = decltype(more_)::value;
      const unsigned then = STAGE - now;
      words nx = sx;
      unsigned nw = sw;
      q8_for<MI>([&](auto m_) {
        constexpr int M = decltype(m_)::value, H = MI / 2;
        if constexpr (M < H) {
          fa[2 * M + 1] = fragment(now, rm + 16 * (2 * M + 1));
          if constexpr (2 * M + 2 < MI) fa[2 * M + 2] = fragment(now, rm + 16 * (2 * M + 2));
        }
        if constexpr (M == H && M + 1 < MI && MORE) meet(Q8Int<LOADS>{});  // (the next stage may be on its way still)
        if constexpr (M + 1 == MI && NEXT) {
          meet(Q8Int<MORE ? EACH * (H - 1) : 0>{});
          if ((s + 1) % Q8_CHUNK == 0) {
            fill(s + 1);
            meet(Q8Int<0>{});
          }
          nx = row_scales(s + 1);
          nw = col_scale(s + 1);
          fa[0] = fragment(then, rm);
        }
        __builtin_amdgcn_sched_barrier(0);
        q8_for<NI>([&](auto n_) {
          constexpr int N = decltype(n_)::value;
          acc[M][N] = q8_mfma<T, 0, M & 3>(fb[N], fa[M], acc[M][N], sw, sx[M / 4]);
          if constexpr (M + 1 == MI && NEXT) fb[N] = fragment(then + BYTES_A, cn + 16 * N);
          if constexpr (M >= H && MORE) {
            constexpr int FIRST = (M - H) * EACH;  // of this step's loads; one behind each NI / EACH columns
            q8_for<EACH>([&](auto x) {
              if constexpr (x.value * NI / EACH == N) load(Q8Int<FIRST + x.value>{}, now);
            });
          }
          if constexpr (M >= H) __builtin_amdgcn_sched_barrier(0);
        });
        __builtin_amdgcn_sched_barrier(0);
      });
      if constexpr (MORE) w += EMM_STAGE;
      sx = nx;
      sw = nw;
    };
    int s = 0;
    unsigned now = 0;
    for (; s + 2 < p.stages; s++) {
      stage(s, now, std::true_type{}, std::true_type{});
      now = STAGE - now;
    }
    if (s + 1 < p.stages) {
      stage(s, now, std::true_type{}, std::false_type{});
      now = STAGE - now;
      s++;
    }
    stage(s, now, std::false_type{}, std::false_type{});
  }
  constexpr int PER = Elem<T>::PER16;
  typedef typename Elem<T>::v16 v16;
  emm_lines_to_lds<T, BN>((lds_char*)lds, acc, rm, cn);
  const auto clamped = [&](v16 v, bool nothing, auto gated, const Pack<T, PER>& gate) {
    if (nothing) v = v16{};  // (a row of zeros)
    if (p.relu) {  // (of what is rounded: the same; NaN and -0 give +0)
#pragma unroll
      for (int x = 0; x < PER; x++) v[x] = static_cast<float>(v[x]) > 0.0f ? v[x] : static_cast<T>(0.0f);
    }
    if constexpr (decltype(gated)::value) {
#pragma unroll
      for (int x = 0; x < PER; x++) v[x] = static_cast<float>(gate.e[x]) > 0.0f ? v[x] : static_cast<T>(0.0f);
    }
    return v;
  };
  constexpr int CHUNKS = BM * BN / PER, EACH_THREAD = CHUNKS / (64 * NW), U = EACH_THREAD < 8 ? EACH_THREAD : 8;
  if (p.NO % PER == 0) {  // U chunks at a time, whose gates and rows are asked for together
    const auto batch = [&](int j0, auto gated) {
      Pack<T, PER> gate[U];
      int row[U], src[U], col[U];
#pragma unroll
      for (int u = 0; u < U; u++) {
        const int x = tid + (j0 + u) * 64 * NW;
        row[u] = m0 + x / (BN / PER);
        col[u] = n0 + x % (BN / PER) * PER;
        const int r = min(row[u], hi - 1);  // (past the end: any that is there)
        src[u] = p.row && owned ? p.row[r] : 0;
        if constexpr (gated.value) gate[u] = load_pack<T, PER>(static_cast<const T*>(p.gate) + (int64_t)r * p.NO + min(col[u], p.NO - PER));
      }
#pragma unroll
      for (int u = 0; u < U; u++) {
        const v16 v = clamped(emm_line<T, BN>((lds_char*)lds, tid + (j0 + u) * 64 * NW), src[u] < 0 || (src[u] >= p.T && owned), gated, gate[u]);
        if (row[u] < hi && col[u] < p.NO) __builtin_nontemporal_store(v, reinterpret_cast<v16*>(static_cast<T*>(p.C) + (int64_t)row[u] * p.NO + col[u]));
      }
    };
    if (p.gate && owned) {
      for (int j0 = 0; j0 < EACH_THREAD; j0 += U) batch(j0, std::true_type{});
    } else {
      for (int j0 = 0; j0 < EACH_THREAD; j0 += U) batch(j0, std::false_type{});
    }
    return;
  }
  for (int x = tid; x < CHUNKS; x += 64 * NW) {
    const int r = m0 + x / (BN / PER), c = n0 + x % (BN / PER) * PER, left = p.NO - c;
    if (r >= hi || left <= 0) continue;
    const int64_t o = (int64_t)r * p.NO + c;
    Pack<T, PER> gate{};
    if (p.gate && owned) {
      const T* const g = static_cast<const T*>(p.gate) + o;
      if (left >= PER) {
        gate = load_pack<T, PER>(g);
      } else {
#pragma unroll
        for (int y = 0; y < PER; y++) gate.e[y] = y < left ? g[y] : static_cast<T>(0.0f);
      }
    }
    const bool nothing = p.row && owned && (p.row[r] < 0 || p.row[r] >= p.T);
    const v16 line = emm_line<T, BN>((lds_char*)lds, x);
    const v16 v = p.gate && owned ? clamped(line, nothing, std::true_type{}, gate) : clamped(line, nothing, std::false_type{}, gate);
    T* const out = static_cast<T*>(p.C) + o;
    if (left >= PER) {
      store_pack<T, PER>(out, __builtin_bit_cast(Pack<T, PER>, v));
    } else {
#pragma unroll
      for (int y = 0; y < PER; y++)
        if (y < left) out[y] = v[y];
    }
  }
}

// A tile of 256 whose expert has 128 rows or fewer left, as every other one has, takes a tile of 128 x 256 instead (0.58 of its time), and these come after the whole ones:
// an XCD's compute units start on them as they get free, not on a last whole tile each.  Uneven shares, (E,R,N,K), us, before and after: (32,16384,4096,2048) 202 and 187,
// (8,16384,2048,4096) 178 and 165, (32,32768,2048,4096) 319 and 302, (64,16384,2048,2048) 114 both; in the order of the experts 202, 178, 316, 115.
template <typename T, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void expert_mm_q8_kernel(Q8Args p) {
  __shared__ __align__(16) char lds[q8_tile_lds<T, BM, BN>()];
  ExpertTile t;
  if (BM == 256 && p.off) {
    unsigned run;
    if (!expert_tile<TILES_FULL>(p.off, p.E, p.R, BM, p.nt, blockIdx.x, &t, &run) &&
        (blockIdx.x / 8 < run || !expert_tile<TILES_SHORT>(p.off, p.E, p.R, BM, p.nt, blockIdx.x - 8 * run, &t)))
      return;
  } else if (!q8_tile(p, BM, &t)) {
    return;
  }
  const int lo = __builtin_amdgcn_readfirstlane(t.lo), hi = __builtin_amdgcn_readfirstlane(t.hi), e = __builtin_amdgcn_readfirstlane(t.e);
  const int m0 = lo + __builtin_amdgcn_readfirstlane(t.m) * BM, n0 = __builtin_amdgcn_readfirstlane(t.n) * BN;
  if constexpr (BM == 256) {
    if (hi - m0 <= BM / 2) return q8_tile_product<T, BM / 2, BN, WM, WN>(p, lds, e, m0, hi, n0);
  }
  q8_tile_product<T, BM, BN, WM, WN>(p, lds, e, m0, hi, n0);
}

// Few rows an expert (a decoding step): 16 rows by 16 CT columns a workgroup, whose wavefronts share the reduction; operands go from memory to registers in the
// matrix instruction's layout, as in expert_rows.hpp.
constexpr int Q8_AHEAD = 4;  // stages in flight of a wavefront

template <typename T, int CT, int WK>
__global__ __launch_bounds__(64 * WK) void expert_few_rows_q8_kernel(Q8Args p) {
  constexpr int U = Q8_AHEAD;
  __shared__ __align__(16) f4 part[WK][CT][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15, q = lane >> 4;
  ExpertTile t;
  if (!q8_tile(p, 16, &t)) return;
  const int hi = __builtin_amdgcn_readfirstlane(t.hi), e = __builtin_amdgcn_readfirstlane(t.e);
  const int m0 = __builtin_amdgcn_readfirstlane(t.lo) + __builtin_amdgcn_readfirstlane(t.m) * 16, n0 = __builtin_amdgcn_readfirstlane(t.n) * (16 * CT);
  const bool owned = e < p.E && p.T > 0;
  f4 acc[CT];
#pragma unroll
  for (int n = 0; n < CT; n++) acc[n] = f4{0, 0, 0, 0};
  if (owned) {
    const int first = (int)((int64_t)p.stages * wave / WK), last = (int)((int64_t)p.stages * (wave + 1) / WK);
    const int64_t ld = (int64_t)p.stages * EMM_STAGE;
    const int r = min(m0 + i, hi - 1);
    const int64_t src = p.row ? min(max(p.row[r], 0), p.T - 1) : r;
    const unsigned char *a = p.A + src * ld + (int64_t)first * EMM_STAGE + 16 * q, *sa = p.SA + src * p.stages;
    const unsigned char* b[CT];
#pragma unroll
    for (int n = 0; n < CT; n++) b[n] = p.W + ((int64_t)e * p.NO + min(n0 + 16 * n + i, p.NO - 1)) * ld + (int64_t)first * EMM_STAGE + 16 * q;
    const int nb = (p.NO + Q8_BLOCK - 1) / Q8_BLOCK;
    const unsigned char* const sw = p.SW + ((int64_t)e * nb + min(n0 / Q8_BLOCK, nb - 1)) * p.stages;  // (all columns' block)
    const auto load = [](const unsigned char* x) {
      const u4 lo = *reinterpret_cast<const u4*>(x), hi = *reinterpret_cast<const u4*>(x + 64);
      return i8v{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
    };
    for (int s = first; s < last; s += U) {
      i8v fb[U][CT], fa[U];
      unsigned xs[U], ws[U];
#pragma unroll
      for (int u = 0; u < U; u++) {
        const int at = min(u, last - 1 - s);  // (past the last stage: that one again, so that loads stay inside; its products are left out below)
#pragma unroll
        for (int n = 0; n < CT; n++) fb[u][n] = load(b[n] + at * EMM_STAGE);
        fa[u] = load(a + at * EMM_STAGE);
        xs[u] = sa[s + at];
        ws[u] = sw[s + at];
      }
#pragma unroll
      for (int u = 0; u < U; u++)
        if (s + u < last) {
#pragma unroll
          for (int n = 0; n < CT; n++) acc[n] = q8_mfma<T, 0, 0>(fb[u][n], fa[u], acc[n], ws[u], xs[u]);
        }
#pragma unroll
      for (int n = 0; n < CT; n++) b[n] += U * EMM_STAGE;
      a += U * EMM_STAGE;
    }
  }
#pragma unroll
  for (int n = 0; n < CT; n++) part[wave][n][lane] = acc[n];
  __syncthreads();
  const bool by4 = (p.NO & 3) == 0;
  for (int n = wave; n < CT; n += WK) {
    const int r = m0 + i, c = n0 + 16 * n + 4 * q;
    f4 v = part[0][n][lane];
#pragma unroll
    for (int w = 1; w < WK; w++) v += part[w][n][lane];
    if (r >= hi || c >= p.NO) continue;
    if (p.row && owned && (p.row[r] < 0 || p.row[r] >= p.T)) v = f4{0, 0, 0, 0};  // (a row of zeros)
    const int64_t o = (int64_t)r * p.NO + c;
#pragma unroll
    for (int x = 0; x < 4; x++) {
      if (p.relu) v[x] = v[x] > 0.0f ? v[x] : 0.0f;  // (NaN and -0 give +0)
      if (p.gate && owned && c + x < p.NO && !(static_cast<float>(static_cast<const T*>(p.gate)[o + x]) > 0.0f)) v[x] = 0.0f;
    }
    emm_store(static_cast<T*>(p.C) + o, p.NO - c, by4, v);
  }
}

}  // namespace tc355
