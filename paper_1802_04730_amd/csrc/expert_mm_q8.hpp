// Products grouped by expert of rows and weights in 8 bits (quantize8.hpp):
//   Y(r,n) = act(sum_b 2^(SX(s,b) + SW(e,n/128,b) - 254) sum_{k of block b} X(s,k) W(e,n,k)),  s = src(r)
// With the transposed form of the weights it is the gradient of the rows too.  What bounds it: 2 R N K operations on the 8-bit matrix core; the weights' bytes where an
// expert has few rows.
//
// Tiles, stages of 128 bytes, their way to LDS and the swizzle are expert_mm.hpp's.  A stage is a block of 128 elements: one matrix instruction of 16 x 16 x 128
// takes a whole stage, with the scales' bytes as operands, so that scaling costs nothing.  A lane's 32 bytes of a row are the chunks q and 4 + q: which elements those are is
// all the same, as long as both operands agree.  While one half of a wavefront's rows is multiplied, the other half's fragments are read.
//
// The 8-bit matrix instruction adds the products of 8 neighbours with the bits down to 2^-13 of the largest one's exponent and cuts the rest; beyond these
// groups its sums keep 24 bits (measured with products that cancel).  So up to 2^-10 of a group's largest product is lost -- operands in e4m3 are
// off by 2^-4 of their own --, a choice for 16-bit outputs, whose rounding is as coarse (2^-16 of an output's norm with normally distributed operands; bfloat16 keeps 2^-9): its rate is over
// three times the 16-bit instruction's (3.8 PFLOP/s against 1.2, both from registers).  float outputs go by the half instruction instead, which takes the same
// values, widened, and sums them in 32 bits.
#pragma once
#include "expert_mm.hpp"
#include "quantize8.hpp"

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

// acc += the products of a stage: w and x 32 bytes of a row each, sw and sx their scales' lowest bytes.
template <typename T>
__device__ __forceinline__ f4 q8_mfma(const i8v& w, const i8v& x, f4 acc, unsigned sw, unsigned sx) {
  if constexpr (sizeof(T) == 2) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, acc, 0, 0, 0, (int)sw, 0, (int)sx);
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
    const int a = (int)(sw & 255), b = (int)(sx & 255);
    const bool nan = a == (int)Q8_NAN || b == (int)Q8_NAN;
#pragma unroll
    for (int v = 0; v < 4; v++) acc[v] += nan ? __builtin_nanf("") : __builtin_amdgcn_ldexpf(sum[v], a + b - 254);
    return acc;
  }
}

// The fragments of M blocks of 16 rows from row r0 on.
template <int M>
__device__ __forceinline__ void q8_fragments(const lds_char* lds, int r0, int i, int q, i8v (&f)[M]) {
#pragma unroll
  for (int m = 0; m < M; m++) {
    const char __attribute__((address_space(3)))* row = lds + (r0 + 16 * m + i) * EMM_STAGE;
    const u4 lo = *(const __attribute__((address_space(3))) u4*)(row + ((q ^ (i & 7)) * 16)), hi = *(const __attribute__((address_space(3))) u4*)(row + (((4 + q) ^ (i & 7)) * 16));
    f[m] = i8v{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
  }
}

// ROWS rows of 128 bytes a stage to LDS, 8 rows an instruction, NW wavefronts; rows lie anywhere.
template <int ROWS, int NW>
struct Q8Rows {
  static constexpr int BYTES = ROWS * EMM_STAGE, PER = ROWS / 8 / NW;
  static_assert(PER * 8 * NW == ROWS, "whole instructions");
  const char* p[PER];
  template <typename F>
  __device__ __forceinline__ void begin(const unsigned char* b, int64_t ld, int wave, int lane, F row) {
#pragma unroll
    for (int j = 0; j < PER; j++) p[j] = reinterpret_cast<const char*>(b) + row((wave * PER + j) * 8 + (lane >> 3)) * ld + ((lane & 7) ^ (lane >> 3)) * 16;
  }
  __device__ __forceinline__ void to_lds(lds_char* lds, int wave) {
#pragma unroll
    for (int j = 0; j < PER; j++) {
      emm_to_lds(p[j], lds + (wave * PER + j) * 1024);
      p[j] += EMM_STAGE;
    }
  }
};

// Reads of the next fragments and loads of a later stage.  (Restricted pointers of a function of their own, as emm_traffic's.)
template <int MH, int NI, typename A, typename B>
__device__ __forceinline__ void q8_traffic(A& a, B& b, const lds_char* __restrict__ now, lds_char* __restrict__ then, bool rows, bool cols, bool more, int rm, int cn, int wave,
                                           int lane, i8v (&fa)[MH], i8v (&fb)[NI]) {
  if (more) {
    a.to_lds(then, wave);
    b.to_lds(then + A::BYTES, wave);
  }
  if (cols) q8_fragments<NI>(now + A::BYTES, cn, lane & 15, lane >> 4, fb);
  if (rows) q8_fragments<MH>(now, rm, lane & 15, lane >> 4, fa);
}

template <typename T, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void expert_mm_q8_kernel(Q8Args p) {
  constexpr int NW = WM * WN, MI = BM / WM / 16, NI = BN / WN / 16, MH = MI / 2;
  static_assert(MH * 2 == MI, "two halves");
  typedef Q8Rows<BM, NW> OpA;
  typedef Q8Rows<BN, NW> OpB;
  constexpr int STAGE = OpA::BYTES + OpB::BYTES, LOADS = OpA::PER + OpB::PER;
  constexpr int OUT = BM * BN * sizeof(T);
  __shared__ __align__(16) char lds[2 * STAGE > OUT ? 2 * STAGE : OUT];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = lane & 15;
  ExpertTile t;
  if (!q8_tile(p, BM, &t)) return;
  const int lo = __builtin_amdgcn_readfirstlane(t.lo), hi = __builtin_amdgcn_readfirstlane(t.hi), e = __builtin_amdgcn_readfirstlane(t.e);
  const int m0 = lo + __builtin_amdgcn_readfirstlane(t.m) * BM, n0 = __builtin_amdgcn_readfirstlane(t.n) * BN;
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
    OpA a;
    OpB b;
    a.begin(p.A, ld, wave, lane, source);
    const int most = p.NO - 1 - n0;
    b.begin(p.W + ((int64_t)e * p.NO + n0) * ld, ld, wave, lane, [&](int j) -> int64_t { return min(j, most); });
    // scales: four stages' in a word, of this lane's rows and of the wavefront's columns (which share a block)
    const unsigned char* sa[MI];
#pragma unroll
    for (int m = 0; m < MI; m++) sa[m] = p.SA + source(rm + 16 * m + i) * p.stages;
    const int nb = (p.NO + Q8_BLOCK - 1) / Q8_BLOCK;
    const unsigned char* const sw = p.SW + ((int64_t)e * nb + min((n0 + cn) / Q8_BLOCK, nb - 1)) * p.stages;
    unsigned va[MI], vw, na[MI], nw;
#pragma unroll
    for (int m = 0; m < MI; m++) na[m] = q8_scales(sa[m], 0, p.stages);
    nw = q8_scales(sw, 0, p.stages);
    i8v fa[2][MH], fb[2][NI];
    lds_char* const mem = (lds_char*)lds;
    a.to_lds(mem, wave);
    b.to_lds(mem + OpA::BYTES, wave);
    if (p.stages > 1) {
      a.to_lds(mem + STAGE, wave);
      b.to_lds(mem + STAGE + OpA::BYTES, wave);
      emm_wait<LOADS>();
    } else {
      emm_wait<0>();
    }
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    q8_traffic<MH, NI>(a, b, mem, mem, true, true, false, rm, cn, wave, lane, fa[0], fb[0]);
    const auto stage = [&](int s, lds_char* now, lds_char* next, i8v (&f)[NI], i8v (&g)[NI]) {
      if ((s & 3) == 0) {
#pragma unroll
        for (int m = 0; m < MI; m++) va[m] = na[m];
        vw = nw;
        if (s + 4 < p.stages) {
#pragma unroll
          for (int m = 0; m < MI; m++) na[m] = q8_scales(sa[m], s + 4, p.stages);
          nw = q8_scales(sw, s + 4, p.stages);
        }
      }
      q8_traffic<MH, NI>(a, b, now, now, true, false, false, rm + 16 * MH, cn, wave, lane, fa[1], g);
#pragma unroll
      for (int m = 0; m < MH; m++)
#pragma unroll
        for (int n = 0; n < NI; n++) acc[m][n] = q8_mfma<T>(f[n], fa[0][m], acc[m][n], vw, va[m]);
      emm_wait<0>();
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_s_barrier();  // the next stage is in LDS, and everyone has read this one
      asm volatile("" ::: "memory");
      q8_traffic<MH, NI>(a, b, next, now, s + 1 < p.stages, s + 1 < p.stages, s + 2 < p.stages, rm, cn, wave, lane, fa[0], g);
#pragma unroll
      for (int m = 0; m < MH; m++)
#pragma unroll
        for (int n = 0; n < NI; n++) acc[MH + m][n] = q8_mfma<T>(f[n], fa[1][m], acc[MH + m][n], vw, va[MH + m]);
#pragma unroll
      for (int m = 0; m < MI; m++) va[m] >>= 8;
      vw >>= 8;
    };
    int s = 0;
    for (; s + 1 < p.stages; s += 2) {
      stage(s, mem, mem + STAGE, fb[0], fb[1]);
      stage(s + 1, mem + STAGE, mem, fb[1], fb[0]);
    }
    if (s < p.stages) stage(s, mem, mem + STAGE, fb[0], fb[1]);
  }
  constexpr int PER = Elem<T>::PER16;
  typedef typename Elem<T>::v16 v16;
  if (p.relu) {
#pragma unroll
    for (int m = 0; m < MI; m++)
#pragma unroll
      for (int n = 0; n < NI; n++)
#pragma unroll
        for (int x = 0; x < 4; x++) acc[m][n][x] = acc[m][n][x] > 0.0f ? acc[m][n][x] : 0.0f;  // (NaN and -0 give +0)
  }
  emm_store_lines<T, BM, BN, 64 * NW>((lds_char*)lds, acc, rm, cn, [&](int row, int col, v16 v) {
    const int r = m0 + row, c = n0 + col, left = p.NO - c;
    if (r >= hi || left <= 0) return;
    const int64_t o = (int64_t)r * p.NO + c;
    if (p.row && owned && (p.row[r] < 0 || p.row[r] >= p.T)) v = v16{};  // (a row of zeros)
    if (p.gate && owned) {
      const T* const gate = static_cast<const T*>(p.gate) + o;
      Pack<T, PER> h;
      if (left >= PER) {
        h = load_pack<T, PER>(gate);
      } else {
#pragma unroll
        for (int x = 0; x < PER; x++) h.e[x] = x < left ? gate[x] : static_cast<T>(0.0f);
      }
#pragma unroll
      for (int x = 0; x < PER; x++) v[x] = static_cast<float>(h.e[x]) > 0.0f ? v[x] : static_cast<T>(0.0f);
    }
    T* const out = static_cast<T*>(p.C) + o;
    if (left >= PER) {
      store_pack<T, PER>(out, __builtin_bit_cast(Pack<T, PER>, v));
    } else {
#pragma unroll
      for (int x = 0; x < PER; x++)
        if (x < left) out[x] = v[x];
    }
  });
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
        const int at = min(u, last - 1 - s);  // (past the last stage: that one again, by the scale of nothing)
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
          for (int n = 0; n < CT; n++) acc[n] = q8_mfma<T>(fb[u][n], fa[u], acc[n], ws[u], xs[u]);
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
