// Products grouped by expert: expert e owns the rows Off(e) .. Off(e+1) of a matrix of R rows, as many as a router gave it.
//   Y(r,n)    = act(sum_k X(src(r),k) * W(e(r),n,k))         rows kernel, both operands along their rows
//   dX(r,k)   = gate(r,k) * sum_n dY(r,n) * W(e(r),n,k)      rows kernel, W across its rows
//   dW(e,n,k) = sum_{r of e} dY(r,n) * X(src(r),k)           weights kernel, both operands across their rows
// What bounds them: 2 R N K operations each on the matrix core, unless an expert has so few rows that its weights' bytes do
// (expert_rows.hpp takes those).
//
// A workgroup computes a BM x BN tile of one expert.  In a stage both operands' next 128 bytes of the reduction (64 elements of 16
// bits, 32 of 32) go straight from memory to LDS, 16 bytes per lane, while the stage before is multiplied: two buffers, one
// barrier a stage.  The fragments of a stage are all read before the next stage's loads are issued: the compiler, which knows of
// the loads to LDS, would wait for them before any LDS read that follows.
//
// Layout in LDS.  Along its rows an operand is [rows][128 bytes]; the 16-byte chunk c of row r lies in slot c ^ (r & 7), so that
// the 16 rows of a fragment read hit all banks.  Across its rows it is [reduction][tile columns]: 16-bit elements are
// read by the transposing LDS read (four rows of 16 columns to 16 lanes of four), 32-bit ones word by word; chunks are swizzled by
// the rows that one instruction reads together.  Lane (i = lane % 16, q = lane / 16) of a matrix instruction supplies row i and, of the
// reduction, elements 8q .. 8q+7 of 32 (16 bits) or, in 4 instructions, 4q .. 4q+3 of 16 (32 bits): the order is free as long as
// both operands keep it.  The operands are exchanged (weights first), so that a lane's four results are neighbours in a row of the output.
//
// Sums are fp32 in the matrix core's accumulators whatever the storage, and each output is rounded once.
#pragma once
#include "expert_types.hpp"

namespace tc355 {

constexpr int EMM_STAGE = 128;  // bytes of the reduction per stage and row

static __device__ __align__(16) const unsigned emm_zeros[4] = {0, 0, 0, 0};  // what stands for elements that are not there

template <int N>
__device__ __forceinline__ void emm_wait() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void emm_to_lds(const char* g, unsigned lds) {  // lane l's 16 bytes to lds + 16 l (a uniform address)
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(uintptr_t)g,
                                   (__attribute__((address_space(3))) void*)(uintptr_t)lds, 16, 0, 0);
}
__device__ __forceinline__ unsigned lds_address(const void* p) {
  return (unsigned)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}

// ---- which rows a tile takes ------------------------------------------------------------------------------------------

struct ExpertTile {
  int e;       // expert; E: the rows that no expert owns
  int lo, hi;  // its rows
  int m, n;    // tile of the expert, in rows and columns
};

// Tile `at` of all, or false.  Off is the device's: whatever it holds, rows stay inside [0, R).  Tiles of one expert follow each
// other in blocks of 8 row tiles by all column tiles, row tiles first, so that workgroups that run together share operands; and every
// XCD (workgroups equal modulo 8) takes a run of its own.
__device__ __forceinline__ bool expert_tile(const int* off, int E, int R, int bm, int nt, unsigned bid, ExpertTile* t) {
  const int lane = threadIdx.x & 63;
  unsigned total = 0;
  for (int base = 0; base <= E; base += 64) {
    const int g = base + lane;
    int c = 0;
    if (g <= E) c = (g < E ? min(max(off[g + 1], 0), R) : R) - min(max(off[g], 0), R);
    unsigned n = c > 0 ? (unsigned)((c + bm - 1) / bm) * nt : 0;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) n += __shfl_xor(n, d);
    total += n;
  }
  const unsigned run = (total + 7) / 8;
  if (bid / 8 >= run) return false;
  const unsigned at = (bid & 7) * run + bid / 8;
  if (at >= total) return false;
  unsigned before = 0;
  for (int base = 0; base <= E; base += 64) {
    const int g = base + lane;
    int lo = 0, hi = 0;
    if (g <= E) {
      lo = min(max(off[g], 0), R);
      hi = g < E ? min(max(off[g + 1], 0), R) : R;
    }
    const unsigned n = hi > lo ? (unsigned)((hi - lo + bm - 1) / bm) * nt : 0;
    unsigned incl = n;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const unsigned o = __shfl_up(incl, d);
      if (lane >= d) incl += o;
    }
    const unsigned long long past = __ballot(at < before + incl);
    if (past) {
      const int src = __ffsll((long long)past) - 1;
      const unsigned local = at - before - __shfl(incl - n, src);
      t->e = base + src;
      t->lo = __shfl(lo, src);
      t->hi = __shfl(hi, src);
      const int mt = (t->hi - t->lo + bm - 1) / bm;
      const int block = (int)(local / (unsigned)(8 * nt)), in = (int)(local % (unsigned)(8 * nt));
      const int rows = min(8, mt - 8 * block);
      t->m = 8 * block + in % rows;
      t->n = in / rows;
      return true;
    }
    before += __shfl(incl, 63);
  }
  return false;
}

// ---- operands: memory to LDS, LDS to fragments ------------------------------------------------------------------------

// 16 bytes of a row from element `at` on, of which `left` elements are there.
template <typename T>
__device__ __forceinline__ u4 emm_load_any(const T* p, int left) {
  constexpr int PER = Elem<T>::PER16;
  Any16<T> v;
  if (left >= PER) {
    v = load16(p);
  } else {
#pragma unroll
    for (int i = 0; i < PER; i++) v.e[i] = i < left ? p[i] : static_cast<T>(0.0f);
  }
  return __builtin_bit_cast(u4, v);
}

// Operand along its rows: ROWS rows of the tile, 128 bytes of the reduction a stage.  NW wavefronts load it, 8 rows an instruction.
template <typename T, int ROWS, int NW>
struct AlongRows {
  static constexpr int BYTES = ROWS * EMM_STAGE;
  static constexpr int PER = ROWS / 8 / NW;  // instructions of a wavefront
  static constexpr int BK = EMM_STAGE / sizeof(T);
  static_assert(PER * 8 * NW == ROWS, "whole instructions");
  const T* p[PER];  // this lane's row, at its chunk of the first stage; nullptr: a row of zeros
  int at;           // element of the reduction where the chunk begins
  int Q;
  u4 held[PER];

  // row(j): the source row of row j of the tile, or -1
  template <typename F>
  __device__ __forceinline__ void begin(const T* base, int64_t ld, int q, int wave, int lane, F row) {
    Q = q;
    at = ((lane & 7) ^ (lane >> 3)) * Elem<T>::PER16;  // (row & 7 = lane / 8)
#pragma unroll
    for (int j = 0; j < PER; j++) {
      const int64_t r = row((wave * PER + j) * 8 + (lane >> 3));
      p[j] = r < 0 ? nullptr : base + r * ld + at;
    }
  }
  __device__ __forceinline__ void to_lds(unsigned lds, int wave) {
    const bool in = at < Q;
#pragma unroll
    for (int j = 0; j < PER; j++) {
      const char* src = in && p[j] ? reinterpret_cast<const char*>(p[j]) : reinterpret_cast<const char*>(emm_zeros);
      emm_to_lds(src, lds + (wave * PER + j) * 1024);
    }
    next();
  }
  __device__ __forceinline__ void hold() {
#pragma unroll
    for (int j = 0; j < PER; j++) {
      held[j] = u4{0, 0, 0, 0};
      if (p[j] && at < Q) held[j] = emm_load_any(p[j], Q - at);
    }
    next();
  }
  __device__ __forceinline__ void put(char* lds, int wave, int lane) {
#pragma unroll
    for (int j = 0; j < PER; j++) *reinterpret_cast<u4*>(lds + (wave * PER + j) * 1024 + lane * 16) = held[j];
  }
  __device__ __forceinline__ void next() {
    at += BK;
#pragma unroll
    for (int j = 0; j < PER; j++) p[j] = p[j] ? p[j] + BK : nullptr;
  }
  // 16 bytes of row r of the tile, chunk 4 s + q
  static __device__ __forceinline__ const char* chunk(const char* lds, int r, int s, int q) {
    return lds + r * EMM_STAGE + (((4 * s + q) ^ (r & 7)) * 16);
  }
};

// Operand across its rows: BK rows of the reduction a stage, COLS columns of the tile.
template <typename T, int COLS, int NW>
struct AcrossRows {
  static constexpr int BK = EMM_STAGE / sizeof(T);
  static constexpr int BYTES = BK * COLS * sizeof(T);
  static constexpr int CPR = COLS * sizeof(T) / 16;  // chunks of a row
  static constexpr int RPI = 64 / CPR;               // rows of an instruction
  static constexpr int PER = BK / RPI / NW;
  static_assert(RPI * CPR == 64 && PER * RPI * NW == BK, "whole instructions");
  const T* base;  // column 0 of the reduction's row 0
  const int* row; // rows of `base` that the reduction goes through, or nullptr: all of them in order
  int64_t ld;
  int q0, Q, rows;  // row of the reduction that the next stage begins with; their number; rows of `base`
  int left[PER];    // (any alignment) elements of the row from the chunk on
  int col[PER];
  int src[PER];
  u4 held[PER];

  // rows that one instruction reads together have different chunks of 64 banks
  static __device__ __forceinline__ int swizzle(int r) {
    if constexpr (sizeof(T) == 2) return 2 * ((r & 3) | ((r >> 1) & 4));
    else return 4 * ((r >> 2) & 3);
  }
  __device__ __forceinline__ int at(int j, int wave, int lane) const { return (wave * PER + j) * RPI + lane / CPR; }

  __device__ __forceinline__ void begin(const T* b, int64_t stride, const int* rw, int q, int total, int c0, int cols, int wave, int lane) {
    base = b;
    row = rw;
    ld = stride;
    q0 = 0;
    Q = q;
    rows = total;
#pragma unroll
    for (int j = 0; j < PER; j++) {
      col[j] = c0 + ((lane % CPR) ^ swizzle(at(j, wave, lane))) * Elem<T>::PER16;
      left[j] = cols - col[j];
    }
    look(wave, lane);
  }
  // the source rows of the stage at q0, -1: zeros
  __device__ __forceinline__ void look(int wave, int lane) {
#pragma unroll
    for (int j = 0; j < PER; j++) {
      const int q = q0 + at(j, wave, lane);
      src[j] = -1;
      if (q < Q) src[j] = row ? row[q] : q;
    }
  }
  __device__ __forceinline__ bool there(int j) const { return src[j] >= 0 && src[j] < rows && left[j] > 0; }
  __device__ __forceinline__ void to_lds(unsigned lds, int wave, int lane) {
#pragma unroll
    for (int j = 0; j < PER; j++) {
      const char* s = there(j) ? reinterpret_cast<const char*>(base + (int64_t)src[j] * ld + col[j]) : reinterpret_cast<const char*>(emm_zeros);
      emm_to_lds(s, lds + (wave * PER + j) * 1024);
    }
    q0 += BK;
    look(wave, lane);
  }
  __device__ __forceinline__ void hold(int wave, int lane) {
#pragma unroll
    for (int j = 0; j < PER; j++) {
      held[j] = u4{0, 0, 0, 0};
      if (there(j)) held[j] = emm_load_any(base + (int64_t)src[j] * ld + col[j], left[j]);
    }
    q0 += BK;
    look(wave, lane);
  }
  __device__ __forceinline__ void put(char* lds, int wave, int lane) {
#pragma unroll
    for (int j = 0; j < PER; j++) *reinterpret_cast<u4*>(lds + (wave * PER + j) * 1024 + lane * 16) = held[j];
  }
  // 16 bits: rows 32 s + 8 q + 4 h + (0..3), columns c .. c+15: this lane's address of the transposing read
  static __device__ __forceinline__ unsigned four(unsigned lds, int c, int s, int h, int i, int q) {
    const int r = 32 * s + 8 * q + 4 * h + (i >> 2), cc = c + (i & 3) * 4;
    return lds + r * (COLS * 2) + (((cc >> 3) ^ swizzle(r)) * 16) + (cc & 7) * 2;
  }
  // 32 bits: row 16 s + 4 q + e, column c
  static __device__ __forceinline__ float word(const char* lds, int c, int s, int e, int q) {
    const int r = 16 * s + 4 * q + e;
    return *reinterpret_cast<const float*>(lds + r * (COLS * 4) + (((c >> 2) ^ swizzle(r)) * 16) + (c & 3) * 4);
  }
};

// A fragment: 16 rows (or columns) of the tile by 64 bytes of the reduction, 16 bytes a lane.
template <typename T, int ROWS, int NW>
__device__ __forceinline__ u4 emm_fragment(const AlongRows<T, ROWS, NW>&, const char* lds, int r0, int s, int i, int q) {
  return *reinterpret_cast<const u4*>(AlongRows<T, ROWS, NW>::chunk(lds, r0 + i, s, q));
}
template <typename T, int COLS, int NW>
__device__ __forceinline__ u4 emm_fragment(const AcrossRows<T, COLS, NW>&, const char* lds, int c0, int s, int i, int q) {
  if constexpr (sizeof(T) == 2) {
    typedef __attribute__((address_space(3))) s4v* at;
    const unsigned base = lds_address(lds);
    const s4v a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((at)(uintptr_t)AcrossRows<T, COLS, NW>::four(base, c0, s, 0, i, q));
    const s4v b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((at)(uintptr_t)AcrossRows<T, COLS, NW>::four(base, c0, s, 1, i, q));
    return __builtin_bit_cast(u4, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
  } else {
    f4 v;
#pragma unroll
    for (int e = 0; e < 4; e++) v[e] = AcrossRows<T, COLS, NW>::word(lds, c0 + i, s, e, q);
    return __builtin_bit_cast(u4, v);
  }
}

template <typename T>
__device__ __forceinline__ f4 emm_mfma(u4 a, u4 b, f4 c) {
  if constexpr (sizeof(T) == 4) {
    const f4 x = __builtin_bit_cast(f4, a), y = __builtin_bit_cast(f4, b);
#pragma unroll
    for (int e = 0; e < 4; e++) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], y[e], c, 0, 0, 0);
    return c;
  } else if constexpr (__is_same(T, bf16)) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(Elem<bf16>::v8, a), __builtin_bit_cast(Elem<bf16>::v8, b), c, 0, 0, 0);
  } else {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(Elem<f16>::v8, a), __builtin_bit_cast(Elem<f16>::v8, b), c, 0, 0, 0);
  }
}

// ---- the loop over the reduction ----------------------------------------------------------------------------------------

// MI x NI blocks of 16 x 16 per wavefront, at row rm and column cn of the tile.
template <typename T, bool ANY, int MI, int NI, typename A, typename B>
__device__ __forceinline__ void emm_stage(const A& a, const B& b, const char* la, const char* lb, int rm, int cn, int i, int q, u4 (&fa)[2][MI], u4 (&fb)[2][NI]) {
#pragma unroll
  for (int s = 0; s < 2; s++) {
#pragma unroll
    for (int m = 0; m < MI; m++) fa[s][m] = emm_fragment(a, la, rm + 16 * m, s, i, q);
#pragma unroll
    for (int n = 0; n < NI; n++) fb[s][n] = emm_fragment(b, lb, cn + 16 * n, s, i, q);
  }
}

template <typename A>
struct EmmIsAcross {
  static constexpr bool value = false;
};
template <typename T, int C, int NW>
struct EmmIsAcross<AcrossRows<T, C, NW>> {
  static constexpr bool value = true;
};

template <typename A>
__device__ __forceinline__ void emm_to_lds(A& a, unsigned lds, int wave, int lane) {
  if constexpr (EmmIsAcross<A>::value) a.to_lds(lds, wave, lane);
  else a.to_lds(lds, wave);
}
template <typename A>
__device__ __forceinline__ void emm_hold(A& a, int wave, int lane) {
  if constexpr (EmmIsAcross<A>::value) a.hold(wave, lane);
  else a.hold();
}

template <typename T, bool ANY, int MI, int NI, typename A, typename B>
__device__ __forceinline__ void emm_loop(A& a, B& b, char* lds, int stages, int rm, int cn, int wave, int lane, f4 (&acc)[MI][NI]) {
  constexpr int STAGE = A::BYTES + B::BYTES;
  const int i = lane & 15, q = lane >> 4;
  const unsigned base = lds_address(lds);
#pragma unroll
  for (int m = 0; m < MI; m++)
#pragma unroll
    for (int n = 0; n < NI; n++) acc[m][n] = f4{0, 0, 0, 0};
  if (stages <= 0) return;
  if constexpr (ANY) {
    emm_hold(a, wave, lane);
    emm_hold(b, wave, lane);
    a.put(lds, wave, lane);
    b.put(lds + A::BYTES, wave, lane);
  } else {
    emm_to_lds(a, base, wave, lane);
    emm_to_lds(b, base + A::BYTES, wave, lane);
  }
  for (int t = 0; t < stages; t++) {
    char* now = lds + (t & 1) * STAGE;
    emm_wait<0>();
    __syncthreads();  // this stage is in LDS, and everyone has read the one before
    u4 fa[2][MI], fb[2][NI];
    emm_stage<T, ANY, MI, NI>(a, b, now, now + A::BYTES, rm, cn, i, q, fa, fb);
    __builtin_amdgcn_sched_barrier(0);
    if (t + 1 < stages) {
      if constexpr (ANY) {
        emm_hold(a, wave, lane);
        emm_hold(b, wave, lane);
      } else {
        const unsigned then = base + ((t + 1) & 1) * STAGE;
        emm_to_lds(a, then, wave, lane);
        emm_to_lds(b, then + A::BYTES, wave, lane);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int s = 0; s < 2; s++)
#pragma unroll
      for (int m = 0; m < MI; m++)
#pragma unroll
        for (int n = 0; n < NI; n++) acc[m][n] = emm_mfma<T>(fb[s][n], fa[s][m], acc[m][n]);
    if constexpr (ANY) {
      if (t + 1 < stages) {
        char* then = lds + ((t + 1) & 1) * STAGE;
        a.put(then, wave, lane);
        b.put(then + A::BYTES, wave, lane);
      }
    }
  }
}

// Four neighbours of an output row from column n on, of which `left` are there.
template <typename TO>
__device__ __forceinline__ void emm_store(TO* p, int left, bool whole, f4 v) {
  if (whole) {
    typename Elem<TO>::v4 o;
#pragma unroll
    for (int e = 0; e < 4; e++) o[e] = narrow<TO>(v[e]);
    *reinterpret_cast<typename Elem<TO>::v4*>(p) = o;
  } else {
#pragma unroll
    for (int e = 0; e < 4; e++)
      if (e < left) p[e] = narrow<TO>(v[e]);
  }
}

// ---- kernels ---------------------------------------------------------------------------------------------------------------

struct ExpertRowsArgs {
  const void* A;     // rows: [T][Q], taken through `row`, or [R][Q]
  const void* W;     // [E][N][K]
  void* C;           // [R][NO]
  const void* gate;  // [R][NO] or nullptr
  const int* off;    // [E+1]
  const int* row;    // [R] or nullptr
  int R, T, E, Q, NO;
  int nt;            // column tiles
  int relu;
};

// ACROSS: the weights' rows are the reduction (dX), else they are the output's columns (Y).
template <typename T, bool ACROSS, bool ANY, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void expert_rows_tile_kernel(ExpertRowsArgs p) {
  constexpr int NW = WM * WN, MI = BM / WM / 16, NI = BN / WN / 16;
  typedef AlongRows<T, BM, NW> OpA;
  typedef std::conditional_t<ACROSS, AcrossRows<T, BN, NW>, AlongRows<T, BN, NW>> OpB;
  __shared__ __align__(16) char lds[2 * (OpA::BYTES + OpB::BYTES)];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  ExpertTile t;
  if (!expert_tile(p.off, p.E, p.R, BM, p.nt, blockIdx.x, &t)) return;
  const int lo = __builtin_amdgcn_readfirstlane(t.lo), hi = __builtin_amdgcn_readfirstlane(t.hi), e = __builtin_amdgcn_readfirstlane(t.e);
  const int m0 = lo + __builtin_amdgcn_readfirstlane(t.m) * BM, n0 = __builtin_amdgcn_readfirstlane(t.n) * BN;
  const int rm = (wave / WN) * (BM / WM), cn = (wave % WN) * (BN / WN);
  f4 acc[MI][NI];
  OpA a;
  OpB b;
  const int64_t ldw = ACROSS ? p.NO : p.Q;
  const bool owned = e < p.E;
  if (owned) {
    const int* row = p.row;
    const int last = hi - 1, total = p.T;
    a.begin(static_cast<const T*>(p.A), p.Q, p.Q, wave, lane, [&](int j) -> int64_t {
      const int r = min(m0 + j, last);  // (rows past the expert's: any will do)
      if (!row) return r;
      const int s = row[r];
      return s >= 0 && s < total ? s : -1;
    });
    const T* w = static_cast<const T*>(p.W) + (int64_t)e * p.Q * p.NO;
    if constexpr (ACROSS) {
      b.begin(w, ldw, nullptr, p.Q, p.Q, n0, p.NO, wave, lane);
    } else {
      const int cols = p.NO - 1;
      b.begin(w, ldw, p.Q, wave, lane, [&](int j) -> int64_t { return min(n0 + j, cols); });
    }
  }
  const int stages = owned ? (p.Q + OpA::BK - 1) / OpA::BK : 0;
  emm_loop<T, ANY, MI, NI>(a, b, lds, stages, rm, cn, wave, lane, acc);
  const int i = lane & 15, q = lane >> 4;
  const bool by4 = (p.NO & 3) == 0;
#pragma unroll
  for (int m = 0; m < MI; m++) {
    const int r = m0 + rm + 16 * m + i;
    if (r >= hi) continue;
#pragma unroll
    for (int n = 0; n < NI; n++) {
      const int c = n0 + cn + 16 * n + 4 * q;
      if (c >= p.NO) continue;
      const int64_t o = (int64_t)r * p.NO + c;
      f4 v = acc[m][n];
      if (p.relu) {
#pragma unroll
        for (int x = 0; x < 4; x++) v[x] = v[x] > 0.0f ? v[x] : 0.0f;  // (NaN and -0 give +0)
      }
      if (p.gate && owned) {
        const T* g = static_cast<const T*>(p.gate) + o;
        if (by4) {
          const typename Elem<T>::v4 h = *reinterpret_cast<const typename Elem<T>::v4*>(g);
#pragma unroll
          for (int x = 0; x < 4; x++) v[x] = static_cast<float>(h[x]) > 0.0f ? v[x] : 0.0f;
        } else {
#pragma unroll
          for (int x = 0; x < 4; x++)
            if (c + x < p.NO) v[x] = static_cast<float>(g[x]) > 0.0f ? v[x] : 0.0f;
        }
      }
      emm_store(static_cast<T*>(p.C) + o, p.NO - c, by4, v);
    }
  }
}

struct ExpertWeightsArgs {
  const void* dY;  // [R][N]
  const void* X;   // [T][K], taken through `row`, or [R][K]
  void* dW;        // [E][N][K]
  const int* off;
  const int* row;
  int R, T, E, N, K;
  int nt, mt;  // tiles of K, of N
  int add;
};

template <typename T, typename TO, bool ANY, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void expert_weights_kernel(ExpertWeightsArgs p) {
  constexpr int NW = WM * WN, MI = BM / WM / 16, NI = BN / WN / 16;
  typedef AcrossRows<T, BM, NW> OpA;
  typedef AcrossRows<T, BN, NW> OpB;
  __shared__ __align__(16) char lds[2 * (OpA::BYTES + OpB::BYTES)];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // every XCD takes a run of tiles of its own
  const unsigned per = p.mt * p.nt, total = per * p.E, run = (total + 7) / 8;
  const unsigned at = (blockIdx.x & 7) * run + blockIdx.x / 8;
  if (blockIdx.x / 8 >= run || at >= total) return;
  const int e = (int)(at / per), in = (int)(at % per);
  const int block = in / (8 * p.nt), rest = in % (8 * p.nt), height = min(8, p.mt - 8 * block);
  const int m0 = (8 * block + rest % height) * BM, n0 = (rest / height) * BN;
  const int lo = min(max(p.off[e], 0), p.R), hi = min(max(p.off[e + 1], 0), p.R), rows = max(hi - lo, 0);
  const int rm = (wave / WN) * (BM / WM), cn = (wave % WN) * (BN / WN);
  f4 acc[MI][NI];
  OpA a;
  OpB b;
  a.begin(static_cast<const T*>(p.dY) + (int64_t)lo * p.N, p.N, nullptr, rows, rows, m0, p.N, wave, lane);
  if (p.row) b.begin(static_cast<const T*>(p.X), p.K, p.row + lo, rows, p.T, n0, p.K, wave, lane);
  else b.begin(static_cast<const T*>(p.X) + (int64_t)lo * p.K, p.K, nullptr, rows, rows, n0, p.K, wave, lane);
  emm_loop<T, ANY, MI, NI>(a, b, lds, (rows + OpA::BK - 1) / OpA::BK, rm, cn, wave, lane, acc);
  const int i = lane & 15, q = lane >> 4;
  const bool by4 = (p.K & 3) == 0;
  TO* out = static_cast<TO*>(p.dW) + (int64_t)e * p.N * p.K;
#pragma unroll
  for (int m = 0; m < MI; m++) {
    const int r = m0 + rm + 16 * m + i;
    if (r >= p.N) continue;
#pragma unroll
    for (int n = 0; n < NI; n++) {
      const int c = n0 + cn + 16 * n + 4 * q;
      if (c >= p.K) continue;
      TO* o = out + (int64_t)r * p.K + c;
      f4 v = acc[m][n];
      if (p.add) {
#pragma unroll
        for (int x = 0; x < 4; x++)
          if (c + x < p.K) v[x] += static_cast<float>(o[x]);
      }
      emm_store(o, p.K - c, by4, v);
    }
  }
}

}  // namespace tc355
