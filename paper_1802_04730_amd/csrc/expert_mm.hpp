// Products grouped by expert: expert e owns the rows Off(e) .. Off(e+1) of a matrix of R rows, as many as a router gave it.
//   Y(r,n)    = act(sum_k X(src(r),k) * W(e(r),n,k))         rows kernel, both operands along their rows
//   dX(r,k)   = gate(r,k) * sum_n dY(r,n) * W(e(r),n,k)      rows kernel, W across its rows
//   dW(e,n,k) = sum_{r of e} dY(r,n) * X(src(r),k)           weights kernel, both operands across their rows
// What bounds them: 2 R N K operations each on the matrix core, unless an expert has so few rows that its weights' bytes do
// (expert_rows.hpp takes those).
//
// A workgroup computes a BM x BN tile of one expert, a stage of 128 bytes of the reduction (64 elements of 16 bits, 32 of 32) at a time:
// whole cache lines of an operand's rows, whose loads take the address path half the time of half lines.  Stages go straight from
// memory to a ring of D buffers in LDS, 16 bytes per lane, D - 1 stages ahead.  A stage is multiplied in two halves; the fragments of the
// next half are read meanwhile, so that the matrix core waits for nothing but the one barrier a stage.
//
// Layout in LDS.  Along its rows an operand is [rows][128 bytes]; the 16-byte chunk c of row r lies in slot c ^ (r & 7), so that
// the 16 rows of a fragment read hit all banks.  Across its rows it is [reduction][tile columns]: 16-bit elements are
// read by the transposing LDS read (four rows of 16 columns to 16 lanes of four), 32-bit ones word by word; chunks are swizzled by
// the rows that one instruction reads together.  Lane (i = lane % 16, q = lane / 16) of a matrix instruction supplies row i and, of the
// half stage, elements 8q .. 8q+7 of 32 (16 bits) or, in 4 instructions, 4q .. 4q+3 of 16 (32 bits): the order is free as long as
// both operands keep it.  The operands are exchanged (weights first), so that a lane's four results are neighbours in a row of the output.
//
// Sums are fp32 in the matrix core's accumulators whatever the storage, and each output is rounded once.
//
// Measured, us a call, bfloat16: one matrix of 8192^3 752 forward (1461 TFLOP/s, tile of 256), 961 dX, 1017 dW (128); 32 experts of 512 rows each, N = 2048,
// K = 4096: 254, 323, 333; of uneven shares 344, 362, 387: the last round of tiles, and last rows of experts, are
// not full.  fp32, 2100 rows of 12 experts, 1001 x 517: 38, 49, 42.  Tried and left: two stages with all fragments read at once
// (uneven shares: 352, 538, 729 us, by spills), four stages of 64 bytes (404, 411, 539), 16 wavefronts a tile of 256 (spills), tiles of 256 x 128
// in a ring of three (1088 TFLOP/s at 8192^3 where this then reached 1268, more lost at ragged ends), the last round's tiles shared by two
// workgroups (no gain), and, for dW, the next tile's first stages requested before this one is stored (488 us from 486 at 32 experts, 2048 x 4096, 612 from 645 at 8, 4096 x 4096).
#pragma once
#include "expert_types.hpp"

namespace tc355 {

constexpr int EMM_STAGE = 128;  // bytes of the reduction per stage and row

static __device__ __align__(16) const unsigned emm_zeros[4] = {0, 0, 0, 0};  // what stands for elements that are not there

template <int N>
__device__ __forceinline__ void emm_wait() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
typedef __attribute__((address_space(3))) char lds_char;
__device__ __forceinline__ void emm_to_lds(const char* g, lds_char* lds) {  // lane l's 16 bytes to lds + 16 l (a uniform address)
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(uintptr_t)g, (__attribute__((address_space(3))) void*)lds, 16, 0, 0);
}

// ---- which rows a tile takes ------------------------------------------------------------------------------------------

struct ExpertTile {
  int e;       // expert; E: the rows that no expert owns
  int lo, hi;  // its rows
  int m, n;    // tile of the expert, in rows and columns
};

// Offsets are the device's: whatever they hold, an expert's rows are [most of Off(0..e), most of Off(0..e+1)), all clamped to [0, R].  So no row
// has two experts, and there are never more tiles than most_row_tiles says.  Offsets that go up, as a router's do, are that already, which a ballot tells.
__device__ __forceinline__ int offset_within(const int* off, int g, int R) { return min(max(off[g], 0), R); }

// Workgroup `bid`'s tile, or false.  Tiles of one expert follow each
// other in blocks of 8 row tiles by all column tiles, row tiles first, so that workgroups that run together share operands; and every
// XCD (workgroups equal modulo 8) takes a run of its own.  One round trip to memory for up to 63 experts.
__device__ __forceinline__ bool expert_tile(const int* off, int E, int R, int bm, int nt, unsigned bid, ExpertTile* t) {
  const int lane = threadIdx.x & 63;
  int lo, hi;
  const auto tiles = [&](int g, int* reached) {  // of expert g; its rows go to lo, hi; reached: by the experts before this lane 0's, then before the next one's
    lo = hi = R;
    if (g <= E) {
      lo = offset_within(off, g, R);
      if (g < E) hi = offset_within(off, g + 1, R);
    }
    if (__ballot(hi < lo || lo < *reached)) {
      lo = max(lo, *reached);
      hi = max(hi, lo);
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        const int o = __shfl_up(hi, d);
        if (lane >= d) hi = max(hi, o);
      }
      const int before = __shfl_up(hi, 1);
      if (lane) lo = before;
    }
    *reached = __shfl(hi, 63);
    return (unsigned)((hi - lo + bm - 1) / bm) * nt;
  };
  const auto up_to = [&](unsigned n) {  // inclusive sums over the lanes
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const unsigned o = __shfl_up(n, d);
      if (lane >= d) n += o;
    }
    return n;
  };
  int reached = 0;
  unsigned n = tiles(lane, &reached), incl = up_to(n), total = __shfl(incl, 63);
  for (int base = 64; base <= E; base += 64) total += __shfl(up_to(tiles(base + lane, &reached)), 63);
  const unsigned run = (total + 7) / 8;
  if (bid / 8 >= run) return false;
  const unsigned at = (bid & 7) * run + bid / 8;
  if (at >= total) return false;
  unsigned before = 0;
  reached = 0;
  for (int base = 0; base <= E; base += 64) {
    if (E >= 64) {
      n = tiles(base + lane, &reached);
      incl = up_to(n);
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

// The first row of expert e, which has rows by its own offsets: the most of Off(0..e); own: Off(e).  (A trip to memory beside that of the expert's
// own: dW of 32 rows of 8 experts, 4096 x 2048, 29.2 us where 28.3 without, of 8020 rows of 64, 2672 x 1824, 199 and 197, of 16384 rows of 32, 2048 x 4096, 350
// and 347.  Asked for before the expert is known, or looked at after the loop: no faster.)
__device__ __forceinline__ int expert_first_row(const int* off, int e, int R, int own) {
  const int lane = threadIdx.x & 63;
  int most = 0;
  if (e < 64) {
    most = offset_within(off, min(lane, e), R);
  } else {
    for (int base = 0; base <= e; base += 256) {
#pragma unroll
      for (int j = 0; j < 4; j++) most = max(most, offset_within(off, min(base + 64 * j + lane, e), R));
    }
  }
  if (!__ballot(most > own)) return own;
#pragma unroll
  for (int d = 32; d; d /= 2) most = max(most, __shfl_xor(most, d));
  return most;
}

// ---- operands: memory to LDS, LDS to fragments ------------------------------------------------------------------------

// How operands reach LDS: WHOLE, straight from rows of whole 16-byte pieces; ANY, through registers, from rows of any width and alignment;
// NARROW, the same element by element, where one operand's rows have less than 16 bytes.
enum { EMM_WHOLE = 0, EMM_ANY = 1, EMM_NARROW = 2 };

// 16 bytes of a row of `width` elements from element `at` on, in two steps: loaded whole from within the row, without a branch, which would make
// each load wait for the one before; and, when they are needed, shifted to their places with zeros past the row's end.
template <typename T, int MODE>
__device__ __forceinline__ u4 emm_load_within(const T* row, int at, int width) {
  constexpr int PER = Elem<T>::PER16;
  if constexpr (MODE != EMM_NARROW) return __builtin_bit_cast(u4, load_pack<T, PER>(row + min(at, width - PER)));
  const int a = width >= PER ? min(at, width - PER) : 0;
  Pack<T, PER> v;
#pragma unroll
  for (int i = 0; i < PER; i++) v.e[i] = a + i < width ? row[a + i] : static_cast<T>(0.0f);
  return __builtin_bit_cast(u4, v);
}
template <typename T>
__device__ __forceinline__ u4 emm_shift(u4 x, int at, int width) {
  constexpr int PER = Elem<T>::PER16, BITS = 8 * sizeof(T);
  const int shift = min(at - (width >= PER ? min(at, width - PER) : 0), PER) * BITS;
  typedef unsigned long long two __attribute__((ext_vector_type(2)));
  const two v = __builtin_bit_cast(two, x);
  const unsigned long long down = v[1] >> (shift & 63);
  const two part = {shift >= 64 ? down : shift ? v[0] >> shift | v[1] << (64 - shift) : v[0], shift >= 64 ? 0 : down};
  return shift >= 128 ? u4{0, 0, 0, 0} : __builtin_bit_cast(u4, part);
}
template <typename T>
__device__ __forceinline__ u4 emm_load_any(const T* row, int at, int width) {
  if (width < Elem<T>::PER16) return emm_shift<T>(emm_load_within<T, EMM_NARROW>(row, at, width), at, width);
  return emm_shift<T>(emm_load_within<T, EMM_ANY>(row, at, width), at, width);
}

// Operand along its rows: ROWS rows of the tile, 128 bytes of the reduction a stage.  NW wavefronts load it, 8 rows an instruction.
// ANYWHERE: the rows lie anywhere (an address per lane and instruction); else within 4 GB of each other, from a base that all share.
template <typename T, int ROWS, int NW, bool ANYWHERE>
struct AlongRows {
  static constexpr bool ACROSS = false;
  static constexpr int BYTES = ROWS * EMM_STAGE;
  static constexpr int PER = ROWS / 8 / NW;  // instructions of a wavefront
  static constexpr int BK = EMM_STAGE / sizeof(T);
  static_assert(PER * 8 * NW == ROWS, "whole instructions");
  const char* p[ANYWHERE ? PER : 1];  // this lane's rows at its chunk of the stage, or the base there
  unsigned off[ANYWHERE ? 1 : PER];
  int at, q0, Q;  // the chunk's first element in a stage; the stage's first one; all
  u4 held[PER];

  // row(j): where row j of the tile lies among those of `b`
  template <typename F>
  __device__ __forceinline__ void begin(const T* b, int64_t ld, int q, int wave, int lane, F row) {
    Q = q;
    q0 = 0;
    at = ((lane & 7) ^ (lane >> 3)) * Elem<T>::PER16;  // (row & 7 = lane / 8)
    if constexpr (!ANYWHERE) p[0] = reinterpret_cast<const char*>(b);
#pragma unroll
    for (int j = 0; j < PER; j++) {
      const int64_t r = row((wave * PER + j) * 8 + (lane >> 3));
      if constexpr (ANYWHERE) p[j] = reinterpret_cast<const char*>(b + r * ld + at);
      else off[j] = (unsigned)(r * ld + at) * (unsigned)sizeof(T);
    }
  }
  __device__ __forceinline__ const char* where(int j) const {
    if constexpr (ANYWHERE) return p[j];
    else return p[0] + off[j];
  }
  __device__ __forceinline__ void to_lds(lds_char* lds, int wave, int) {
    if (q0 + BK <= Q) {
#pragma unroll
      for (int j = 0; j < PER; j++) emm_to_lds(where(j), lds + (wave * PER + j) * 1024);
    } else {
      const bool in = q0 + at < Q;
#pragma unroll
      for (int j = 0; j < PER; j++) emm_to_lds(in ? where(j) : reinterpret_cast<const char*>(emm_zeros), lds + (wave * PER + j) * 1024);
    }
    next();
  }
  template <int MODE>
  __device__ __forceinline__ void hold(int, int) {
#pragma unroll
    for (int j = 0; j < PER; j++) {
      held[j] = emm_load_within<T, MODE>(reinterpret_cast<const T*>(where(j)) - (q0 + at), q0 + at, Q);
    }
    next();
  }
  __device__ __forceinline__ void put(lds_char* lds, int wave, int lane) {  // (what was fetched last: the stage before q0)
    if (q0 > Q) {
#pragma unroll
      for (int j = 0; j < PER; j++) held[j] = emm_shift<T>(held[j], q0 - BK + at, Q);
    }
#pragma unroll
    for (int j = 0; j < PER; j++) *(__attribute__((address_space(3))) u4*)(lds + (wave * PER + j) * 1024 + lane * 16) = held[j];
  }
  __device__ __forceinline__ void next() {
    q0 += BK;
#pragma unroll
    for (int j = 0; j < (ANYWHERE ? PER : 1); j++) p[j] += EMM_STAGE;
  }
  // rows r0 .. r0+15 of the tile, half s of the stage: 16 bytes of row r0 + i, chunk 4 s + q
  static __device__ __forceinline__ u4 fragment(const lds_char* lds, int r0, int s, int i, int q) {
    return *(const __attribute__((address_space(3))) u4*)(lds + (r0 + i) * EMM_STAGE + (((4 * s + q) ^ (i & 7)) * 16));
  }
};

// Operand across its rows: BK rows of the reduction a stage, COLS columns of the tile.
// ANYWHERE: the reduction goes through rows that a list names; else through neighbours.
template <typename T, int COLS, int NW, bool ANYWHERE>
struct AcrossRows {
  static constexpr bool ACROSS = true;
  static constexpr int BK = EMM_STAGE / sizeof(T);
  static constexpr int BYTES = BK * COLS * sizeof(T);
  static constexpr int CPR = COLS * sizeof(T) / 16;  // chunks of a row
  static constexpr int RPI = 64 / CPR;               // rows of an instruction
  static constexpr int PER = BK / RPI / NW;
  static_assert(RPI * CPR == 64 && PER * RPI * NW == BK, "whole instructions");
  const T* base;    // the stage's first row; ANYWHERE: row 0
  const int* row;   // ANYWHERE: rows of `base` that the reduction goes through, from the next but one stage on
  int64_t ld;
  int q0, Q, rows;  // the stage's first row of the reduction, their number; rows of `base`
  int cols;
  int col[PER];     // first column of the chunk; beyond the last column any chunk will do
  unsigned off[ANYWHERE ? 1 : PER];
  int src[ANYWHERE ? PER : 1];
  u4 held[PER];
  unsigned fetched;  // which of them are there
  bool edge;         // the tile passes the last column

  // rows that one instruction reads together have different chunks of 64 banks
  static __device__ __forceinline__ int swizzle(int r) {
    if constexpr (sizeof(T) == 4) return 4 * ((r >> 2) & 3);
    else if constexpr (CPR >= 16) return 2 * ((r & 3) | ((r >> 1) & 4));
    else return 2 * (((r >> 1) & 1) | ((r >> 2) & 2));  // (a row is half the banks: neighbouring rows differ anyway)
  }
  static __device__ __forceinline__ int at(int j, int wave, int lane) { return (wave * PER + j) * RPI + lane / CPR; }

  template <int MODE>
  __device__ __forceinline__ void begin(const T* b, int64_t stride, const int* rw, int q, int total, int c0, int width, int wave, int lane) {
    base = b;
    row = rw;
    ld = stride;
    q0 = 0;
    Q = q;
    rows = total;
    cols = width;
    edge = c0 + COLS > width;
    fetched = 0;
#pragma unroll
    for (int j = 0; j < PER; j++) {
      col[j] = c0 + ((lane % CPR) ^ swizzle(at(j, wave, lane))) * Elem<T>::PER16;
      if (MODE == EMM_WHOLE) col[j] = min(col[j], cols - Elem<T>::PER16);
      if constexpr (!ANYWHERE) off[j] = (unsigned)(at(j, wave, lane) * ld + col[j]) * (unsigned)sizeof(T);
    }
    if constexpr (ANYWHERE) look(wave, lane);
  }
  // the source rows of the stage at q0; -1: zeros
  __device__ __forceinline__ void look(int wave, int lane) {
#pragma unroll
    for (int j = 0; j < PER; j++) {
      const int q = q0 + at(j, wave, lane);
      src[j] = -1;
      if (q < Q) src[j] = row[q];
    }
  }
  __device__ __forceinline__ const T* where(int j) const {
    if constexpr (ANYWHERE) return base + (int64_t)src[j] * ld + col[j];
    else return reinterpret_cast<const T*>(reinterpret_cast<const char*>(base) + off[j]);
  }
  __device__ __forceinline__ bool there(int j, int wave, int lane) const {
    if constexpr (ANYWHERE) return src[j] >= 0 && src[j] < rows;
    else return q0 + at(j, wave, lane) < Q;
  }
  __device__ __forceinline__ void to_lds(lds_char* lds, int wave, int lane) {
    if (!ANYWHERE && q0 + BK <= Q) {
#pragma unroll
      for (int j = 0; j < PER; j++) emm_to_lds(reinterpret_cast<const char*>(where(j)), lds + (wave * PER + j) * 1024);
    } else {
#pragma unroll
      for (int j = 0; j < PER; j++) {
        const char* s = there(j, wave, lane) ? reinterpret_cast<const char*>(where(j)) : reinterpret_cast<const char*>(emm_zeros);
        emm_to_lds(s, lds + (wave * PER + j) * 1024);
      }
    }
    next(wave, lane);
  }
  template <int MODE>
  __device__ __forceinline__ void hold(int wave, int lane) {
#pragma unroll
    for (int j = 0; j < PER; j++) {
      const bool in = there(j, wave, lane);  // (a row that is not there: any that is, made zeros when it is put)
      const T* r = ANYWHERE ? base + (int64_t)(in ? src[ANYWHERE ? j : 0] : 0) * ld : base + (in ? (int64_t)at(j, wave, lane) : (int64_t)-q0) * ld;
      if (rows > 0) held[j] = emm_load_within<T, MODE>(r, col[j], cols);
      fetched = (fetched & ~(1u << j)) | (in ? 1u << j : 0);
    }
    next(wave, lane);
  }
  __device__ __forceinline__ void put(lds_char* lds, int wave, int lane) {
    if (edge) {
#pragma unroll
      for (int j = 0; j < PER; j++) held[j] = emm_shift<T>(held[j], col[j], cols);
    }
    if (ANYWHERE || q0 > Q) {
#pragma unroll
      for (int j = 0; j < PER; j++) held[j] = fetched >> j & 1 ? held[j] : u4{0, 0, 0, 0};
    }
#pragma unroll
    for (int j = 0; j < PER; j++) *(__attribute__((address_space(3))) u4*)(lds + (wave * PER + j) * 1024 + lane * 16) = held[j];
  }
  __device__ __forceinline__ void next(int wave, int lane) {
    q0 += BK;
    if constexpr (ANYWHERE) look(wave, lane);
    else base += BK * ld;
  }
  // columns c0 .. c0+15 of the tile, half s of the stage, the reduction's elements as along rows
  static __device__ __forceinline__ u4 fragment(const lds_char* lds, int c0, int s, int i, int q) {
    if constexpr (sizeof(T) == 2) {
      // rows 32 s + 8 q + 4 h + (0..3): this lane's address of the transposing read is that of 4 elements of one row
      s4v v[2];
#pragma unroll
      for (int h = 0; h < 2; h++) {
        const int r = 32 * s + 8 * q + 4 * h + (i >> 2), c = c0 + (i & 3) * 4;
        v[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4v*)(const_cast<lds_char*>(lds) + r * (COLS * 2) +
                                                                                              (((c >> 3) ^ swizzle(r)) * 16) + (c & 7) * 2));
      }
      return __builtin_bit_cast(u4, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      f4 v;
#pragma unroll
      for (int e = 0; e < 4; e++) {
        const int r = 16 * s + 4 * q + e, c = c0 + i;
        v[e] = *(const __attribute__((address_space(3))) float*)(lds + r * (COLS * 4) + (((c >> 2) ^ swizzle(r)) * 16) + (c & 3) * 4);
      }
      return __builtin_bit_cast(u4, v);
    }
  }
};

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

// Traffic of half a stage: what goes into buffer `then`, and the fragments of half s that come out of buffer `now`.  (Restricted
// pointers of a function of their own: the compiler would wait for all loads to LDS before any LDS read that they might concern.)
template <int MODE, int MI, int NI, typename A, typename B>
__device__ __forceinline__ void emm_traffic(A& a, B& b, const lds_char* __restrict__ now, lds_char* __restrict__ then, int s, bool read, bool more, bool held,
                                            int rm, int cn, int wave, int lane, u4 (&fa)[MI], u4 (&fb)[NI]) {
  const int i = lane & 15, q = lane >> 4;
  if constexpr (MODE != EMM_WHOLE) {
    if (held) {
      a.put(then, wave, lane);
      b.put(then + A::BYTES, wave, lane);
    }
    if (more) {
      a.template hold<MODE>(wave, lane);
      b.template hold<MODE>(wave, lane);
    }
  } else {
    if (more) {
      a.to_lds(then, wave, lane);
      b.to_lds(then + A::BYTES, wave, lane);
    }
  }
  if (read) {
#pragma unroll
    for (int n = 0; n < NI; n++) fb[n] = B::fragment(now + A::BYTES, cn + 16 * n, s, i, q);
#pragma unroll
    for (int m = 0; m < MI; m++) fa[m] = A::fragment(now, rm + 16 * m, s, i, q);
  }
}

// Until at most `stages` stages' loads (P a stage) are in flight.
template <int P, int MOST>
__device__ __forceinline__ void emm_wait_stages(int stages) {
  if constexpr (MOST > 0) {
    if (stages < MOST) return emm_wait_stages<P, MOST - 1>(stages);
  }
  emm_wait<P * MOST>();
}

// MI x NI blocks of 16 x 16 per wavefront, at row rm and column cn of the tile.
template <typename T, int MODE, int D, int MI, int NI, typename A, typename B>
__device__ __forceinline__ void emm_loop(A& a, B& b, lds_char* lds, int stages, int rm, int cn, int wave, int lane, f4 (&acc)[MI][NI]) {
  constexpr int STAGE = A::BYTES + B::BYTES, P = A::PER + B::PER;
#pragma unroll
  for (int m = 0; m < MI; m++)
#pragma unroll
    for (int n = 0; n < NI; n++) acc[m][n] = f4{0, 0, 0, 0};
  if (stages <= 0) return;
  u4 fa[2][MI], fb[2][NI];
  if constexpr (MODE != EMM_WHOLE) {  // stage t + 2 is written, and t + 3 fetched, while the second half of stage t is multiplied
    static_assert(D == 2, "buffers");
#pragma unroll
    for (int j = 0; j < 2; j++) {
      a.template hold<MODE>(wave, lane);
      b.template hold<MODE>(wave, lane);
      a.put(lds + j * STAGE, wave, lane);
      b.put(lds + j * STAGE + A::BYTES, wave, lane);
    }
    a.template hold<MODE>(wave, lane);
    b.template hold<MODE>(wave, lane);
  } else {
#pragma unroll
    for (int j = 0; j < D; j++)
      if (j < stages) {
        a.to_lds(lds + j * STAGE, wave, lane);
        b.to_lds(lds + j * STAGE + A::BYTES, wave, lane);
      }
    emm_wait_stages<P, D - 1>(stages - 1);
  }
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  emm_traffic<MODE, MI, NI>(a, b, lds, lds, 0, true, false, false, rm, cn, wave, lane, fa[0], fb[0]);
  int at = 0;  // buffer of stage t
  for (int t = 0; t < stages; t++) {
    lds_char* const now = lds + at * STAGE;
    at = at + 1 == D ? 0 : at + 1;
    emm_traffic<MODE, MI, NI>(a, b, now, now, 1, true, false, false, rm, cn, wave, lane, fa[1], fb[1]);
#pragma unroll
    for (int m = 0; m < MI; m++)
#pragma unroll
      for (int n = 0; n < NI; n++) acc[m][n] = emm_mfma<T>(fb[0][n], fa[0][m], acc[m][n]);
    if constexpr (MODE == EMM_WHOLE) emm_wait_stages<P, D - 2>(stages - 2 - t);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();  // stage t + 1 is in LDS, and everyone has read stage t
    asm volatile("" ::: "memory");
    emm_traffic<MODE, MI, NI>(a, b, lds + at * STAGE, now, 0, t + 1 < stages, t + (MODE != EMM_WHOLE ? 3 : D) < stages, t + 2 < stages, rm, cn, wave, lane, fa[0], fb[0]);
#pragma unroll
    for (int m = 0; m < MI; m++)
#pragma unroll
      for (int n = 0; n < NI; n++) acc[m][n] = emm_mfma<T>(fb[1][n], fa[1][m], acc[m][n]);
  }
}

// Four neighbours of an output row from column n on, of which `left` are there.  (Through the caches: these are parts of lines, which
// cost a write to memory each where they pass them by: forward and gradients of (E,R,N,K) = (32,16384,2048,4096) 1320 us instead of 1170.)
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

// A tile of results by whole lines: through LDS (16-byte chunk c of row r in slot c ^ (r & 7)), then 16 bytes a lane, neighbours along the
// row, past the caches.  put(row, column, values): stores 16 bytes of the tile.  (The accumulators' own pieces of 8 or 16 bytes: the
// gradient of the weights of (E,R,N,K) = (32,16384,2048,4096) in bfloat16 486 us instead of 395, 8192^3 forward 863 instead of 785.)
template <typename TO, int BM, int BN, int THREADS, int MI, int NI, typename Put>
__device__ __forceinline__ void emm_store_lines(lds_char* lds, const f4 (&acc)[MI][NI], int rm, int cn, Put put) {
  constexpr int PER = Elem<TO>::PER16, ROW = BN * sizeof(TO);
  const int tid = threadIdx.x, lane = tid & 63, i = lane & 15, q = lane >> 4;
  typedef typename Elem<TO>::v4 v4;
  __syncthreads();  // (everyone has read the last stage)
#pragma unroll
  for (int m = 0; m < MI; m++)
#pragma unroll
    for (int n = 0; n < NI; n++) {
      v4 o;
#pragma unroll
      for (int x = 0; x < 4; x++) o[x] = narrow<TO>(acc[m][n][x]);
      const int r = rm + 16 * m + i, c = cn + 16 * n + 4 * q;
      *(__attribute__((address_space(3))) v4*)(lds + r * ROW + (((c / PER) ^ (r & 7)) * 16) + c % PER * (int)sizeof(TO)) = o;
    }
  __syncthreads();
#pragma unroll 4
  for (int x = tid; x < BM * BN / PER; x += THREADS) {
    const int r = x / (BN / PER), c = x % (BN / PER);
    const u4 v = *(const __attribute__((address_space(3))) u4*)(lds + r * ROW + ((c ^ (r & 7)) * 16));
    put(r, PER * c, __builtin_bit_cast(typename Elem<TO>::v16, v));
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
template <typename T, bool ACROSS, int MODE, int BM, int BN, int WM, int WN, int D>
__global__ __launch_bounds__(64 * WM * WN) void expert_rows_tile_kernel(ExpertRowsArgs p) {
  constexpr int NW = WM * WN, MI = BM / WM / 16, NI = BN / WN / 16;
  // (a tile of 256 has no registers left for addresses anywhere: the host sees to it that its rows lie within 4 GB)
  typedef AlongRows<T, BM, NW, BM != 256> OpA;
  typedef std::conditional_t<ACROSS, AcrossRows<T, BN, NW, false>, AlongRows<T, BN, NW, false>> OpB;
  __shared__ __align__(16) char lds[D * (OpA::BYTES + OpB::BYTES)];
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
  const bool owned = e < p.E && p.T > 0;
  if (owned) {
    const int* row = p.row;
    const int last = hi - 1, total = p.T;
    a.begin(static_cast<const T*>(p.A), p.Q, p.Q, wave, lane, [&](int j) -> int64_t {
      const int r = min(m0 + j, last);  // (rows past the expert's: any will do)
      return row ? min(max(row[r], 0), total - 1) : r;
    });
    const T* w = static_cast<const T*>(p.W) + (int64_t)e * p.Q * p.NO;
    if constexpr (ACROSS) {
      b.template begin<MODE>(w, ldw, nullptr, p.Q, p.Q, n0, p.NO, wave, lane);
    } else {
      const int most = p.NO - 1 - n0;
      b.begin(w + n0 * ldw, ldw, p.Q, wave, lane, [&](int j) -> int64_t { return min(j, most); });
    }
  }
  const int stages = owned ? (p.Q + OpA::BK - 1) / OpA::BK : 0;
  emm_loop<T, MODE, D, MI, NI>(a, b, (lds_char*)lds, stages, rm, cn, wave, lane, acc);
  if constexpr (MODE != EMM_NARROW) {
    typedef typename Elem<T>::v16 v16;
    constexpr int PER = Elem<T>::PER16;
    if (p.NO % PER == 0) {
      if (p.relu) {
#pragma unroll
        for (int m = 0; m < MI; m++)
#pragma unroll
          for (int n = 0; n < NI; n++)
#pragma unroll
            for (int x = 0; x < 4; x++) acc[m][n][x] = acc[m][n][x] > 0.0f ? acc[m][n][x] : 0.0f;  // (NaN and -0 give +0)
      }
      emm_store_lines<T, BM, BN, 64 * NW>((lds_char*)lds, acc, rm, cn, [&](int row, int col, v16 v) {
        const int r = m0 + row, c = n0 + col;
        if (r >= hi || c >= p.NO) return;
        const int64_t o = (int64_t)r * p.NO + c;
        if (p.row && owned && (p.row[r] < 0 || p.row[r] >= p.T)) v = v16{};  // (a row of zeros)
        if (p.gate && owned) {
          const v16 h = *reinterpret_cast<const v16*>(static_cast<const T*>(p.gate) + o);
#pragma unroll
          for (int x = 0; x < PER; x++) v[x] = static_cast<float>(h[x]) > 0.0f ? v[x] : static_cast<T>(0.0f);
        }
        __builtin_nontemporal_store(v, reinterpret_cast<v16*>(static_cast<T*>(p.C) + o));
      });
      return;
    }
  }
  const int i = lane & 15, q = lane >> 4;
  const bool by4 = (p.NO & 3) == 0;
#pragma unroll
  for (int m = 0; m < MI; m++) {
    const int r = m0 + rm + 16 * m + i;
    if (r >= hi) continue;
    const bool nothing = p.row && owned && (p.row[r] < 0 || p.row[r] >= p.T);  // (a row of zeros)
#pragma unroll
    for (int n = 0; n < NI; n++) {
      const int c = n0 + cn + 16 * n + 4 * q;
      if (c >= p.NO) continue;
      const int64_t o = (int64_t)r * p.NO + c;
      f4 v = acc[m][n];
      if (nothing) v = f4{0, 0, 0, 0};
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

// With parts, blockIdx.y takes its share of the expert's rows (whole stages but for the last part's end) and dW is the workspace,
// [parts][E][N][K] of fp32, which expert_weights_join_kernel adds up in the parts' order.
struct ExpertWeightsArgs {
  const void* dY;  // [R][N]
  const void* X;   // [T][K], taken through `row`, or [R][K]
  void* dW;        // [E][N][K]
  const int* off;
  const int* row;
  int R, T, E, N, K;
  int nt, mt;  // tiles of K, of N
  int add, parts;
};

template <typename T, typename TO, int MODE, bool LIST, int BM, int BN, int WM, int WN, int D>
__global__ __launch_bounds__(64 * WM * WN) void expert_weights_kernel(ExpertWeightsArgs p) {
  constexpr int NW = WM * WN, MI = BM / WM / 16, NI = BN / WN / 16;
  typedef AcrossRows<T, BM, NW, false> OpA;
  typedef AcrossRows<T, BN, NW, LIST> OpB;
  __shared__ __align__(16) char lds[D * (OpA::BYTES + OpB::BYTES)];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // every XCD (workgroups equal modulo 8) takes an eighth of each expert's tiles: experts' rows, and with them tiles' times, differ
  const int per = p.mt * p.nt, share = (per + 7) / 8;
  const int e = (int)(blockIdx.x / 8) / share, in = (int)(blockIdx.x & 7) * share + (int)(blockIdx.x / 8) % share;
  if (e >= p.E || in >= per) return;
  const int block = in / (8 * p.nt), rest = in % (8 * p.nt), height = min(8, p.mt - 8 * block);
  const int m0 = (8 * block + rest % height) * BM, n0 = (rest / height) * BN;
  int lo = offset_within(p.off, e, p.R), hi = offset_within(p.off, e + 1, p.R);
  if (lo < hi) lo = __builtin_amdgcn_readfirstlane(expert_first_row(p.off, e, p.R, lo));
  hi = max(lo, hi);
  if (p.parts > 1) {
    constexpr int BK = OpA::BK;
    const int share = (hi - lo + p.parts * BK - 1) / (p.parts * BK) * BK;
    hi = (int)min((int64_t)hi, lo + (int64_t)(blockIdx.y + 1) * share);
    lo = (int)min((int64_t)hi, lo + (int64_t)blockIdx.y * share);
  }
  const int rows = hi - lo;
  const int rm = (wave / WN) * (BM / WM), cn = (wave % WN) * (BN / WN);
  f4 acc[MI][NI];
  OpA a;
  OpB b;
  a.template begin<MODE>(static_cast<const T*>(p.dY) + (int64_t)lo * p.N, p.N, nullptr, rows, rows, m0, p.N, wave, lane);
  if constexpr (LIST) b.template begin<MODE>(static_cast<const T*>(p.X), p.K, p.row + lo, rows, p.T, n0, p.K, wave, lane);
  else b.template begin<MODE>(static_cast<const T*>(p.X) + (int64_t)lo * p.K, p.K, nullptr, rows, rows, n0, p.K, wave, lane);
  emm_loop<T, MODE, D, MI, NI>(a, b, (lds_char*)lds, (rows + OpA::BK - 1) / OpA::BK, rm, cn, wave, lane, acc);
  TO* const out = static_cast<TO*>(p.dW) + ((int64_t)blockIdx.y * p.E + e) * p.N * p.K;
  if constexpr (MODE != EMM_NARROW) {
    typedef typename Elem<TO>::v16 v16;
    // (16-bit results that are added to are rounded once, from the accumulators, below)
    if (p.K % Elem<TO>::PER16 == 0 && !(p.add && sizeof(TO) == 2)) {
      const auto at = [&](int row, int col) -> v16* {
        const int r = m0 + row, c = n0 + col;
        return r < p.N && c < p.K ? reinterpret_cast<v16*>(out + (int64_t)r * p.K + c) : nullptr;
      };
      if (sizeof(TO) == 4 && p.parts > 1) {  // (read back at once)
        emm_store_lines<TO, BM, BN, 64 * NW>((lds_char*)lds, acc, rm, cn, [&](int row, int col, v16 v) {
          if (v16* o = at(row, col)) *o = v;
        });
      } else {
        emm_store_lines<TO, BM, BN, 64 * NW>((lds_char*)lds, acc, rm, cn, [&](int row, int col, v16 v) {
          if (v16* o = at(row, col)) {
            if (p.add) v += *o;
            __builtin_nontemporal_store(v, o);
          }
        });
      }
      return;
    }
  }
  const int i = lane & 15, q = lane >> 4;
  const bool by4 = (p.K & 3) == 0;
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

// dW (+)= the sum of the parts, four neighbours a thread.
template <typename TO>
__global__ __launch_bounds__(WG_THREADS) void expert_weights_join_kernel(const float* part, void* dW, int64_t n, int parts, int add) {
  const int64_t at = ((int64_t)blockIdx.x * WG_THREADS + threadIdx.x) * 4;
  if (at >= n) return;
  const int left = (int)min((int64_t)4, n - at);
  f4 v = {0, 0, 0, 0};
  if (left == 4) {
#pragma unroll 4
    for (int s = 0; s < parts; s++) v += __builtin_bit_cast(f4, load_pack<float, 4>(part + s * n + at));
  } else {
    for (int s = 0; s < parts; s++)
#pragma unroll
      for (int x = 0; x < 4; x++)
        if (x < left) v[x] += part[s * n + at + x];
  }
  TO* o = static_cast<TO*>(dW) + at;
  if (add) {
#pragma unroll
    for (int x = 0; x < 4; x++)
      if (x < left) v[x] += static_cast<float>(o[x]);
  }
  emm_store(o, left, left == 4, v);
}

}  // namespace tc355
