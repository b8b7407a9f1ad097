// Tiles of keys or queries of one head in LDS for the bf16 matrix-core kernels over key ranges, heads of up to DHP = 64 or 128
// columns (narrower ones are zero beyond their width).  Rows come straight from memory into LDS.
//
// All kernels work on transposed score tiles S^T[key, query] = K Q^T: a lane owns one query (forward, dQ) or one key (dK/dV),
// element e of a 32 x 32 result is tile row (e >> 2) * 8 + (lane >> 5) * 4 + (e & 3), and 8 such elements in a row are the
// operand of the second product, whose other operand is read against its storage order by ds_read_b64_tr_b16.
//
// A row is 2 DHP bytes, unpadded, so the layout is a swizzle of its 16-byte chunks: chunk c of row r lies in place c ^ swz(r).
// A fragment read takes 16 consecutive rows at a time: their swz (and, at 128 bytes, which half of the banks the row is in) put the
// same chunk of each into 16 different places.  A transposing read takes 64 bytes of four consecutive rows: those differ in
// the bits that choose the quarter of the banks.
#pragma once
#include "attn_range.h"
#include "lds_load.h"

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ bf16x8 acc_to_frag(const f32x16& a, int c) {
  bf16x8 r;
#pragma unroll
  for (int u = 0; u < 8; u++) r[u] = (__bf16)a[8 * c + u];
  return r;
}

// The kernel's arguments (RangeAttn is the first of them), read anew: for what comes after a loop, or hardly ever, so that it holds no
// registers in the loop.
__device__ __forceinline__ RangeAttn args_again() {
  unsigned long long p = (unsigned long long)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  typedef const __attribute__((address_space(4))) unsigned long long word;
  static_assert(sizeof(RangeAttn) % 8 == 0, "whole words");
  union { RangeAttn a; unsigned long long w[sizeof(RangeAttn) / 8]; } r;
#pragma unroll
  for (unsigned i = 0; i < sizeof(RangeAttn) / 8; i++) r.w[i] = ((word*)p)[i];
  return r.a;
}

// The lane number, asked for where it is used: what is worked out from it then holds no register from tile to tile.
__device__ __forceinline__ int lane_now() {
  unsigned none = 0;
  asm volatile("" : "+v"(none));
  return (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, none));
}

// ---- tiles ----
template <int DHP> __device__ __forceinline__ int swz(int r) {
  return DHP == 128 ? ((r & 3) << 2) | ((r >> 2) & 3) : (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
}
// rows of one head: address of row 0's first column of the head, row stride and width in bytes
struct HeadRows { const unsigned char* base; i64 ldb; int width; };
// rows r0 .. r0 + n - 1 as a buffer: what lies behind them reads as zeros without traffic (n <= 0: all of it)
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_buffer(const HeadRows& h, int r0, int n) {
  return __builtin_amdgcn_make_buffer_rsrc((void*)(h.base + (i64)r0 * h.ldb), (short)0, n <= 0 ? 0 : (int)((n - 1) * h.ldb + h.width), 0x00020000);
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t words_buffer(const void* p, int r0, int n) {
  return __builtin_amdgcn_make_buffer_rsrc((void*)((const unsigned char*)p + (i64)r0 * 4), (short)0, n <= 0 ? 0 : n * 4, 0x00020000);
}
template <int DHP> struct Tiles {
  static constexpr int ROW = DHP * 2, CPR = DHP / 8, RPL = 64 / CPR;       // bytes and chunks per row, rows per wave-load
  static constexpr int KK = DHP / 16, DT = DHP / 32;                        // steps of a product over the width, column blocks
  static constexpr unsigned LOADS = 16 / RPL;                               // wave-loads per 16 rows
  static constexpr unsigned BYTES = 64u * ROW;                              // of a tile of 64 rows
  // 16 rows of a buffer, from row0 on, to LDS at dst
  static __device__ __forceinline__ void load16(__amdgpu_buffer_rsrc_t rs, unsigned ldb, int width, int row0, unsigned dst) {
    const int lane = lane_now();
    const unsigned c = (unsigned)((lane % CPR) ^ swz<DHP>(lane / CPR)), mine = (unsigned)(lane / CPR) * ldb;      // (one multiplication per lane)
#pragma unroll
    for (unsigned i = 0; i < LOADS; i++) {
      const unsigned chunk = c ^ (i * (DHP == 128 ? 1u : 2u));              // swz(RPL i + a) = swz(a) ^ ..
      unsigned off = mine + chunk * 16u + __builtin_amdgcn_readfirstlane((unsigned)(row0 + (int)i * RPL) * ldb);
      if (width < ROW) off = (int)(chunk * 16u) < width ? off : OOB;
      load_lds_b128(rs, __builtin_amdgcn_readfirstlane(dst + i * 1024u), off);
    }
  }
  // per-lane byte offsets: fragments of rows lane & 31 (step kk: ^ kk * 32), transposed ones (column block: ^ dtile * 64)
  static __device__ __forceinline__ unsigned row_base(int lane) { return (unsigned)(lane & 31) * ROW + (unsigned)((lane >> 5) ^ swz<DHP>(lane & 15)) * 16u; }
  static __device__ __forceinline__ unsigned col_base(int lane) {
    const int blk = lane >> 4, i16 = lane & 15, row = 4 * (blk >> 1) + (i16 >> 2), c = 2 * (blk & 1) + ((i16 & 3) >> 1);
    return (unsigned)row * ROW + (unsigned)(c ^ swz<DHP>(row)) * 16u + (unsigned)(i16 & 1) * 8u;
  }
  static __device__ __forceinline__ bf16x8 cols(const unsigned char* tile, unsigned base, int rb, int dtile) {
    const unsigned at = base ^ (unsigned)(dtile * 64);
    s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(tile + rb * ROW + at));
    s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(tile + rb * ROW + 8 * ROW + (at ^ 32u)));     // rows + 8
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
  static __device__ __forceinline__ void read_cols(bf16x8 (&f)[DT], const unsigned char* tile, unsigned cbase, int c) {
#pragma unroll
    for (int d = 0; d < DT; d++) f[d] = cols(tile, cbase, c * 16, d);
  }
  // one row of a head as operand fragments of a product over the width; ok = false: zeros
  static __device__ __forceinline__ void load_frags(const bf16* row, bool ok, int dh, int g, bf16x8 (&f)[KK]) {
#pragma unroll
    for (int kk = 0; kk < KK; kk++) {
      uint4 t = make_uint4(0, 0, 0, 0);
      if (ok && kk * 16 + g * 8 < dh) t = *(const uint4*)(row + kk * 16 + g * 8);
      f[kk] = __builtin_bit_cast(bf16x8, t);
    }
  }
  // the compiler's own wait for fragments just loaded belongs here, not into a loop that has tiles on their way
  static __device__ __forceinline__ void arrived(bf16x8 (&f)[KK]) {
#pragma unroll
    for (int kk = 0; kk < KK; kk++) asm volatile("" : "+v"(f[kk]));
  }
  // acc^T[column, lane] += tile^T p over N rows of a tile, the next 16 rows' fragments read while this one's are multiplied
  template <int N> static __device__ __forceinline__ void cols_times(f32x16 (&acc)[DT], const unsigned char* tile, unsigned cbase, const bf16x8 (&p)[N / 16], bf16x8 (&first)[DT]) {
    bf16x8 f[2][DT];
#pragma unroll
    for (int d = 0; d < DT; d++) f[0][d] = first[d];
#pragma unroll
    for (int c = 0; c < N / 16; c++) {
      if (c < N / 16 - 1) read_cols(f[(c + 1) & 1], tile, cbase, c + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int d = 0; d < DT; d++) acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[c & 1][d], p[c], acc[d], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  // the same with p as two bf16 numbers, which hold 16 bits of it: a is the accumulator layout's tiles of 32 rows
  template <int N> static __device__ __forceinline__ void cols_times_split(f32x16 (&acc)[DT], const unsigned char* tile, unsigned cbase, const f32x16* a, bf16x8 (&first)[DT]) {
    bf16x8 f[2][DT];
#pragma unroll
    for (int d = 0; d < DT; d++) f[0][d] = first[d];
#pragma unroll
    for (int c = 0; c < N / 16; c++) {
      if (c < N / 16 - 1) read_cols(f[(c + 1) & 1], tile, cbase, c + 1);
      const bf16x8 hi = acc_to_frag(a[c >> 1], c & 1);
      bf16x8 lo;
#pragma unroll
      for (int u = 0; u < 8; u++) lo[u] = (__bf16)(a[c >> 1][8 * (c & 1) + u] - (float)hi[u]);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int d = 0; d < DT; d++) acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[c & 1][d], hi, acc[d], 0, 0, 0);
#pragma unroll
      for (int d = 0; d < DT; d++) acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[c & 1][d], lo, acc[d], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  // one row times f; the lanes of a half hold 4 of 8 columns
  static __device__ __forceinline__ void store(bf16* row, const f32x16 (&acc)[DT], float f, int dh, int g) {
#pragma unroll
    for (int d = 0; d < DT; d++)
#pragma unroll
      for (int e = 0; e < 4; e++) {
        bf16x4 r;
#pragma unroll
        for (int i = 0; i < 4; i++) r[i] = (__bf16)(acc[d][e * 4 + i] * f);
        if (d * 32 + e * 8 < dh) *(bf16x4*)(row + d * 32 + e * 8 + g * 4) = r;
      }
  }
  static __device__ __forceinline__ bool finite(const f32x16 (&acc)[DT]) {      // in every lane (a value that is not, times zero, is no number)
    float z[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int d = 0; d < DT; d++)
#pragma unroll
      for (int e = 0; e < 16; e++) z[e & 3] = __builtin_fmaf(acc[d][e], 0.f, z[e & 3]);
    return __all((z[0] + z[1]) + (z[2] + z[3]) == 0.f);
  }
};
__device__ __forceinline__ void phase_end() {     // reads of this phase have returned, then everybody's
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("" ::: "memory");
}
__device__ __forceinline__ float both_halves_max(float x) {       // of lane l and lane l ^ 32
  const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
  return fmaxf(__builtin_bit_cast(float, (unsigned)r[0]), __builtin_bit_cast(float, (unsigned)r[1]));
}
__device__ __forceinline__ float both_halves_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
  return __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
}

// Scores in units of log2: q.k times f, or capped, cap2 tanh(q.k x1), less slope2 times the distance.
enum { CAPPED = 1, BIASED = 2 };                    // the parts that a kernel has (MOD); 0: f is positive
struct ScoreForm { float f, x1, cap2, slope2; };
__device__ __forceinline__ ScoreForm score_form(const RangeAttn& a, int h) {
  ScoreForm s;
  s.f = a.scale * LOG2E;
  s.x1 = a.cap > 0.f ? a.scale / a.cap : 0.f;
  s.cap2 = a.cap * LOG2E;
  s.slope2 = a.slopes ? a.slopes[h] * LOG2E : 0.f;
  return s;
}
// q.k to tanh(q.k x1) where the kernel caps.  Forward (SERIES), up to |x| = 0.8, which the scores of a wave hardly ever pass (a cap is
// there for the ones that do): x times a polynomial in x^2, fitted to the least relative error there (6e-8).  Beyond, and in the
// backward kernels, 1 - 2 / (e^2x + 1), off by some 2^-22, which for a cap of 30 made the error of lse four times as large.  Eight
// multiplications and additions take as long as an exponential and a reciprocal: within 2 % of each other at 4095 x 16 of 64.
template <int MOD, bool SERIES> __device__ __forceinline__ void tanh_scores(const ScoreForm& sf, f32x16& a) {
  if constexpr (MOD & CAPPED) {
    float big = 0.f;
#pragma unroll
    for (int e = 0; e < 16; e += 2) big = fmaxf(fmaxf(big, fabsf(a[e])), fabsf(a[e + 1]));
    if (!SERIES || __any(big * fabsf(sf.x1) > 0.8f)) {
#pragma unroll
      for (int e = 0; e < 16; e++) a[e] = fmaf(-2.f, __builtin_amdgcn_rcpf(fast_exp2(a[e] * (sf.x1 * (2.f * LOG2E))) + 1.f), 1.f);
    } else {
#pragma unroll
      for (int e = 0; e < 16; e++) {
        const float x = a[e] * sf.x1, u = x * x;
        float p = fmaf(u, -4.355297423899174e-3f, 1.909329742193222e-2f);
        p = fmaf(u, p, -5.311431363224983e-2f);
        p = fmaf(u, p, 1.3321048021316528e-1f);
        p = fmaf(u, p, -3.333267569541931e-1f);
        p = fmaf(u, p, 9.999999403953552e-1f);
        a[e] = p * x;
      }
    }
  }
}
// from q.k (its tanh, where the kernel caps) and the distance; keep: what a gradient at the score is multiplied by to be one at scale q.k
template <int MOD> __device__ __forceinline__ float final_score(const ScoreForm& sf, float x, float distance, float* keep) {
  *keep = 1.f;
  if constexpr (MOD & CAPPED) {
    *keep = fmaf(-x, x, 1.f);
    x *= sf.cap2;
  } else x *= sf.f;
  if constexpr (MOD & BIASED) x = fmaf(-sf.slope2, fabsf(distance), x);
  return x;
}
