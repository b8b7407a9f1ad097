// Products of 8-bit integers on the matrix cores: c[m, n] = (sum_k a[m, k] b[n, k]) sa[m] sb[n] + bias[n], both operands rows x k (a layer's
// tokens and its weights' output channels), sums exact in 32-bit integers, one rounding to the result's type after float32 products.
//
// v_mfma_i32_32x32x32_i8 takes 16 bytes of a row per lane, as the bfloat16 instruction does, for twice as many k's; so a k-tile is
// 128 bytes of each row and lies in LDS as in operand_bf16.h: 16-byte chunk c of row r in place c ^ ((r >> 1) & 7), filled
// by loads straight from memory.  Rows past the end, and chunks past k, are loaded as zeros; the bytes of the last chunk that lie past k are
// cleared in a's fragments.
#include "lds_load.h"
#include <math.h>

typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(16))) int i32x16;

namespace {

constexpr int KB = 128;                  // bytes of k per tile

// rows row0 .. of an operand as a buffer: offsets count from row0, what lies behind the last row reads as zeros.  As the four words that loads into LDS take,
// and as what loads into registers do.
__device__ __forceinline__ unsigned rows_bytes(i64 ld, int row0, int rows, int K) {
  const i64 n = rows > row0 ? ((i64)(rows - row0 - 1) * ld + K + 3) & ~3ll : 0;
  return (unsigned)(n < (i64)OOB ? n : (i64)OOB);
}
__device__ __forceinline__ u32x4 rows_desc(const signed char* p, i64 ld, int row0, int rows, int K) {
  const unsigned long long at = (unsigned long long)(p + (i64)row0 * ld);
  u32x4 d = {(unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)at), (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)(at >> 32)),
             (unsigned)__builtin_amdgcn_readfirstlane((int)rows_bytes(ld, row0, rows, K)), 0x00020000u};
  return d;
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_of(const signed char* p, i64 ld, int row0, int rows, int K) {
  return __builtin_amdgcn_make_buffer_rsrc((void*)(p + (i64)row0 * ld), (short)0, (int)rows_bytes(ld, row0, rows, K), 0x00020000);
}
__device__ __forceinline__ i32x4 fragment(const unsigned char* tile, int r, int kk, int lane) {
  return *(const i32x4*)(tile + r * KB + (((kk * 2 + (lane >> 5)) ^ ((r >> 1) & 7)) << 4));
}
__device__ __forceinline__ i32x16 mfma(i32x4 a, i32x4 b, i32x16 c) { return __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, c, 0, 0, 0); }
// the first n bytes of a chunk
__device__ __forceinline__ i32x4 first_bytes(i32x4 v, int n) {
#pragma unroll
  for (int i = 0; i < 4; i++) { const int b = min(max(n - 4 * i, 0), 4); v[i] &= b == 4 ? ~0 : (1 << (8 * b)) - 1; }
  return v;
}

// Two neighbouring lanes (columns n, n + 1) hold rows r and r + 1: after the swap the even lane has row r, the odd one r + 1, both columns.
__device__ __forceinline__ void pair_rows(bool odd, float x0, float x1, float* left, float* right) {
  const float send = odd ? x0 : x1;
  const float recv = __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, send), 0xB1, 0xf, 0xf, false));
  *left = odd ? recv : x0;
  *right = odd ? x1 : recv;
}
// 32 x 32 sums at row m0, column n0 to their results.  Lane: column lane & 31, rows 8 (e >> 2) + 4 (lane >> 5) + (e & 3).
template <class T> __device__ __forceinline__ void put_block(const GemmI8& g, int m0, int n0, const i32x16& acc) {
  const int lane = threadIdx.x & 63, n = n0 + (lane & 31), mb = m0 + 4 * (lane >> 5);
  const float sb = g.sb[min(n, g.N - 1)], bias = g.bias ? to_f(((const T*)g.bias)[min(n, g.N - 1)]) : 0.f;
  float v[16];
#pragma unroll
  for (int e = 0; e < 16; e++) {
    const int m = min(mb + 8 * (e >> 2) + (e & 3), g.M - 1);
    v[e] = fmaf((float)acc[e] * g.sa[m], sb, bias);
  }
  T* c = (T*)g.c;
  if (sizeof(T) == 2 && !(g.ldc & 1) && !((uintptr_t)c & 3)) {
    const bool odd = lane & 1;
    typedef __attribute__((ext_vector_type(2))) T V2;
#pragma unroll
    for (int e = 0; e < 16; e += 2) {
      float l, r;
      pair_rows(odd, v[e], v[e + 1], &l, &r);
      const int m = mb + 8 * (e >> 2) + (e & 3) + (odd ? 1 : 0), nl = n - (odd ? 1 : 0);
      if (m < g.M) {
        T* p = c + (i64)m * g.ldc + nl;
        if (nl + 1 < g.N) { V2 w; w[0] = from_f<T>(l); w[1] = from_f<T>(r); *(V2*)p = w; }
        else if (nl < g.N) *p = from_f<T>(l);
      }
    }
    return;
  }
#pragma unroll
  for (int e = 0; e < 16; e++) {
    const int m = mb + 8 * (e >> 2) + (e & 3);
    if (m < g.M && n < g.N) c[(i64)m * g.ldc + n] = from_f<T>(v[e]);
  }
}

// Which tile a workgroup takes: consecutive ids go to the eight XCDs in turn, and each XCD gets a run of tiles that walks down 8 rows of
// tiles before it moves a column on, so that it finds both operands in its L2.
__device__ __forceinline__ bool place(int tiles_m, int tiles_n, int* by, int* bx) {
  const int all = tiles_m * tiles_n, per = (all + 7) / 8, t = (int)(blockIdx.x & 7) * per + (int)(blockIdx.x >> 3);
  if ((int)(blockIdx.x >> 3) >= per || t >= all) return false;
  const int band = t / (8 * tiles_n), rows = min(8, tiles_m - band * 8), in = t - band * 8 * tiles_n;
  *bx = in / rows;
  *by = band * 8 + in - *bx * rows;
  return true;
}

// ---- tiles of BM x BN, waves WGM x (NW / WGM), NS stages of LDS: NS - 1 k-tiles are on their way while one is multiplied ----
template <class T, int BM, int BN, int WGM, int NW, int NS>
__global__ void __launch_bounds__(NW * 64) gemm_i8_k(GemmI8 g) {
  constexpr int WM = BM / WGM, WN = BN / (NW / WGM), TM = WM / 32, TN = WN / 32, STAGE = (BM + BN) * KB;
  constexpr int LOADS = (BM + BN) * KB / 1024 / NW, ALOADS = BM * KB / 1024;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  int by, bx;
  if (!place((g.M + BM - 1) / BM, (g.N + BN - 1) / BN, &by, &bx)) return;
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = (wv / (NW / WGM)) * WM, wn = (wv % (NW / WGM)) * WN, m0 = by * BM, n0 = bx * BN;
  const u32x4 da = rows_desc(g.a, g.lda, m0, g.M, g.K), db = rows_desc(g.b, g.ldb, n0, g.N, g.K);
  const int nk = (g.K + KB - 1) / KB;
  unsigned base[LOADS];
  int chunk[LOADS];                                  // first k of the chunk in a tile
#pragma unroll
  for (int i = 0; i < LOADS; i++) {
    const int j = wv * LOADS + i, pos = (j < ALOADS ? j : j - ALOADS) * 64 + lane, r = pos >> 3, c = (pos & 7) ^ ((r >> 1) & 7);
    const bool in = j < ALOADS ? m0 + r < g.M : n0 + r < g.N;
    base[i] = in ? (unsigned)r * (unsigned)(j < ALOADS ? g.lda : g.ldb) + c * 16u : OOB;
    chunk[i] = c * 16;
  }
  const unsigned lw = __builtin_amdgcn_readfirstlane(lds_address(smem) + (unsigned)wv * LOADS * 1024u);
  auto issue = [&](int kt, int i) {
    const unsigned off = base[i] != OOB && kt * KB + chunk[i] < g.K ? base[i] + (unsigned)kt * KB : OOB;
    load_lds_b128(wv * LOADS + i < ALOADS ? da : db, lw + (unsigned)(kt % NS) * STAGE + i * 1024u, off);
  };
  i32x16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; i++)
#pragma unroll
    for (int j = 0; j < TN; j++) acc[i][j] = i32x16{};
#pragma unroll
  for (int p = 0; p < NS - 1; p++)
#pragma unroll
    for (int i = 0; i < LOADS; i++) issue(p, i);
  for (int kt = 0; kt < nk; kt++) {
    wait_vmcnt<LOADS * (NS - 2)>();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    const unsigned char* st = smem + (kt % NS) * STAGE;
    const bool ragged = (kt + 1) * KB > g.K && (g.K & 15);
#pragma unroll
    for (int kk = 0; kk < 4; kk++) {
#pragma unroll
      for (int i = kk * LOADS / 4; i < (kk + 1) * LOADS / 4; i++) issue(kt + NS - 1, i);
      i32x4 fa[TM], fb[TN];
#pragma unroll
      for (int i = 0; i < TM; i++) fa[i] = fragment(st, wm + i * 32 + (lane & 31), kk, lane);
#pragma unroll
      for (int j = 0; j < TN; j++) fb[j] = fragment(st + BM * KB, wn + j * 32 + (lane & 31), kk, lane);
      if (ragged) {
#pragma unroll
        for (int i = 0; i < TM; i++) fa[i] = first_bytes(fa[i], g.K - kt * KB - kk * 32 - (lane >> 5) * 16);
      }
#pragma unroll
      for (int i = 0; i < TM; i++)
#pragma unroll
        for (int j = 0; j < TN; j++) acc[i][j] = mfma(fa[i], fb[j], acc[i][j]);
    }
  }
  wait_vmcnt<0>();                                   // the zero-filled loads past the last tile
#pragma unroll
  for (int i = 0; i < TM; i++)
#pragma unroll
    for (int j = 0; j < TN; j++)
      if (m0 + wm + i * 32 < g.M && n0 + wn + j * 32 < g.N) put_block<T>(g, m0 + wm + i * 32, n0 + wn + j * 32, acc[i][j]);
}

// ---- 256 x 256 in phases ----
// A k-tile is two phases over half tiles, each half tile refilled as soon as it has been read, and the two waves of a SIMD are half a phase apart: one
// multiplies while the other reads its fragments and asks for loads (the scheme of gemm_mfma.hip's tile, whose barriers and counts these are):
//   phase 0: read A0 B0 B1, multiply A0 x (B0 B1), ask for A1 of k-tile t + 1
//   phase 1: read A1,       multiply A1 x (B0 B1), ask for A0 B0 B1 of k-tile t + 2
// 8 waves as 2 x 4, a wave owns 64 rows x 2 x 32 columns of each half.  At the end of a read segment a wave waits for all but its youngest 8
// loads, which covers the half tiles that the next phase reads; fragments are in registers when it ends, so a half tile is overwritten only after
// everybody has read it.
template <class T> __global__ void __launch_bounds__(512) gemm_i8_phased_k(GemmI8 g) {
  constexpr unsigned HALF = 128 * KB, STAGE = 4 * HALF;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  int by, bx;
  if (!place((g.M + 255) / 256, (g.N + 255) / 256, &by, &bx)) return;
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m0 = by * 256, n0 = bx * 256;
  const int wm = (wv >> 2) * 64, wn = (wv & 3) * 32;  // inside a half
  const u32x4 da = rows_desc(g.a, g.lda, m0, g.M, g.K), db = rows_desc(g.b, g.ldb, n0, g.N, g.K);
  const int nk = (g.K + KB - 1) / KB, whole = g.K / KB;
  unsigned base[4][2];
  int chunk[2];
#pragma unroll
  for (int i = 0; i < 2; i++) {
    const int pos = (wv * 2 + i) * 64 + lane, r = pos >> 3, c = (pos & 7) ^ ((r >> 1) & 7);
    chunk[i] = c * 16;
#pragma unroll
    for (int h = 0; h < 2; h++) {
      base[h][i] = m0 + h * 128 + r < g.M ? (unsigned)(h * 128 + r) * (unsigned)g.lda + c * 16u : OOB;
      base[2 + h][i] = n0 + h * 128 + r < g.N ? (unsigned)(h * 128 + r) * (unsigned)g.ldb + c * 16u : OOB;
    }
  }
  const unsigned lw = __builtin_amdgcn_readfirstlane(lds_address(smem) + (unsigned)wv * 2048u);
  auto issue = [&](int kt, int hf) {                 // this wave's part of half tile hf (A0 A1 B0 B1) of k-tile kt
    const unsigned dst = lw + (unsigned)(kt & 1) * STAGE + hf * HALF, soff = (unsigned)kt * KB;
#pragma unroll
    for (int i = 0; i < 2; i++)
      load_lds_b128_s(hf < 2 ? da : db, dst + i * 1024u, kt < whole || kt * KB + chunk[i] < g.K ? base[hf][i] : OOB, soff);
  };
  i32x16 acc[4][2];
#pragma unroll
  for (int i = 0; i < 4; i++)
#pragma unroll
    for (int j = 0; j < 2; j++) acc[i][j] = i32x16{};
  auto issue3 = [&](int kt) { issue(kt, 0); issue(kt, 2); issue(kt, 3); };
  issue3(0); issue(0, 1);
  issue3(1);
  wait_vmcnt<8>();                                   // A0 B0 B1 of k-tile 0
  __builtin_amdgcn_s_barrier();
  if (wv >= 4) __builtin_amdgcn_s_barrier();         // waves 4-7 half a phase behind
  const bool lower = g.M - m0 > 128;
  i32x4 fa[2][4], fb[2][4];
  for (int kt = 0; kt < nk; kt++) {
    const unsigned char* st = smem + (unsigned)(kt & 1) * STAGE;
    const bool ragged = kt == whole && (g.K & 15);
#pragma unroll
    for (int p = 0; p < 2; p++) {
      if (p == 0 || lower) {
#pragma unroll
        for (int kk = 0; kk < 4; kk++) {
#pragma unroll
          for (int i = 0; i < 2; i++) fa[i][kk] = fragment(st + p * HALF, wm + i * 32 + (lane & 31), kk, lane);
          if (p == 0)
#pragma unroll
            for (int j = 0; j < 2; j++) fb[j][kk] = fragment(st + (2 + j) * HALF, wn + (lane & 31), kk, lane);
        }
        if (ragged) {
#pragma unroll
          for (int kk = 0; kk < 4; kk++)
#pragma unroll
            for (int i = 0; i < 2; i++) fa[i][kk] = first_bytes(fa[i][kk], g.K - kt * KB - kk * 32 - (lane >> 5) * 16);
        }
      }
      if (p == 0) issue(kt + 1, 1); else issue3(kt + 2);
      wait_vmcnt<8>();
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(1);
      if (p == 0 || lower)
#pragma unroll
      for (int kk = 0; kk < 4; kk++)
#pragma unroll
        for (int i = 0; i < 2; i++)
#pragma unroll
          for (int j = 0; j < 2; j++) acc[p * 2 + i][j] = mfma(fa[i][kk], fb[j][kk], acc[p * 2 + i][j]);
      __builtin_amdgcn_s_setprio(0);
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
    }
  }
  if (wv < 4) __builtin_amdgcn_s_barrier();
  wait_vmcnt<0>();                                   // the zero-filled loads past the last k-tile
#pragma unroll
  for (int i = 0; i < 4; i++)
#pragma unroll
    for (int j = 0; j < 2; j++) {
      const int m = m0 + (i >> 1) * 128 + wm + (i & 1) * 32, n = n0 + j * 128 + wn;
      if (m < g.M && n < g.N) put_block<T>(g, m, n, acc[i][j]);
    }
}

// ---- a few rows: tiles of 32 x 32, whose k-tiles the eight waves share out ----
// Reading b bounds it, of which every workgroup asks for all that it needs at once, or nearly: no k-tile waits for another one's place in LDS.
// Fragments come from memory as they are, a row's 128 bytes by four loads; the waves' sums meet in LDS.
template <class T> __global__ void __launch_bounds__(512) gemm_i8_few_k(GemmI8 g) {
  constexpr int NW = 8;
  __shared__ int part[NW][1024];
  const int tiles_n = (g.N + 31) / 32, by = (int)blockIdx.x / tiles_n, m0 = by * 32, n0 = ((int)blockIdx.x - by * tiles_n) * 32;
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 31, c = (lane >> 5) * 16;
  const __amdgpu_buffer_rsrc_t ra = rows_of(g.a, g.lda, m0, g.M, g.K), rb = rows_of(g.b, g.ldb, n0, g.N, g.K);
  const unsigned ba = m0 + r < g.M ? (unsigned)r * (unsigned)g.lda + c : OOB, bb = n0 + r < g.N ? (unsigned)r * (unsigned)g.ldb + c : OOB;
  i32x16 acc = {};
  for (int kt = wv; kt * KB < g.K; kt += 2 * NW) {
    i32x4 fa[2][4], fb[2][4];
#pragma unroll
    for (int u = 0; u < 2; u++)
#pragma unroll
      for (int kk = 0; kk < 4; kk++) {
        const int k = (kt + u * NW) * KB + kk * 32;
        const bool in = k + c < g.K;
        fb[u][kk] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rb, in ? bb + k : OOB, 0, 0));
        fa[u][kk] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(ra, in ? ba + k : OOB, 0, 0));
      }
#pragma unroll
    for (int u = 0; u < 2; u++)
#pragma unroll
      for (int kk = 0; kk < 4; kk++) {
        const int k = (kt + u * NW) * KB + kk * 32;
        if (k + 32 > g.K && (g.K & 15)) fa[u][kk] = first_bytes(fa[u][kk], g.K - k - c);
        acc = mfma(fa[u][kk], fb[u][kk], acc);
      }
  }
#pragma unroll
  for (int e = 0; e < 16; e++) part[wv][e * 64 + lane] = acc[e];
  __syncthreads();
  for (int j = threadIdx.x; j < 1024; j += NW * 64) {
    const int e = j >> 6, l = j & 63, m = m0 + 8 * (e >> 2) + 4 * (l >> 5) + (e & 3), n = n0 + (l & 31);
    if (m >= g.M || n >= g.N) continue;
    int s = 0;
#pragma unroll
    for (int w = 0; w < NW; w++) s += part[w][j];
    const float bias = g.bias ? to_f(((const T*)g.bias)[n]) : 0.f;
    ((T*)g.c)[(i64)m * g.ldc + n] = from_f<T>(fmaf((float)s * g.sa[m], g.sb[n], bias));
  }
}

// ---- any shape and alignment: a thread per result ----
template <class T> __global__ void __launch_bounds__(256) gemm_i8_any_k(GemmI8 g) {
  const int n = blockIdx.x * 256 + threadIdx.x;
  if (n >= g.N) return;
  const signed char* b = g.b + (i64)n * g.ldb;
  const float sb = g.sb[n], bias = g.bias ? to_f(((const T*)g.bias)[n]) : 0.f;
  for (int m = blockIdx.y; m < g.M; m += gridDim.y) {
    const signed char* a = g.a + (i64)m * g.lda;
    int s = 0;
    for (int k = 0; k < g.K; k++) s += (int)a[k] * (int)b[k];
    ((T*)g.c)[(i64)m * g.ldc + n] = from_f<T>(fmaf((float)s * g.sa[m], sb, bias));
  }
}

// The matrix-core shapes: rows and columns of a tile, threads, workgroups that all CUs hold at once, and what a round of those takes per 128 k's
struct Shape { int bm, bn, threads, round; float us; };
constexpr Shape SHAPES[] = {{256, 256, 512, 256, 1.93f}, {128, 256, 512, 256, 1.20f}, {128, 128, 512, 256, 0.72f}, {64, 64, 256, 512, 0.49f}, {32, 32, 512, 0, 0.f}};
constexpr int FIRST = 2, FEW = 6;                    // forms of the first shape and of the last, which splits k instead
static_assert(sizeof(SHAPES) / sizeof(Shape) == GEMM_I8_FORMS && FIRST + GEMM_I8_FORMS - 1 == FEW, "forms 2 .. are the shapes in order");
i64 tiles_of(const GemmI8& g, const Shape& x) { return ((i64)g.M + x.bm - 1) / x.bm * (((i64)g.N + x.bn - 1) / x.bn); }
bool launches(const GemmI8& g, const Shape& x) { return (tiles_of(g, x) + 7) / 8 * 8 * x.threads < (i64)1 << 32; }

template <class K> void launch(K kernel, std::atomic<unsigned long long>& attr_mask, int form, size_t smem, const GemmI8& g, hipStream_t s) {
  if (attr_needed(attr_mask)) {
    (void)hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    attr_done(attr_mask);
  }
  const Shape& x = SHAPES[form - FIRST];
  hipLaunchKernelGGL(kernel, dim3((unsigned)((tiles_of(g, x) + 7) / 8 * 8)), dim3(x.threads), smem, s, g);
}
template <class T, int FORM, int WGM, int NS> void go(const GemmI8& g, hipStream_t s) {
  static std::atomic<unsigned long long> mask{0};
  constexpr Shape X = SHAPES[FORM - FIRST];
  launch(gemm_i8_k<T, X.bm, X.bn, WGM, X.threads / 64, NS>, mask, FORM, (size_t)NS * (X.bm + X.bn) * KB, g, s);
}
// Which shape a product gets: the one with the least rounds of workgroups times what a round takes per 128 k's (us, measured with every CU busy):
//   256 x 256 in phases 1.93, 128 x 256 1.20, 128 x 128 0.72, 64 x 64 (two per CU) 0.49.
// Measured, bfloat16 results, us for these four: 8192 x 14336, k 4096: 437 541 648 886 (2.2 * 10^15 multiplications and additions a second); 8192 x 2048,
// k 2048: 39 45 50 71; 2048 x 11264, k 2048: 66 63 73 96; 611 x 11264, k 2048: 30 22 25 33; 2048 x 2048, k 2048: 29 19 15 19; 611 x 2048, k 2048:
// 28 18 12 11; 256 x 4096, k 4096: 44 28 19 15; 8 x 6144, k 2048: 20 15 11 8.
// A tile of 32 x 32 each, where no CU gets two (us, then the best of the others): 8 x 6144, k 2048: 5.2, 8.1; 48 x 4096, k 14336: 27, 39; 128 x 2048, k 5632:
// 12.9, 17.3; beyond, 48 x 6144, k 2048: 8.9, 8.5; 8 x 14336, k 4096: 14.5, 13.6; 128 x 4096, k 14336: 52, 39.
int form_for(const GemmI8& g) {
  if (tiles_of(g, SHAPES[FEW - FIRST]) <= 256) return FEW;
  int best = FIRST;
  float least = INFINITY;
  for (int form = FIRST; form < FEW; form++) {
    const Shape& x = SHAPES[form - FIRST];
    const float cost = (float)((tiles_of(g, x) + x.round - 1) / x.round) * x.us;
    if (cost < least && launches(g, x)) { least = cost; best = form; }
  }
  return best;
}
template <class T> void go(const GemmI8& g, int form, hipStream_t s) {
  static std::atomic<unsigned long long> mask{0};
  switch (form ? form : form_for(g)) {
    case 1: {                                        // (2^31 threads at most)
      const int blocks = cdiv(g.N, 256), most = (1 << 23) / blocks;
      hipLaunchKernelGGL((gemm_i8_any_k<T>), dim3(blocks, g.M < 4096 ? (g.M < most ? g.M : most) : (most < 4096 ? most : 4096)), dim3(256), 0, s, g);
      break;
    }
    case 2: launch(gemm_i8_phased_k<T>, mask, 2, 2 * 512 * KB, g, s); break;
    case 3: go<T, 3, 2, 3>(g, s); break;
    case 4: go<T, 4, 4, 4>(g, s); break;
    case FEW: hipLaunchKernelGGL((gemm_i8_few_k<T>), dim3((unsigned)tiles_of(g, SHAPES[FEW - FIRST])), dim3(512), 0, s, g); break;
    default: go<T, 5, 2, 4>(g, s);
  }
}

}  // namespace

bool gemm_i8_takes(const GemmI8& g) {
  return (g.lda | g.ldb) % 16 == 0 && ((uintptr_t)g.a | (uintptr_t)g.b) % 16 == 0 && g.lda < (1 << 22) && g.ldb < (1 << 22);
}
// M, N below 2^30 and fewer than 2^36 results: 256 x 256 always does, and the slow kernel
bool gemm_i8_launches(const GemmI8& g, int form) {
  return g.M < 1 << 30 && g.N < 1 << 30 && (i64)g.M * g.N < (i64)1 << 36 && (form < FIRST || launches(g, SHAPES[form - FIRST]));
}
void launch_gemm_i8(const GemmI8& g, int form, hipStream_t s) {
  if (g.M < 1 || g.N < 1) return;
  if (g.dt == 0) go<float>(g, form, s); else go<bf16>(g, form, s);
}
