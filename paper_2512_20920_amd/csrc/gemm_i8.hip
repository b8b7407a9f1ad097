// Products of 8-bit integers on the matrix cores: c[m, n] = (sum_k a[m, k] b[n, k]) sa[m] sb[n] + bias[n], both operands rows x k (a layer's
// tokens and its weights' output channels), sums exact in 32-bit integers, one rounding to the result's type after float32 products.
//
// v_mfma_i32_32x32x32_i8 takes 16 bytes of a row per lane, as the bfloat16 instruction does, for twice as many k's; so a k-tile is
// 128 bytes of each row and lies in LDS as in operand_bf16.h: 16-byte chunk c of row r in place c ^ ((r >> 1) & 7), filled
// by loads straight from memory.  Rows past the end, and chunks past k, are loaded as zeros; the bytes of the last chunk that lie past k are
// cleared in a's fragments.
#include "lds_load.h"

typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(16))) int i32x16;

namespace {

constexpr int KB = 128;                  // bytes of k per tile

// rows row0 .. of an operand as a buffer: offsets count from row0, what lies behind the last row reads as zeros
__device__ __forceinline__ u32x4 rows_desc(const signed char* p, i64 ld, int row0, int rows, int K) {
  const unsigned long long at = (unsigned long long)(p + (i64)row0 * ld);
  const i64 n = rows > row0 ? ((i64)(rows - row0 - 1) * ld + K + 3) & ~3ll : 0;
  u32x4 d = {(unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)at), (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)(at >> 32)),
             (unsigned)__builtin_amdgcn_readfirstlane((int)(n < (i64)OOB ? n : (i64)OOB)), 0x00020000u};
  return d;
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

template <class T, int BM, int BN, int WGM, int NW, int NS> void go(const GemmI8& g, hipStream_t s) {
  constexpr size_t smem = (size_t)NS * (BM + BN) * KB;
  static std::atomic<unsigned long long> attr_mask{0};
  if (attr_needed(attr_mask)) {
    (void)hipFuncSetAttribute((const void*)gemm_i8_k<T, BM, BN, WGM, NW, NS>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    attr_done(attr_mask);
  }
  const i64 tiles = (i64)cdiv(g.M, BM) * cdiv(g.N, BN);
  hipLaunchKernelGGL((gemm_i8_k<T, BM, BN, WGM, NW, NS>), dim3((unsigned)((tiles + 7) / 8 * 8)), dim3(NW * 64), smem, s, g);
}
template <class T> void go(const GemmI8& g, int form, hipStream_t s) {
  if (form == 1) hipLaunchKernelGGL((gemm_i8_any_k<T>), dim3(cdiv(g.N, 256), g.M < 4096 ? g.M : 4096), dim3(256), 0, s, g);
  else go<T, 128, 128, 4, 8, 4>(g, s);
}

}  // namespace

bool gemm_i8_takes(const GemmI8& g) {
  return (g.lda | g.ldb) % 16 == 0 && ((uintptr_t)g.a | (uintptr_t)g.b) % 16 == 0 && g.lda < (1 << 22) && g.ldb < (1 << 22);
}
void launch_gemm_i8(const GemmI8& g, int form, hipStream_t s) {
  if (g.M < 1 || g.N < 1) return;
  if (g.dt == 0) go<float>(g, form, s); else go<bf16>(g, form, s);
}
