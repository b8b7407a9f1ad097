// Attention over key ranges, row by row: any head width up to 512, any stride and alignment, float32 or bfloat16 storage
// with float32 arithmetic.  It serves what the matrix-core kernels don't take.  Also the ranges themselves.
#include "attn_range.h"

// One thread per query row; a document's rows are found by bisection of cu_q, from a copy in LDS where that is shorter than a bisection's loads in
// memory: documents, rows, us with and without it, launches back to back: 7, 2048: 2.22 2.34; 100, 8192: 2.47 2.70; 1000, 65536: 3.10 3.17; 2000, 65536: 3.56
// 3.33.  (A launch of its own between others: 4.8.)
#define CU_LDS 1024
__global__ void __launch_bounds__(256) attn_ranges_k(const int* __restrict__ cu_q, const int* __restrict__ cu_k, const int* __restrict__ prefix,
                                                     int n_docs, int causal, int window, int Tq, int Tk, int* __restrict__ lo, int* __restrict__ hi,
                                                     int* __restrict__ at, int* __restrict__ used) {
  const i64 i = (i64)blockIdx.x * 256 + threadIdx.x;
  __shared__ int table[CU_LDS];
  const int *cq = cu_q, *ck = cu_k ? cu_k : cu_q;
  if (cu_q && n_docs < CU_LDS) {
    for (int d = threadIdx.x; d <= n_docs; d += 256) table[d] = cu_q[d];
    __syncthreads();
    cq = table;
    if (!cu_k) ck = table;
  }
  if (i == 0 && used) {
    used[0] = cq ? min(max(cq[n_docs], 0), Tq) : Tq;
    used[1] = ck ? min(max(ck[n_docs], 0), Tk) : Tk;
  }
  if (i >= Tq) return;
  const int eq = Tq / n_docs, ek = Tk / n_docs;
  int doc;
  if (cq) {
    int a = 0, b = n_docs + 1;                      // cu_q[0 .. a - 1] <= i < cu_q[b ..]
    while (a < b) {
      const int m = a + (b - a) / 2;
      if (cq[m] <= i) a = m + 1; else b = m;
    }
    doc = a - 1;
  } else doc = (int)(i / eq);
  i64 l = 0, h = 0, p = 0;
  if (doc >= 0 && doc < n_docs) {
    const i64 q0 = cq ? cq[doc] : (i64)doc * eq, q1 = cq ? cq[doc + 1] : q0 + eq;
    const i64 k0 = ck ? ck[doc] : (i64)doc * ek, k1 = ck ? ck[doc + 1] : k0 + ek;
    p = k1 - q1 + i;                                // the queries are the last of the document's rows
    l = k0;
    h = k1;
    if (causal) {
      h = p + 1;
      if (prefix && k0 + prefix[doc] > h) h = k0 + prefix[doc];
      if (h > k1) h = k1;
      if (window > 0 && p + 1 - window > l) l = p + 1 - window;
    }
  }
  if (l < 0) l = 0;
  if (h > Tk) h = Tk;
  if (l >= h) l = h = 0;
  lo[i] = (int)l;
  hi[i] = (int)h;
  if (at) at[i] = (int)p;
}
void launch_attn_ranges(const int* cu_q, const int* cu_k, const int* prefix, int n_docs, int causal, int window, int Tq, int Tk,
                        int* lo, int* hi, int* at, int* used, hipStream_t s) {
  const int grid = Tq > 0 ? cdiv(Tq, 256) : 1;      // (without rows: `used` alone)
  hipLaunchKernelGGL(attn_ranges_k, dim3(grid), dim3(256), 0, s, cu_q, cu_k, prefix, n_docs, causal, window, Tq, Tk, lo, hi, at, used);
}

// a workgroup is four rows of one head, a wave each
enum { ROW_FWD, ROW_DQ, ROW_DKV };
template <class T, int WHAT> __global__ void __launch_bounds__(256) range_rows_k(RangeAttn a) {
  extern __shared__ float lds[];
  const int heads = WHAT == ROW_DKV ? a.Hkv : a.H, row4 = (int)(blockIdx.x / heads), h = (int)blockIdx.x - row4 * heads;
  const int w = threadIdx.x >> 6, r = row4 * 4 + w, rows = rows_in_use(a), keys = keys_in_use(a);
  float* mine = lds + w * 2 * a.dh;
  if (r >= (WHAT == ROW_DKV ? keys : rows)) return;
  if constexpr (WHAT == ROW_FWD) range_row_fwd<T>(a, r, h, keys, mine);
  else if constexpr (WHAT == ROW_DQ) range_row_dq<T>(a, r, h, keys, mine);
  else range_row_dkv<T>(a, r, h, rows, keys, mine);
}
template <int WHAT> static void rows(const RangeAttn& a, int n, int heads, hipStream_t s) {
  if (n <= 0) return;
  const dim3 grid((unsigned)((i64)cdiv(n, 4) * heads));
  const size_t smem = (size_t)4 * 2 * a.dh * 4;
  if (a.dt == 0) hipLaunchKernelGGL((range_rows_k<float, WHAT>), grid, dim3(256), smem, s, a);
  else hipLaunchKernelGGL((range_rows_k<bf16, WHAT>), grid, dim3(256), smem, s, a);
}
void launch_range_fwd_rows(const RangeAttn& a, hipStream_t s) { rows<ROW_FWD>(a, a.Tq, a.H, s); }
void launch_range_bwd_rows(const RangeAttn& a, hipStream_t s) {
  rows<ROW_DQ>(a, a.Tq, a.H, s);                    // (writes D, which the other one reads)
  rows<ROW_DKV>(a, a.Tk, a.Hkv, s);
}
