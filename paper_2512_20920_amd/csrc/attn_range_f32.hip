// Attention over key ranges in float32 on the matrix cores (v_mfma_f32_32x32x2_f32), heads of up to 128 columns (a multiple of 4).
//
// Transposed score tiles: in S^T[key, row] = K Q^T a lane owns one row, element e of the result is key (e >> 2) * 8 + (lane >> 5)
// * 4 + (e & 3), and that is what the second product wants as its operand: instruction e contracts over the two keys that
// the two halves of the wave hold in element e.  So probabilities stay in the registers they were computed in, at full
// precision, and keys and values are read from memory as operands directly: K 16 bytes of its own row per lane, V a row of 32
// consecutive columns per half.  32 rows (keys) per workgroup, tiles of 32 shared out to the waves.
// Bound by the matrix pipe's 64 clocks per instruction and, in small calls, the chain of loads around them: 2048 rows x 16 heads of 128
// (documents of 1500 and 548) 167, 229 and 328 us, 62 to 68 of the 154 TFLOP/s of a large float32 product; 751 x 4 of 64: 13, 19, 23.
#include "attn_range_few.h"

typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) float f32x4;

__device__ __forceinline__ int elem_row(int e, int half) { return (e >> 2) * 8 + half * 4 + (e & 3); }
__device__ __forceinline__ float half_sum(float v) { return v + __shfl_xor(v, 32, WAVE); }
// this lane's half of a row as an operand of a product over the width: columns 8 c + 4 half .. + 3
template <int DHP> __device__ __forceinline__ void load_row(const float* row, bool ok, int dh, int half, float f, float (&r)[DHP / 2]) {
#pragma unroll
  for (int c = 0; c < DHP / 8; c++) {
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (ok && c * 8 + half * 4 < dh) v = *(const f32x4*)(row + c * 8 + half * 4);
#pragma unroll
    for (int i = 0; i < 4; i++) r[c * 4 + i] = v[i] * f;
  }
}
// Products of a tile's rows, read from memory, go in groups of 16 instructions (128 columns; about 1000 clocks), the next group's loads on
// their way meanwhile.
template <int DHP> struct Chunks {                   // a group of a row's chunks of 4 columns: c = 4 n .. 4 n + 3
  f32x4 v[4];
  __device__ __forceinline__ void load(const float* row, int dh, int half, int n) {
#pragma unroll
    for (int c = 0; c < 4; c++) {
      const int col = (n * 4 + c) * 8 + half * 4;
      v[c] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (col < dh) v[c] = *(const f32x4*)(row + col);
    }
  }
  template <class F> __device__ __forceinline__ void times(f32x16& a, int n, F other) const {      // other(c): 4 columns of the other operand
#pragma unroll
    for (int c = 0; c < 4; c++) {
      const f32x4 o = other(n * 4 + c);
#pragma unroll
      for (int i = 0; i < 4; i++) a = __builtin_amdgcn_mfma_f32_32x32x2f32(v[c][i], o[i], a, 0, 0, 0);
    }
  }
};
template <int DHP> __device__ __forceinline__ f32x4 piece(const float (&r)[DHP / 2], int c) { return f32x4{r[c * 4], r[c * 4 + 1], r[c * 4 + 2], r[c * 4 + 3]}; }
template <int DHP, class F> __device__ __forceinline__ f32x16 scores(const float* row, int dh, int half, F other) {
  constexpr int N = DHP / 32;
  Chunks<DHP> x[2];
  f32x16 a = {};
  x[0].load(row, dh, half, 0);
#pragma unroll
  for (int n = 0; n < N; n++) {
    if (n < N - 1) x[(n + 1) & 1].load(row, dh, half, n + 1);
    __builtin_amdgcn_sched_barrier(0);
    x[n & 1].times(a, n, other);
    __builtin_amdgcn_sched_barrier(0);
  }
  return a;
}
// two products of that kind one after the other
template <int DHP, class F, class G> __device__ __forceinline__ void scores2(f32x16& a, f32x16& b, const float* ra, const float* rb, int dh, int half, F fa, G fb) {
  constexpr int N = DHP / 32;
  Chunks<DHP> x[2];
  a = f32x16{};
  b = f32x16{};
  x[0].load(ra, dh, half, 0);
#pragma unroll
  for (int n = 0; n < 2 * N; n++) {
    if (n < 2 * N - 1) x[(n + 1) & 1].load(n + 1 < N ? ra : rb, dh, half, (n + 1) % N);
    __builtin_amdgcn_sched_barrier(0);
    if (n < N) x[n & 1].times(a, n, fa);
    else x[n & 1].times(b, n - N, fb);
    __builtin_amdgcn_sched_barrier(0);
  }
}
// acc^T[column, lane] += X^T[column, row] p[row, lane] over the 32 rows of X from r0 on (rows past the last one are that one: p is
// zero there); group n: elements 4 n .. 4 n + 3.  The first group is loaded ahead.
template <int DHP> struct Columns {
  float v[4][DHP / 32];
  __device__ __forceinline__ void load(const float* x, i64 ld, int dh, int r0, int last, int lane, int n) {
#pragma unroll
    for (int e = 0; e < 4; e++) {
      const float* row = x + (i64)min(r0 + elem_row(n * 4 + e, lane >> 5), last) * ld + (lane & 31);
#pragma unroll
      for (int i = 0; i < DHP / 32; i++) v[e][i] = (lane & 31) + i * 32 < dh ? row[i * 32] : 0.f;
    }
  }
};
template <int DHP> __device__ __forceinline__ void accumulate(f32x16 (&acc)[DHP / 32], const Columns<DHP>& first, const float* x, i64 ld, int dh, int r0, int last, const f32x16& p, int lane) {
  Columns<DHP> c[2];
  c[0] = first;
#pragma unroll
  for (int n = 0; n < 4; n++) {
    if (n < 3) c[(n + 1) & 1].load(x, ld, dh, r0, last, lane, n + 1);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int e = 0; e < 4; e++)
#pragma unroll
      for (int i = 0; i < DHP / 32; i++) acc[i] = __builtin_amdgcn_mfma_f32_32x32x2f32(c[n & 1].v[e][i], p[n * 4 + e], acc[i], 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
  }
}
// a wave's accumulators to LDS, [column][32 rows]
template <int DHP> __device__ __forceinline__ void spill(float* t, const f32x16 (&acc)[DHP / 32], int lane) {
#pragma unroll
  for (int i = 0; i < DHP / 32; i++)
#pragma unroll
    for (int e = 0; e < 16; e++) t[(i * 32 + elem_row(e, lane >> 5)) * 32 + (lane & 31)] = acc[i][e];
}
// CAP: with the tanh, whose code the other calls would fetch for nothing
template <int DHP, int NW, bool CAP> __global__ void __launch_bounds__(NW * 64, 2) range_fwd_f32_k(RangeAttn a, FewShape f) {
  extern __shared__ float sm[];                      // NW results [DHP][32], statistics
  int tile, split, head, t0;
  few_place(a, f, (int)blockIdx.x, &tile, &split, &head);
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, kh = head % a.Hkv;
  FewRow row = few_row(a, f, tile, head, lane & 31, a.Tq);
  const int2 stored = stored_range(a, row.i);
  const float slope = a.slopes ? a.slopes[row.h] : 0.f;
  const int at = row.ok && a.at ? a.at[row.i] : row.i;
  const float *k = (const float*)a.k + (i64)kh * a.dh, *v = (const float*)a.v + (i64)kh * a.dh;
  float qf[DHP / 2];
  load_row<DHP>((const float*)a.q + (i64)row.i * a.ldq + (i64)row.h * a.dh, row.ok, a.dh, half, a.scale, qf);
  const int rows = rows_in_use(a), keys = keys_in_use(a);
  if (tile * f.qpt >= rows) return;
  row.ok = row.ok && row.i < rows;
  const FewKeys fk = few_keys(f, row, stored, split, keys, &t0);
  f32x16 acc[DHP / 32] = {};
  float m = -INFINITY, l = 0.f;
  for (int t = fk.live_from(t0 + wv, NW); t < fk.t1; t = fk.live_from(t + NW, NW)) {
    const int kv = fk.first + t * 32;
    f32x16 s = scores<DHP>(k + (i64)min(kv + (lane & 31), fk.end - 1) * a.ldk, a.dh, half, [&](int c) { return piece<DHP>(qf, c); });
    Columns<DHP> first;
    first.load(v, a.ldv, a.dh, kv, fk.end - 1, lane, 0);
    float mx = -INFINITY;
#pragma unroll
    for (int e = 0; e < 16; e++) {
      const int j = kv + elem_row(e, half);
      float keep;
      s[e] = j >= fk.r.x && j < fk.r.y ? range_score<CAP>(s[e], a.cap, slope, at, j, &keep) : -INFINITY;
      mx = fmaxf(mx, s[e]);
    }
    mx = fmaxf(mx, __shfl_xor(mx, 32, WAVE));
    const float mn = fmaxf(m, mx), ms = mn == -INFINITY ? 0.f : mn, alpha = expf(m - ms);
    float rs = 0.f;
#pragma unroll
    for (int e = 0; e < 16; e++) { s[e] = expf(s[e] - ms); rs += s[e]; }
    l = l * alpha + rs;
    m = mn;
#pragma unroll
    for (int i = 0; i < DHP / 32; i++) acc[i] *= alpha;
    accumulate<DHP>(acc, first, v, a.ldv, a.dh, kv, fk.end - 1, s, lane);
  }
  l = half_sum(l);
  float* stats = sm + NW * DHP * 32;
  spill<DHP>(sm + wv * DHP * 32, acc, lane);
  if (half == 0) { stats[wv * 64 + lane] = m * LOG2E; stats[wv * 64 + 32 + lane] = l; }
  __syncthreads();
  few_finish<float, DHP, NW>(a, f, tile, split, head, rows, keys, sm, stats, sm);
}

// dQ of 32 rows, and D = <o, dO>; where there are few workgroups the keys are split as in the forward pass (751 rows x 4 heads of
// 64: 28 us, 19 + 4.6 split in two; 1000 x 4: all passes 116 -> 99).  The last workgroups of the launch (from `tiles` on) note instead, a wave per block of 64 queries, the first key that
// some of them see and one past the last.
template <int DHP, int NW, bool CAP> __global__ void __launch_bounds__(NW * 64, 2) range_dq_f32_k(RangeAttn a, FewShape f, int tiles, BlockSeen* __restrict__ blocks) {
  extern __shared__ float sm[];                      // Q and dO of the rows, later NW results [DHP][32]
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
  if ((int)blockIdx.x >= tiles) {
    const int b = ((int)blockIdx.x - tiles) * NW + wv;
    const BlockSeen r = block_seen(a, b, rows_in_use(a), keys_in_use(a), lane);
    if (lane == 0 && b * 64 < a.Tq) blocks[b] = r;
    return;
  }
  int tile, split, head, t0;
  few_place(a, f, (int)blockIdx.x, &tile, &split, &head);
  const int kh = head % a.Hkv;
  FewRow row = few_row(a, f, tile, head, lane & 31, a.Tq);
  const int2 stored = stored_range(a, row.i);
  const float slope = a.slopes ? a.slopes[row.h] : 0.f;
  const int at = row.ok && a.at ? a.at[row.i] : row.i;
  const float *k = (const float*)a.k + (i64)kh * a.dh, *v = (const float*)a.v + (i64)kh * a.dh;
  const i64 orow = (i64)row.i * a.ldo + (i64)row.h * a.dh, qrow = (i64)row.i * a.ldq + (i64)row.h * a.dh, srow = (i64)row.h * a.Tq + row.i;
  // the rows' operands, the same for all waves, in LDS as in the kernel below
  f32x4 *qf = (f32x4*)sm, *dof = qf + DHP / 8 * 64;
  float D = 0.f;
#pragma unroll
  for (int c = 0; c < DHP / 8; c++) {
    const int col = c * 8 + half * 4;
    f32x4 x = {0.f, 0.f, 0.f, 0.f}, y = x, z = x;
    if (row.ok && col < a.dh) {
      if (c % NW == wv) x = *(const f32x4*)((const float*)a.q + qrow + col);
      y = *(const f32x4*)((const float*)a.d_o + orow + col);
      z = *(const f32x4*)((const float*)a.o + orow + col);
    }
    if (c % NW == wv) {
      qf[c * 64 + lane] = x * a.scale;
      dof[c * 64 + lane] = y;
    }
#pragma unroll
    for (int u = 0; u < 4; u++) D = fmaf(y[u], z[u], D);
  }
  const float L = row.ok ? a.lse[srow] : -INFINITY;
  const int rows = rows_in_use(a), keys = keys_in_use(a);
  if (tile * f.qpt >= rows) return;
  row.ok = row.ok && row.i < rows;
  const FewKeys fk = few_keys(f, row, stored, split, keys, &t0);
  D = half_sum(D);
  if (split == 0 && wv == 0 && half == 0 && row.ok) a.dvec[srow] = D;
  __syncthreads();
  f32x16 acc[DHP / 32] = {};
  for (int t = fk.live_from(t0 + wv, NW); t < fk.t1; t = fk.live_from(t + NW, NW)) {
    const int kv = fk.first + t * 32, jc = min(kv + (lane & 31), fk.end - 1);
    f32x16 s, dp;
    scores2<DHP>(s, dp, k + (i64)jc * a.ldk, v + (i64)jc * a.ldv, a.dh, half, [&](int c) { return qf[c * 64 + lane]; }, [&](int c) { return dof[c * 64 + lane]; });
    Columns<DHP> first;
    first.load(k, a.ldk, a.dh, kv, fk.end - 1, lane, 0);
#pragma unroll
    for (int e = 0; e < 16; e++) {
      const int j = kv + elem_row(e, half);
      float keep;
      const float x = range_score<CAP>(s[e], a.cap, slope, at, j, &keep);
      s[e] = j >= fk.r.x && j < fk.r.y && L != -INFINITY ? expf(x - L) * (dp[e] - D) * keep : 0.f;
    }
    accumulate<DHP>(acc, first, k, a.ldk, a.dh, kv, fk.end - 1, s, lane);
  }
  __syncthreads();                                   // (the results lie where the operands were)
  spill<DHP>(sm + wv * DHP * 32, acc, lane);
  __syncthreads();
  const FewRow mine = few_row(a, f, tile, head, threadIdx.x & 31, rows);
  if (f.splits > 1) {                               // (the launch below adds them)
    (void)few_store<float, DHP, NW>(sm, f.part + (((i64)mine.i * a.H + mine.h) * f.splits + split) * DHP, mine.ok, DHP, 1.f);
    return;
  }
  const bool fine = few_store<float, DHP, NW>(sm, (float*)a.dq + (i64)mine.i * a.ldq + (i64)mine.h * a.dh, mine.ok, a.dh, a.scale);
  if (__syncthreads_or(!fine))
    for (int x = wv; x < 32; x += NW) {
      const FewRow again = few_row(a, f, tile, head, x, rows);
      if (again.ok) range_row_dq<float>(a, again.i, again.h, keys, sm + wv * 2 * DHP);
    }
}

// dQ from the splits' sums, a wave per query row and head
template <int DHP> __global__ void __launch_bounds__(256) range_dq_sum_f32_k(RangeAttn a, FewShape f) {
  __shared__ float lds[4][2 * DHP];
  constexpr int C = DHP / 64;
  const int rows = rows_in_use(a), lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const i64 n = (i64)blockIdx.x * 4 + wv;
  const int i = (int)(n / a.H), h = (int)(n - (i64)i * a.H);
  if (i >= rows) return;
  float v[C] = {}, z = 0.f;
  const float* p = f.part + n * f.splits * DHP + lane * C;
#pragma unroll 4
  for (int x = 0; x < f.splits; x++)
#pragma unroll
    for (int c = 0; c < C; c++) v[c] += p[x * DHP + c];
#pragma unroll
  for (int c = 0; c < C; c++) z = fmaf(v[c], 0.f, z);
  if (!__all(z == 0.f)) {                           // a value that is not finite: seen, or only in a tile with seen ones?
    range_row_dq<float>(a, i, h, keys_in_use(a), lds[wv]);
    return;
  }
  float* dq = (float*)a.dq + (i64)i * a.ldq + (i64)h * a.dh;
#pragma unroll
  for (int c = 0; c < C; c++) if (lane * C + c < a.dh) dq[lane * C + c] = v[c] * a.scale;
}
// dK, dV of 32 keys of a key head: the waves share out the blocks of 32 queries that see some of them, of every head that shares it.
template <int DHP, int NW, bool CAP> __global__ void __launch_bounds__(NW * 64, 2) range_dkv_f32_k(RangeAttn a, const BlockSeen* __restrict__ blocks, float* __restrict__ sums, int parts) {
  extern __shared__ float sm[];                      // K and V of the keys, later NW results [DHP][32]; then 5 x 32 words per wave
  const int per = a.Hkv * parts, kt = (int)blockIdx.x / per, r0 = (int)blockIdx.x - kt * per, kh = r0 % a.Hkv, part = r0 / a.Hkv, k0 = kt * 32;
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, myk = k0 + (lane & 31);
  float* words = sm + NW * DHP * 32 + wv * 160;
  // the keys' operands, the same for all waves: chunk c of lane l at [c][l], which costs LDS reads but the registers of two waves per SIMD
  f32x4 *kf = (f32x4*)sm, *vf = kf + DHP / 8 * 64;
#pragma unroll
  for (int c = wv; c < DHP / 8; c += NW) {
    const int col = c * 8 + half * 4;
    f32x4 x = {0.f, 0.f, 0.f, 0.f}, y = x;
    if (myk < a.Tk && col < a.dh) {
      x = *(const f32x4*)((const float*)a.k + (i64)myk * a.ldk + (i64)kh * a.dh + col);
      y = *(const f32x4*)((const float*)a.v + (i64)myk * a.ldv + (i64)kh * a.dh + col);
    }
    kf[c * 64 + lane] = x * a.scale;
    vf[c * 64 + lane] = y;
  }
  const int rows = rows_in_use(a), keys = keys_in_use(a);
  if (k0 >= keys) return;
  __syncthreads();
  f32x16 dka[DHP / 32] = {}, dva[DHP / 32] = {};
  const int nb = (rows + 63) / 64;
  int n = part * NW + wv;                            // this wave's next one of the pairs of a block, 2 G to a block
  for (int b0 = 0; b0 < nb; b0 += 64) {
    const int2 r = b0 + lane < nb ? *(const int2*)(blocks + b0 + lane) : make_int2(INT_MAX, 0);
    unsigned long long live = __ballot(r.x < k0 + 32 && r.y > k0);
    while (live) {
      const int b = b0 + __builtin_ctzll(live);
      live &= live - 1;
      for (; n < 2 * a.G; n += NW * parts) {
        const int q0 = b * 64 + (n & 1) * 32, h = kh * a.G + (n >> 1), i = q0 + (lane & 31);
        if (q0 >= rows) continue;
        const int2 see = i < rows ? key_range(a, i, keys) : make_int2(0, 0);
        if (!__any(see.x < k0 + 32 && see.y > k0)) continue;
        const int ic = min(i, rows - 1);
        wave_lds_fence();
        if (half == 0) {
          words[lane] = a.lse[(i64)h * a.Tq + ic];
          words[32 + lane] = a.dvec[(i64)h * a.Tq + ic];
          ((int*)words)[64 + lane] = a.at ? a.at[ic] : ic;
        } else {
          ((int*)words)[96 + lane - 32] = see.x;
          ((int*)words)[128 + lane - 32] = see.y;
        }
        wave_lds_fence();
        const float *q = (const float*)a.q + (i64)h * a.dh, *d_o = (const float*)a.d_o + (i64)h * a.dh;
        f32x16 s, dp;
        scores2<DHP>(s, dp, q + (i64)ic * a.ldq, d_o + (i64)ic * a.ldo, a.dh, half, [&](int c) { return kf[c * 64 + lane]; }, [&](int c) { return vf[c * 64 + lane]; });
        Columns<DHP> first;
        first.load(d_o, a.ldo, a.dh, q0, rows - 1, lane, 0);
        const float slope = a.slopes ? a.slopes[h] : 0.f;
#pragma unroll
        for (int e = 0; e < 16; e++) {
          const int x = elem_row(e, half);
          const float L = words[x];
          const bool sees = myk >= ((const int*)words)[96 + x] && myk < ((const int*)words)[128 + x] && L != -INFINITY;
          float keep;
          const float p = expf(range_score<CAP>(s[e], a.cap, slope, ((const int*)words)[64 + x], myk, &keep) - L);
          dp[e] = sees ? p * (dp[e] - words[32 + x]) * keep : 0.f;
          s[e] = sees ? p : 0.f;
        }
        accumulate<DHP>(dva, first, d_o, a.ldo, a.dh, q0, rows - 1, s, lane);
        first.load(q, a.ldq, a.dh, q0, rows - 1, lane, 0);
        accumulate<DHP>(dka, first, q, a.ldq, a.dh, q0, rows - 1, dp, lane);
      }
      n -= 2 * a.G;
    }
  }
  __syncthreads();                                   // (the results lie where the keys were)
  const int r = k0 + (int)(threadIdx.x & 31);
  if (parts > 1) {
    float* row = sums + ((((i64)part * 2) * a.Tk + r) * a.Hkv + kh) * DHP;
    spill<DHP>(sm + wv * DHP * 32, dka, lane);
    __syncthreads();
    (void)few_store<float, DHP, NW>(sm, row, r < keys, DHP, 1.f);
    __syncthreads();
    spill<DHP>(sm + wv * DHP * 32, dva, lane);
    __syncthreads();
    (void)few_store<float, DHP, NW>(sm, row + (i64)a.Tk * a.Hkv * DHP, r < keys, DHP, 1.f);
    return;
  }
  spill<DHP>(sm + wv * DHP * 32, dka, lane);
  __syncthreads();
  bool fine = few_store<float, DHP, NW>(sm, (float*)a.dk + (i64)r * a.ldk + (i64)kh * a.dh, r < keys, a.dh, a.scale);
  __syncthreads();
  spill<DHP>(sm + wv * DHP * 32, dva, lane);
  __syncthreads();
  fine &= few_store<float, DHP, NW>(sm, (float*)a.dv + (i64)r * a.ldv + (i64)kh * a.dh, r < keys, a.dh, 1.f);
  if (__syncthreads_or(!fine))
    for (int x = wv; x < 32 && k0 + x < keys; x += NW) range_row_dkv<float>(a, k0 + x, kh, rows, keys, sm + wv * 2 * DHP);
}

// rows are read 4 elements at a time
bool range_f32_takes(const RangeAttn& a, bool back) {
  if (a.dt != 0 || a.dh > 128 || a.dh % 4) return false;
  uintptr_t p = (uintptr_t)a.q | (uintptr_t)a.k | (uintptr_t)a.v;
  p |= back ? (uintptr_t)a.o | (uintptr_t)a.d_o | (uintptr_t)a.dq | (uintptr_t)a.dk | (uintptr_t)a.dv : (uintptr_t)a.out;
  return !(p & 15) && !((a.ldq | a.ldk | a.ldv | a.ldo) & 3);
}
template <class K> static void set_lds(std::atomic<unsigned long long>& mask, K kernel, size_t bytes) {
  if (attr_needed(mask)) {
    (void)hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    attr_done(mask);
  }
}
template <int DHP, int NW, bool CAP> static void fwd(const RangeAttn& a, float* work, hipStream_t s) {
  constexpr size_t smem = (size_t)(NW * DHP * 32 + NW * 64) * 4;
  static std::atomic<unsigned long long> mask{0};
  set_lds(mask, range_fwd_f32_k<DHP, NW, CAP>, smem);
  const FewShape f = few_shape(a, work);
  hipLaunchKernelGGL((range_fwd_f32_k<DHP, NW, CAP>), dim3((unsigned)((i64)f.tiles * f.splits * a.Hkv * f.hb)), dim3(NW * 64), smem, s, a, f);
  join_splits<float, DHP>(a, f, s);
}
// dK/dV: the pairs of a block of 32 queries and a head in parts, where the workgroups leave CUs idle
static int dkv_parts(const RangeAttn& a) {
  const i64 workgroups = (i64)cdiv(a.Tk, 32) * a.Hkv, pairs = (i64)cdiv(a.Tq, 32) * a.G;
  const int waves = few_waves(a);
  int n = 1;
  while (n < 8 && workgroups * n * 2 * waves <= 2048 && pairs >= 2 * n * waves) n *= 2;
  return n;
}
// the sums of dQ's splits or of dK's and dV's parts, one after the other in the same memory
size_t range_f32_sum_floats(const RangeAttn& a) {
  const int n = dkv_parts(a);
  const size_t kv = n > 1 ? (size_t)n * 2 * a.Tk * a.Hkv * (a.dh <= 64 ? 64 : 128) : 0, q = few_floats(a);
  return kv > q ? kv : q;
}
template <int DHP, int NW, bool CAP> static void bwd(const RangeAttn& a, void* blocks, float* sums, hipStream_t s) {
  constexpr size_t smem = (size_t)NW * DHP * 32 * 4, smem_kv = smem + NW * 160 * 4;
  static std::atomic<unsigned long long> mask_q{0}, mask_kv{0};
  set_lds(mask_q, range_dq_f32_k<DHP, NW, CAP>, smem);
  set_lds(mask_kv, range_dkv_f32_k<DHP, NW, CAP>, smem_kv);
  FewShape f = few_shape(a, nullptr);
  f.part = sums;
  const int tiles = f.tiles * f.splits * a.Hkv * f.hb;
  if (a.Tq > 0)
    hipLaunchKernelGGL((range_dq_f32_k<DHP, NW, CAP>), dim3((unsigned)(tiles + cdiv(a.Tq, 64 * NW))), dim3(NW * 64), smem, s, a, f, tiles, (BlockSeen*)blocks);
  if (f.splits > 1) hipLaunchKernelGGL((range_dq_sum_f32_k<DHP>), dim3((unsigned)cdiv((i64)a.Tq * a.H, 4)), dim3(256), 0, s, a, f);
  if (a.Tk <= 0) return;
  const int parts = dkv_parts(a);
  hipLaunchKernelGGL((range_dkv_f32_k<DHP, NW, CAP>), dim3((unsigned)((i64)cdiv(a.Tk, 32) * a.Hkv * parts)), dim3(NW * 64), smem_kv, s, a,
                     (const BlockSeen*)blocks, sums, parts);
  sum_parts<float, DHP>(a, sums, parts, s);
}
#define BY_FORM(call)                                                  \
  do {                                                                 \
    if (a.dh <= 64 && few_waves(a) == 8) { if (a.cap > 0.f) call(64, 8, true); else call(64, 8, false); } \
    else if (a.dh <= 64) { if (a.cap > 0.f) call(64, 4, true); else call(64, 4, false); } \
    else if (a.cap > 0.f) call(128, 4, true);                          \
    else call(128, 4, false);                                          \
  } while (0)
void launch_range_fwd_f32(const RangeAttn& a, float* work, hipStream_t s) {
  if (a.Tq <= 0) return;
#define FWD(D, W, C) fwd<D, W, C>(a, work, s)
  BY_FORM(FWD);
}
void launch_range_bwd_f32(const RangeAttn& a, void* blocks, float* sums, hipStream_t s) {
#define BWD(D, W, C) bwd<D, W, C>(a, blocks, sums, s)
  BY_FORM(BWD);
}
