// The forms of attention over key ranges for few rows: a workgroup takes 32 rows, which are queries of all (at most 32) heads that share
// a key head, so that its keys are read once for all of them, and its four or eight waves (few_waves) share the keys out in tiles of 32.  The keys may
// be split further over several workgroups, whose results a second launch joins.
#pragma once
#include "attn_range.h"

struct FewShape {
  int gp, hb;              // heads of a workgroup, head blocks per key head (more than one: more than 32 heads to a key head)
  int inv;                 // r / gp = r inv >> 16 for r < 32
  int qpt, tiles;          // queries of a workgroup, tiles of them
  int splits;              // of the keys
  float2* stats;           // splits > 1: [query row, head][split] maximum (units of log2) and sum
  float* part;             //             [query row, head][split][DHP] unnormalised result
};
struct FewRow { int i, h; bool ok; };
__device__ __forceinline__ FewRow few_row(const RangeAttn& a, const FewShape& f, int tile, int head, int r, int rows) {
  const int kh = head % a.Hkv, hb = head / a.Hkv, q = r * f.inv >> 16, hg = hb * f.gp + r - q * f.gp;
  FewRow x;
  x.i = tile * f.qpt + q;
  x.ok = q < f.qpt && hg < a.G && x.i < rows;
  x.h = kh * a.G + min(hg, a.G - 1);
  return x;
}
// workgroup id -> tile, split, head block (fastest: consecutive workgroups go to different XCDs, a key head stays with one)
__device__ __forceinline__ void few_place(const RangeAttn& a, const FewShape& f, int id, int* tile, int* split, int* head) {
  const int heads = a.Hkv * f.hb, row = id / heads;
  *head = id - row * heads;
  *tile = row / f.splits;
  *split = row - *tile * f.splits;
  *tile = f.tiles - 1 - *tile;                       // late queries tend to have the long ranges
}
// the keys that the 32 rows see, in tiles of 32 from the first one on
struct FewKeys {
  int2 r;                  // of this lane's row (lane & 31); lo = INT_MAX, hi = 0: none
  int first, end, t1;      // t1: one past this workgroup's last tile
  // the first tile from t on, in steps of `step`, that some row sees; t1 or more: there is none
  __device__ __forceinline__ int live_from(int t, int step) const {
    while (t < t1) {
      const int kv = first + t * 32;
      if (__any(r.x < kv + 32 && r.y > kv)) return t;
      const int v = wave_imin(r.y > kv ? r.x : INT_MAX);      // the next key that anybody sees
      if (v == INT_MAX) return t1;
      t += max(1, ((v - first) / 32 - t + step - 1) / step) * step;
    }
    return t;
  }
};
__device__ __forceinline__ FewKeys few_keys(const FewShape& f, const FewRow& row, int2 stored, int split, int keys, int* t0) {
  FewKeys k;
  k.r = row.ok ? clamped(stored, keys) : make_int2(0, 0);
  if (k.r.x == k.r.y) k.r = make_int2(INT_MAX, 0);
  k.first = wave_imin(k.r.x);
  k.end = wave_imax(k.r.y);
  const int n = k.first < k.end ? (k.end - k.first + 31) / 32 : 0, per = (n + f.splits - 1) / f.splits;
  *t0 = min(split * per, n);
  k.t1 = min(*t0 + per, n);
  return k;
}

// The waves' partial results, [column][32 rows] in LDS each, with their maxima (units of log2) and sums, to the row's result or to this split's
// part of it.  slow: 2 dh floats of LDS per wave for rows that are worked out again.
template <class T, int DHP, int NW>
__device__ __forceinline__ void few_finish(const RangeAttn& a, const FewShape& f, int tile, int split, int head, int rows, int keys,
                                           const float* part, const float* stats, float* slow) {
  constexpr int C = DHP * 32 / (NW * 64);            // columns per thread
  const int r = threadIdx.x & 31, c0 = (int)(threadIdx.x >> 5) * C;
  const FewRow row = few_row(a, f, tile, head, r, rows);
  float M = -INFINITY, w[NW], tot = 0.f, v[C];
#pragma unroll
  for (int j = 0; j < NW; j++) M = fmaxf(M, stats[j * 64 + r]);
  const float Ms = M == -INFINITY ? 0.f : M;
#pragma unroll
  for (int j = 0; j < NW; j++) { w[j] = exp2f(stats[j * 64 + r] - Ms); tot += w[j] * stats[j * 64 + 32 + r]; }
#pragma unroll
  for (int c = 0; c < C; c++) {
    v[c] = 0.f;
#pragma unroll
    for (int j = 0; j < NW; j++) v[c] = fmaf(w[j], part[(j * DHP + c0 + c) * 32 + r], v[c]);
  }
  if (f.splits > 1) {
    if (!row.ok) return;
    const i64 at = ((i64)row.i * a.H + row.h) * f.splits + split;
    if (threadIdx.x < 32) f.stats[at] = make_float2(M, tot);
    if (tot == 0.f) return;                          // (nothing seen: the second launch leaves it out)
#pragma unroll
    for (int c = 0; c < C; c += 4) *(float4*)(f.part + at * DHP + c0 + c) = make_float4(v[c], v[c + 1], v[c + 2], v[c + 3]);
    return;
  }
  const float inv = tot == 0.f ? 0.f : 1.f / tot;
  float z = 0.f;
  T* o = (T*)a.out + (i64)row.i * a.ldo + (i64)row.h * a.dh;
#pragma unroll
  for (int c = 0; c < C; c += 4) {
    typedef __attribute__((ext_vector_type(4))) T V4;
    V4 x;
#pragma unroll
    for (int i = 0; i < 4; i++) { z = fmaf(v[c + i], 0.f, z); x[i] = from_f<T>(v[c + i] * inv); }
    if (row.ok && c0 + c < a.dh) *(V4*)(o + c0 + c) = x;
  }
  if (threadIdx.x < 32 && row.ok && a.lse) a.lse[(i64)row.h * a.Tq + row.i] = tot == 0.f ? -INFINITY : (M + log2f(tot)) * LN2;
  // a value that is not finite: seen by its row, or only multiplied by zero in a tile that it sees a part of?
  if (__syncthreads_or(row.ok && z != 0.f))
    for (int x = (int)(threadIdx.x >> 6); x < 32; x += NW) {
      const FewRow again = few_row(a, f, tile, head, x, rows);
      if (again.ok) range_row_fwd<T>(a, again.i, again.h, keys, slow + (threadIdx.x >> 6) * 2 * DHP);
    }
}
// The sum of the waves' partial results, [column][32 rows] in LDS each, times f, to row threadIdx.x & 31; whether all of it is finite
template <class T, int DHP, int NW> __device__ __forceinline__ bool few_store(const float* part, T* row, bool ok, int dh, float f) {
  constexpr int C = DHP * 32 / (NW * 64);
  typedef __attribute__((ext_vector_type(4))) T V4;
  const int r = threadIdx.x & 31, c0 = (int)(threadIdx.x >> 5) * C;
  float z = 0.f;
#pragma unroll
  for (int c = 0; c < C; c += 4) {
    V4 v;
#pragma unroll
    for (int i = 0; i < 4; i++) {
      float t = 0.f;
#pragma unroll
      for (int w = 0; w < NW; w++) t += part[(w * DHP + c0 + c + i) * 32 + r];
      z = fmaf(t, 0.f, z);
      v[i] = from_f<T>(t * f);
    }
    if (ok && c0 + c < dh) *(V4*)(row + c0 + c) = v;
  }
  return !ok || z == 0.f;
}
// block of 64 queries: the first key that some of them see and one past the last (none: INT_MAX, 0), and between which keys all 64
// see (one that is not there sees nothing)
typedef int4 BlockSeen;
__device__ __forceinline__ BlockSeen block_seen(const RangeAttn& a, int b, int rows, int keys, int lane) {
  const int i = b * 64 + lane;
  const int2 r = i < rows ? key_range(a, i, keys) : make_int2(0, 0);
  const bool sees = r.x < r.y;
  return make_int4(wave_imin(sees ? r.x : INT_MAX), wave_imax(r.y), wave_imax(sees ? r.x : INT_MAX), wave_imin(r.y));
}
// Joins the splits of a (query row, head), W waves each a share of them (16 at most), all their loads in flight at once; DHP / 64
// columns per lane.  (One wave for all, eight splits in flight: 64 splits of 160 rows 10.8 us, 4.8 like this.)
template <class T, int DHP, int W> __global__ void __launch_bounds__(256) range_join_k(RangeAttn a, FewShape f) {
  __shared__ float sums[4][DHP], slow[4][2 * DHP];
  constexpr int C = DHP / 64;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wv = W == 4 ? wave : 0, rows = rows_in_use(a);
  const i64 n = W == 4 ? (i64)blockIdx.x : (i64)blockIdx.x * 4 + wave;
  const int i = (int)(n / a.H), h = (int)(n - (i64)i * a.H);
  if (i >= rows) return;                             // (W = 4: all waves, W = 1: no barrier)
  const float2 st = lane < f.splits ? f.stats[n * f.splits + lane] : make_float2(-INFINITY, 0.f);
  const unsigned long long live = __ballot(st.y != 0.f);
  const float* p = f.part + n * f.splits * DHP + lane * C;
  float x[16][C];
#pragma unroll
  for (int k = 0; k < 16; k++) {
    const int s = k * W + wv;
#pragma unroll
    for (int c = 0; c < C; c++) x[k][c] = (live >> s) & 1 ? p[s * DHP + c] : 0.f;
  }
  const float M = wave_max(st.x), Ms = M == -INFINITY ? 0.f : M;
  const float w = st.y == 0.f ? 0.f : exp2f(st.x - Ms);
  const float tot = wave_sum(w * st.y);
  float v[C] = {};
#pragma unroll
  for (int k = 0; k < 16; k++) {
    const float ws = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w), k * W + wv));
#pragma unroll
    for (int c = 0; c < C; c++) v[c] = fmaf(ws, x[k][c], v[c]);
  }
  if constexpr (W == 4) {
#pragma unroll
    for (int c = 0; c < C; c++) sums[wv][lane * C + c] = v[c];
    __syncthreads();
    if (wv) return;
#pragma unroll
    for (int c = 0; c < C; c++) {
      const int k = lane * C + c;
      v[c] = (sums[0][k] + sums[1][k]) + (sums[2][k] + sums[3][k]);
    }
  }
  float z = 0.f;
#pragma unroll
  for (int c = 0; c < C; c++) z = fmaf(v[c], 0.f, z);
  if (!__all(z == 0.f)) {
    range_row_fwd<T>(a, i, h, keys_in_use(a), slow[wave]);
    return;
  }
  const float inv = tot == 0.f ? 0.f : 1.f / tot;
  T* o = (T*)a.out + (i64)i * a.ldo + (i64)h * a.dh;
#pragma unroll
  for (int c = 0; c < C; c++) if (lane * C + c < a.dh) o[lane * C + c] = from_f<T>(v[c] * inv);
  if (lane == 0 && a.lse) a.lse[(i64)h * a.Tq + i] = tot == 0.f ? -INFINITY : (M + log2f(tot)) * LN2;
}
template <class T, int DHP> static void join_splits(const RangeAttn& a, const FewShape& f, hipStream_t s) {
  const i64 n = (i64)a.Tq * a.H;
  if (f.splits > 16) hipLaunchKernelGGL((range_join_k<T, DHP, 4>), dim3((unsigned)n), dim3(256), 0, s, a, f);
  else if (f.splits > 1) hipLaunchKernelGGL((range_join_k<T, DHP, 1>), dim3((unsigned)cdiv(n, 4)), dim3(256), 0, s, a, f);
}

// dK and dV from the parts' sums, [part][dk, dv][key row, head][DHP]: one wave per key row and head, DHP / 64 columns per lane
template <class T, int DHP> __global__ void __launch_bounds__(256) range_dkv_sum_k(RangeAttn a, const float* __restrict__ sums, int parts) {
  __shared__ float lds[4][2 * DHP];
  constexpr int C = DHP / 64;
  const int rows = rows_in_use(a), keys = keys_in_use(a), lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const i64 n = (i64)blockIdx.x * 4 + wv;
  const int j = (int)(n / a.Hkv), kh = (int)(n - (i64)j * a.Hkv);
  if (j >= keys) return;
  float k[C] = {}, v[C] = {};
  const i64 half = (i64)a.Tk * a.Hkv * DHP;
  const float* p = sums + n * DHP + lane * C;
#pragma unroll 4
  for (int i = 0; i < parts; i++)
#pragma unroll
    for (int c = 0; c < C; c++) { k[c] += p[(i64)i * 2 * half + c]; v[c] += p[(i64)i * 2 * half + half + c]; }
  float z = 0.f;
#pragma unroll
  for (int c = 0; c < C; c++) z = __builtin_fmaf(k[c], 0.f, __builtin_fmaf(v[c], 0.f, z));
  if (!__all(z == 0.f)) {                           // a value that is not finite: seen, or only in a tile with seen ones?
    range_row_dkv<T>(a, j, kh, rows, keys, lds[wv]);
    return;
  }
  T *dk = (T*)a.dk + (i64)j * a.ldk + (i64)kh * a.dh, *dv = (T*)a.dv + (i64)j * a.ldv + (i64)kh * a.dh;
#pragma unroll
  for (int c = 0; c < C; c++)
    if (lane * C + c < a.dh) { dk[lane * C + c] = from_f<T>(k[c] * a.scale); dv[lane * C + c] = from_f<T>(v[c]); }
}

template <class T, int DHP> static void sum_parts(const RangeAttn& a, const float* sums, int parts, hipStream_t s) {
  if (parts > 1) hipLaunchKernelGGL((range_dkv_sum_k<T, DHP>), dim3((unsigned)cdiv((i64)a.Tk * a.Hkv, 4)), dim3(256), 0, s, a, sums, parts);
}

// Waves of a workgroup: four; eight in float32 with heads of 64, whose registers allow it, unless even the splits of the keys leave half of
// the CUs without a workgroup: then the work had better go to more CUs' matrix pipes.  Training step of float32, four -> eight, us: 250 rows x 4
// heads (32 workgroups) 47 -> 56, 400 x 4 (52, in two) 57 -> 70, 751 x 4 (94, in two) 67 -> 64, 1000 x 4 (126, in two) 87 -> 97, 1500 x 8 281 -> 201,
// 4000 x 4 752 -> 537; five single tokens against 16500 keys 20.8 -> 19.3.
inline i64 few_splits(const RangeAttn& a, i64 workgroups, int waves) {
  const i64 most = cdiv(a.Tk, 32 * waves), n = workgroups ? 2048 / waves / workgroups : 1;
  return n < most ? (n < 64 ? n : 64) : (most < 64 ? most : 64);
}
inline i64 few_workgroups(const RangeAttn& a) {
  const int gp = a.G < 32 ? a.G : 32;
  return (i64)cdiv(a.Tq, 32 / gp) * a.Hkv * cdiv(a.G, gp);
}
inline int few_waves(const RangeAttn& a) {
  if (a.dt != 0 || a.dh > 64) return 4;
  const i64 workgroups = few_workgroups(a), n = few_splits(a, workgroups, 8);
  return workgroups * (n < 1 ? 1 : n) < 128 ? 4 : 8;
}
// Workgroups that give every CU eight waves, of a tile of keys per wave at least.  A second launch costs 4 us and more, so few splits
// don't pay in bfloat16: 600 rows x 12 heads of 128 whole 13.2 us, in two 15.9 + 5.7; 1000 x 8 of 64 10.6, 11 + 4.9.  Float32, whose products take
// eight times as long: 751 x 4 of 64 whole 19.4, in two 13.4 + 4.1.
inline FewShape few_shape(const RangeAttn& a, float* work) {
  const int waves = few_waves(a);
  FewShape f;
  f.gp = a.G < 32 ? a.G : 32;
  f.hb = cdiv(a.G, f.gp);
  f.qpt = 32 / f.gp;
  f.inv = (65536 + f.gp - 1) / f.gp;
  f.tiles = cdiv(a.Tq, f.qpt);
  const i64 n = few_splits(a, few_workgroups(a), waves);
  f.splits = n < (a.dt == 0 ? 2 : 4) ? 1 : (int)n;
  f.stats = (float2*)work;
  f.part = work ? work + 2 * (i64)a.Tq * a.H * f.splits : nullptr;
  if ((2 * (i64)a.Tq * a.H * f.splits) % 4) f.part += 2;     // (16-byte aligned)
  return f;
}
inline size_t few_floats(const RangeAttn& a) {
  const FewShape f = few_shape(a, nullptr);
  return f.splits > 1 ? (size_t)a.Tq * a.H * f.splits * (2 + (a.dh <= 64 ? 64 : 128)) + 2 : 0;
}
