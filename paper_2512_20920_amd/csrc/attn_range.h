// Shared pieces of the kernels for attention over key ranges: which keys a query sees, scores, and the row-by-row forms of
// the three passes, in which one wave works on one result row and touches only what that row sees.
#pragma once
#include "kernels.h"

#define LOG2E 1.4426950408889634f
#define LN2 0.6931471805599453f
#define RANGE_MAX_DH 512

// ---- integers over the 64 lanes, as the sums and maxima of floats ----
template <int CTRL, int ROW_MASK> __device__ __forceinline__ int dpp_i(int keep, int v) { return __builtin_amdgcn_update_dpp(keep, v, CTRL, ROW_MASK, 0xf, false); }
__device__ __forceinline__ int wave_imax(int v) {
  v = max(v, dpp_i<0x111, 0xf>(v, v));
  v = max(v, dpp_i<0x112, 0xf>(v, v));
  v = max(v, dpp_i<0x114, 0xf>(v, v));
  v = max(v, dpp_i<0x118, 0xf>(v, v));
  v = max(v, dpp_i<0x142, 0xa>(v, v));
  v = max(v, dpp_i<0x143, 0xc>(v, v));
  return __builtin_amdgcn_readlane(v, 63);
}
__device__ __forceinline__ int wave_imin(int v) { return -1 - wave_imax(-1 - v); }

__device__ __forceinline__ int rows_in_use(const RangeAttn& a) { return a.used ? min(max(a.used[0], 0), a.Tq) : a.Tq; }
__device__ __forceinline__ int keys_in_use(const RangeAttn& a) { return a.used ? min(max(a.used[1], 0), a.Tk) : a.Tk; }
// clamped; lo = hi = 0 if there is none
__device__ __forceinline__ int2 clamped(int2 r, int keys) {
  r = make_int2(max(r.x, 0), min(r.y, keys));
  if (r.x >= r.y) r.x = r.y = 0;
  return r;
}
// A workgroup's first loads wait for nothing: ranges (and queries) are read by clamped row number while the rows and keys in use
// are on their way too.
__device__ __forceinline__ int2 stored_range(const RangeAttn& a, int i) { i = min(i, a.Tq - 1); return make_int2(a.lo[i], a.hi[i]); }
__device__ __forceinline__ int2 key_range(const RangeAttn& a, int i, int keys) { return clamped(make_int2(a.lo[i], a.hi[i]), keys); }
// the score from z = scale q.k, and what a gradient at the score is multiplied by to be one at z
template <bool CAPPED = true> __device__ __forceinline__ float range_score(float z, float cap, float slope, int at, int j, float* keep) {
  *keep = 1.f;
  if (CAPPED && cap > 0.f) {
    const float t = tanhf(z / cap);
    z = t * cap;
    *keep = 1.f - t * t;
  }
  return slope != 0.f ? z - slope * fabsf((float)(at - j)) : z;
}

// Values of one wave that its other lanes read back: the LDS accesses of a wave are in order, the compiler's need this.
__device__ __forceinline__ void wave_lds_fence() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
template <class T> __device__ __forceinline__ float row_dot(const T* row, const float* other, int dh) {
  float s0 = 0.f, s1 = 0.f;
  int c = 0;
  for (; c + 1 < dh; c += 2) { s0 = fmaf(to_f(row[c]), other[c], s0); s1 = fmaf(to_f(row[c + 1]), other[c + 1], s1); }
  if (c < dh) s0 = fmaf(to_f(row[c]), other[c], s0);
  return s0 + s1;
}
// acc[u] += w(lane n) * row n of x for the lanes in `live`; columns lane + 64 u
template <class T> __device__ __forceinline__ void add_rows(float (&acc)[RANGE_MAX_DH / 64], const T* x, i64 ld, float w, unsigned long long live, int dh, int lane) {
  while (live) {
    const int n = __builtin_ctzll(live);
    live &= live - 1;
    const float f = __shfl(w, n, WAVE);
    const T* row = x + (i64)n * ld;
#pragma unroll
    for (int u = 0; u < RANGE_MAX_DH / 64; u++) if (lane + 64 * u < dh) acc[u] = fmaf(f, to_f(row[lane + 64 * u]), acc[u]);
  }
}

// lds: 2 dh floats of this wave's own.  A wave's lanes take 64 keys (queries) at a time for the products over the head width, then
// the columns of the result.
template <class T> __device__ void range_row_fwd(const RangeAttn& a, int i, int h, int keys, float* lds) {
  const int lane = threadIdx.x & 63, dh = a.dh, kh = h / a.G;
  const int2 r = key_range(a, i, keys);
  const T* q = (const T*)a.q + (i64)i * a.ldq + (i64)h * dh;
  const T* k = (const T*)a.k + (i64)kh * dh;
  const T* v = (const T*)a.v + (i64)kh * dh;
  wave_lds_fence();
  for (int c = lane; c < dh; c += 64) lds[c] = to_f(q[c]);
  wave_lds_fence();
  const float slope = a.slopes ? a.slopes[h] : 0.f;
  const int at = a.at ? a.at[i] : i;
  float acc[RANGE_MAX_DH / 64] = {}, m = -INFINITY, l = 0.f;
  for (int j0 = r.x; j0 < r.y; j0 += 64) {
    const int j = j0 + lane;
    const bool sees = j < r.y;
    float s = -INFINITY, keep;
    if (sees) s = range_score(row_dot(k + (i64)j * a.ldk, lds, dh) * a.scale, a.cap, slope, at, j, &keep);
    const float mn = fmaxf(m, wave_max(s)), ms = mn == -INFINITY ? 0.f : mn;
    const float p = sees ? expf(s - ms) : 0.f, alpha = expf(m - ms);
    l = l * alpha + wave_sum(p);
#pragma unroll
    for (int u = 0; u < RANGE_MAX_DH / 64; u++) acc[u] *= alpha;
    m = mn;
    add_rows(acc, v + (i64)j0 * a.ldv, a.ldv, p, __ballot(sees), dh, lane);
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  T* o = (T*)a.out + (i64)i * a.ldo + (i64)h * dh;
#pragma unroll
  for (int u = 0; u < RANGE_MAX_DH / 64; u++) if (lane + 64 * u < dh) o[lane + 64 * u] = from_f<T>(acc[u] * inv);
  if (lane == 0 && a.lse) a.lse[(i64)h * a.Tq + i] = l == 0.f ? -INFINITY : m + logf(l);
}

// dq of a row, and D = <o, d_o>
template <class T> __device__ void range_row_dq(const RangeAttn& a, int i, int h, int keys, float* lds) {
  const int lane = threadIdx.x & 63, dh = a.dh, kh = h / a.G;
  const int2 r = key_range(a, i, keys);
  const i64 qrow = (i64)i * a.ldq + (i64)h * dh, orow = (i64)i * a.ldo + (i64)h * dh;
  const T* k = (const T*)a.k + (i64)kh * dh;
  const T* v = (const T*)a.v + (i64)kh * dh;
  float* dos = lds + dh;
  float D = 0.f;
  wave_lds_fence();
  for (int c = lane; c < dh; c += 64) {
    lds[c] = to_f(((const T*)a.q)[qrow + c]);
    const float d = to_f(((const T*)a.d_o)[orow + c]);
    dos[c] = d;
    D = fmaf(d, to_f(((const T*)a.o)[orow + c]), D);
  }
  wave_lds_fence();
  D = wave_sum(D);
  if (lane == 0) a.dvec[(i64)h * a.Tq + i] = D;
  const float slope = a.slopes ? a.slopes[h] : 0.f, L = a.lse[(i64)h * a.Tq + i];
  const int at = a.at ? a.at[i] : i;
  float acc[RANGE_MAX_DH / 64] = {};
  if (L != -INFINITY)
    for (int j0 = r.x; j0 < r.y; j0 += 64) {
      const int j = j0 + lane;
      const bool sees = j < r.y;
      float ds = 0.f;
      if (sees) {
        float keep;
        const float s = range_score(row_dot(k + (i64)j * a.ldk, lds, dh) * a.scale, a.cap, slope, at, j, &keep);
        ds = expf(s - L) * (row_dot(v + (i64)j * a.ldv, dos, dh) - D) * keep;
      }
      add_rows(acc, k + (i64)j0 * a.ldk, a.ldk, ds, __ballot(sees), dh, lane);
    }
  T* dq = (T*)a.dq + qrow;
#pragma unroll
  for (int u = 0; u < RANGE_MAX_DH / 64; u++) if (lane + 64 * u < dh) dq[lane + 64 * u] = from_f<T>(acc[u] * a.scale);
}

// dk and dv of a key row, over the query heads that share it
template <class T> __device__ void range_row_dkv(const RangeAttn& a, int j, int kh, int rows, int keys, float* lds) {
  const int lane = threadIdx.x & 63, dh = a.dh;
  float* vs = lds + dh;
  const i64 krow = (i64)j * a.ldk + (i64)kh * dh, vrow = (i64)j * a.ldv + (i64)kh * dh;
  wave_lds_fence();
  for (int c = lane; c < dh; c += 64) { lds[c] = to_f(((const T*)a.k)[krow + c]); vs[c] = to_f(((const T*)a.v)[vrow + c]); }
  wave_lds_fence();
  float dka[RANGE_MAX_DH / 64] = {}, dva[RANGE_MAX_DH / 64] = {};
  for (int i0 = 0; i0 < rows; i0 += 64) {
    const int i = i0 + lane;
    const int2 r = i < rows ? key_range(a, i, keys) : make_int2(0, 0);
    const bool in = r.x <= j && j < r.y;
    if (!__any(in)) continue;
    for (int h = kh * a.G; h < (kh + 1) * a.G; h++) {
      const T* q = (const T*)a.q + (i64)i0 * a.ldq + (i64)h * dh;
      const T* d_o = (const T*)a.d_o + (i64)i0 * a.ldo + (i64)h * dh;
      float p = 0.f, ds = 0.f;
      const float L = in ? a.lse[(i64)h * a.Tq + i] : -INFINITY;
      const bool sees = in && L != -INFINITY;
      if (sees) {
        float keep;
        const float s = range_score(row_dot(q + (i64)lane * a.ldq, lds, dh) * a.scale, a.cap, a.slopes ? a.slopes[h] : 0.f, a.at ? a.at[i] : i, j, &keep);
        p = expf(s - L);
        ds = p * (row_dot(d_o + (i64)lane * a.ldo, vs, dh) - a.dvec[(i64)h * a.Tq + i]) * keep;
      }
      const unsigned long long live = __ballot(sees);
      add_rows(dva, d_o, a.ldo, p, live, dh, lane);
      add_rows(dka, q, a.ldq, ds, live, dh, lane);
    }
  }
  T *dk = (T*)a.dk + krow, *dv = (T*)a.dv + vrow;
#pragma unroll
  for (int u = 0; u < RANGE_MAX_DH / 64; u++)
    if (lane + 64 * u < dh) {
      dk[lane + 64 * u] = from_f<T>(dka[u] * a.scale);
      dv[lane + 64 * u] = from_f<T>(dva[u]);
    }
}
