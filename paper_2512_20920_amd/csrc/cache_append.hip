// New keys and values into the pages of a cache, keys and queries turned to their positions on the way.
//
// A workgroup takes the new rows of one page (a sequence's pages one after the other: find_item) and a head's or two's keys or values (several heads at a
// time where a page's rows of one are too few): it reads them once, into registers, and writes them once, the largest of all of a head's in between, from
// the waves' maxima in LDS.  Bound by memory for long prompts (8192 rows of 32 heads and 8 key heads of 128: 46.5 us, 4.0 TB/s), by the chain of lists, loads and
// maximum for next tokens (6 us).  Other workgroups take four or eight rows' queries, which nothing but the launch has in common with these.
//
// Keys are turned in float64: sines, cosines and products, so that a key differs from the exact one by its rounding alone.  In float32 one
// in some 10^6 keys ends up on the other side of a border between two 8-bit numbers, half a step of 2^-4 of its value.  It costs no more: the series below
// are 15 multiply-adds, and the vector units do those at the rate of float32.
#include "cache.h"

// cosine and sine of a part of a turn, both within 3e-14: the nearest quarter is taken off, and the series summed for what is left, at most pi / 4
__device__ __forceinline__ double2 turn_of(double turns) {
  turns -= rint(turns);
  const double quarter = rint(4.0 * turns), x = (turns - 0.25 * quarter) * 6.283185307179586, u = x * x;
  double s = fma(u, 1.0 / 6227020800.0, -1.0 / 39916800.0), c = fma(u, -1.0 / 87178291200.0, 1.0 / 479001600.0);
  s = fma(u, s, 1.0 / 362880.0);   c = fma(u, c, -1.0 / 3628800.0);
  s = fma(u, s, -1.0 / 5040.0);    c = fma(u, c, 1.0 / 40320.0);
  s = fma(u, s, 1.0 / 120.0);      c = fma(u, c, -1.0 / 720.0);
  s = fma(u, s, -1.0 / 6.0);       c = fma(u, c, 1.0 / 24.0);
  s = fma(u * x, s, x);            c = fma(u, c, -0.5);
  c = fma(u, c, 1.0);
  const int q = (int)quarter & 3;
  const double a = q & 1 ? s : c, b = q & 1 ? c : s;
  return make_double2(q == 1 || q == 2 ? -a : a, q >= 2 ? -b : b);
}

// Eight columns of a row as they lie (WIDE: 16 bytes at a time), and as numbers
template <class T> struct Raw8 { __attribute__((ext_vector_type(8))) T v; };
template <class T, bool WIDE> __device__ __forceinline__ Raw8<T> load8(const T* p) {
  Raw8<T> r;
  if constexpr (WIDE && sizeof(T) == 2) r.v = *(const decltype(r.v)*)p;
  else if constexpr (WIDE) {
    const float4 u = *(const float4*)p, w = *(const float4*)(p + 4);
    r.v[0] = u.x; r.v[1] = u.y; r.v[2] = u.z; r.v[3] = u.w; r.v[4] = w.x; r.v[5] = w.y; r.v[6] = w.z; r.v[7] = w.w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++) r.v[i] = p[i];
  }
  return r;
}
template <class T, bool WIDE> __device__ __forceinline__ void store8(T* p, const float* x) {
  if constexpr (WIDE && sizeof(T) == 2) {
    typedef __attribute__((ext_vector_type(8))) T V;
    V v;
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = from_f<T>(x[i]);
    *(V*)p = v;
  } else if constexpr (WIDE) {
    *(float4*)p = make_float4(x[0], x[1], x[2], x[3]);
    *(float4*)(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++) p[i] = from_f<T>(x[i]);
  }
}
// The least power of two by which values up to m lie within 448 = 1.75 * 2^8, between 2^-96 and 2^119 (beyond, 448 units are no float)
__device__ __forceinline__ float power_for(float m) {
  const int b = __builtin_bit_cast(int, m), e = (b >> 23) - 127 - ((b & 0x7fffff) <= 0x600000 ? 8 : 7);
  return __builtin_bit_cast(float, (m == 0.f ? 31 : min(max(e, -96), 119) + 127) << 23);
}
__device__ __forceinline__ float larger_finite(float m, float x) { x = fabsf(x); return x < INFINITY ? fmaxf(m, x) : m; }
__device__ __forceinline__ float in_units(float x, float inv) {
  const float y = __builtin_amdgcn_fmed3f(x * inv, -448.f, 448.f);
  return fabsf(x) < INFINITY ? y : __builtin_nanf("");
}
__device__ __forceinline__ unsigned four_e4m3(float a, float b, float c, float d) {
  return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
}
// four numbers in another unit
__device__ __forceinline__ unsigned rescaled(unsigned w, float f) {
  return four_e4m3(__builtin_amdgcn_cvt_f32_fp8((int)w, 0) * f, __builtin_amdgcn_cvt_f32_fp8((int)w, 1) * f, __builtin_amdgcn_cvt_f32_fp8((int)w, 2) * f,
                   __builtin_amdgcn_cvt_f32_fp8((int)w, 3) * f);
}
// the bytes of a word whose first is token t, for tokens lo .. hi - 1
__device__ __forceinline__ unsigned byte_mask(int t, int lo, int hi) {
  const int a = min(max(lo - t, 0), 4), b = min(max(hi - t, 0), 4);
  const unsigned below_b = b == 4 ? ~0u : (1u << (8 * b)) - 1u, below_a = a == 4 ? ~0u : (1u << (8 * a)) - 1u;
  return below_b & ~below_a;
}

// float64 to float32.  What is rounded again, to fewer bits, goes by these 32 (the compiler may not make one rounding of the two).
__device__ __forceinline__ float to_f32(double d) {
  float f = (float)d;
  asm("" : "+v"(f));
  return f;
}
// Where the two halves of unit cu of a head lie: 16 columns, which are 8 pairs where they are turned (cu < dims / 16)
template <bool INTER> __device__ __forceinline__ int first_half(const CacheAppend& a, int cu) { return INTER || cu >= a.dims >> 4 ? 16 * cu : 8 * cu; }
template <bool INTER> __device__ __forceinline__ int second_half(const CacheAppend& a, int cu) { return INTER || cu >= a.dims >> 4 ? 16 * cu + 8 : a.dims / 2 + 8 * cu; }
// the unit's 16 numbers, turned (turn: where its 8 cosines and sines are)
template <class T, bool INTER> __device__ __forceinline__ void turned(const Raw8<T>& first, const Raw8<T>& second, bool turn, const double2* cs, float* v) {
#pragma unroll
  for (int i = 0; i < 8; i++) { v[i] = to_f(first.v[i]); v[8 + i] = to_f(second.v[i]); }
  if (turn) {
#pragma unroll
    for (int i = 0; i < 8; i++) {
      float &p = v[INTER ? 2 * i : i], &q = v[INTER ? 2 * i + 1 : 8 + i];
      const double dp = p, dq = q;
      p = to_f32(fma(dp, cs[i].x, -(dq * cs[i].y)));
      q = to_f32(fma(dq, cs[i].x, dp * cs[i].y));
    }
  }
}
__device__ __forceinline__ double2 angle(const CacheAppend& a, int pos, int pair) {
  double2 r = turn_of((double)pos * a.freq[pair]);
  r.x *= a.mag; r.y *= a.mag;
  return r;
}

// Queries: a wave per row, whose angles it works out once, into LDS, and streams all heads past them
template <class T, bool INTER, bool WIDE> __device__ __forceinline__ void turn_queries(const CacheAppend& a, i64 i, double2* cs) {
  const CacheView& c = a.c;
  const int lane = threadIdx.x & 63;
  if (i >= a.T) return;
  for (int s0 = 0; s0 < c.n_seqs; s0 += 64) {
    int2 r = make_int2(0, 0);
    if (s0 + lane < c.n_seqs) r = cache_rows(c, s0 + lane, a.T);
    const unsigned long long hit = __ballot(i >= r.x && i < r.x + r.y);
    if (!hit) continue;
    const int l = __builtin_ctzll(hit), at = cache_len(c, s0 + l) - __builtin_amdgcn_readlane(r.y, l) + (int)(i - __builtin_amdgcn_readlane(r.x, l));
    if (at < 0 || at >= cache_room(c)) return;       // (a row without a place)
    const int pos = a.pos ? a.pos[i] : at, upr = c.dh >> 4, units = a.H * upr;
    const T* q = (const T*)a.q + i * a.ldq;
    T* o = (T*)a.q_out + i * a.ldqo;
    constexpr int N = 4;                             // units whose loads are on their way together
    for (int u0 = lane; u0 - lane < units; u0 += 64 * N) {
      Raw8<T> x[N], y[N];
      int cu[N], at[N];
#pragma unroll
      for (int n = 0; n < N; n++) {
        const int u = min(u0 + 64 * n, units - 1), h = u / upr;
        cu[n] = u - h * upr;
        at[n] = h * c.dh;
        x[n] = load8<T, WIDE>(q + at[n] + first_half<INTER>(a, cu[n]));
        y[n] = load8<T, WIDE>(q + at[n] + second_half<INTER>(a, cu[n]));
      }
      if (u0 == lane) {
        for (int p = lane; p < a.dims >> 1; p += 64) cs[p] = angle(a, pos, p);
        wave_lds_fence();
      }
#pragma unroll
      for (int n = 0; n < N; n++) {
        float v[16];
        turned<T, INTER>(x[n], y[n], cu[n] < a.dims >> 4, cs + 8 * cu[n], v);
        if (u0 + 64 * n < units) {
          store8<T, WIDE>(o + at[n] + first_half<INTER>(a, cu[n]), v);
          store8<T, WIDE>(o + at[n] + second_half<INTER>(a, cu[n]), v + 8);
        }
      }
    }
    return;
  }
}

// A head's rows of a page are `units` of 16 columns: UN per lane of WPH waves.  A workgroup has WPH waves if those are more than four, else four, and
// 4 / WPH heads at a time, `loop` (1 or 2) of them one after the other, all of whose loads are asked for first.  Roles by blockIdx.x: the pages' values
// and keys (vblocks workgroups of each role for each of `visits` pages), then the queries.
template <class T, int UN, int WPH, bool INTER, bool WIDE>
__global__ void __launch_bounds__(WPH > 4 ? WPH * 64 : 256) cache_append_k(CacheAppend a, int visits, int vblocks, int loop) {
  constexpr int WAVES = WPH > 4 ? WPH : 4, HEADS = WAVES / WPH, LANES = 64 * WPH;
  __shared__ float tops[2][WAVES];
  __shared__ double2 turns[WAVES][ROTARY_MAX_DIMS / 2];
  const CacheView& c = a.c;
  const int wv = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), hw = wv / WPH, tid = (int)threadIdx.x - hw * LANES;
  const int role = (int)blockIdx.x / visits, visit = (int)blockIdx.x - role * visits;
  if (role >= 2 * vblocks) {                         // (queries: beyond the pages' workgroups)
    turn_queries<T, INTER, WIDE>(a, (i64)((int)blockIdx.x - 2 * vblocks * visits) * WAVES + wv, turns[wv]);
    return;
  }
  const int P = 1 << c.lg, room = cache_room(c), dh = c.dh;
  int s, nth;
  auto pages_of = [&](int s) {
    const int n = cache_rows(c, s, a.T).y, len = cache_len(c, s), first = max(len - n, 0), end = min(len, room);
    return end > first ? ((end - 1) >> c.lg) - (first >> c.lg) + 1 : 0;
  };
  if (!find_item(c.n_seqs, visit, pages_of, &s, &nth)) return;
  const int2 rows = cache_rows(c, s, a.T);
  const int len = cache_len(c, s), start = len - rows.y, first = max(start, 0), p = (first >> c.lg) + nth, at0 = p << c.lg;
  const int page = cache_page(c, s, p), r0 = max(first - at0, 0), r1 = min(min(len, room) - at0, P);      // rows r0 .. r1 - 1 of the page
  const i64 token0 = (i64)rows.x + (at0 - start);    // row 0 of the page, as a row of the call (may lie before the first)
  if (page < 0) return;
  const bool keys = role >= vblocks;
  const int h0 = (keys ? role - vblocks : role) * loop * HEADS + hw;           // then h0 + HEADS

  // the unit to use: the least that brings `top` of all the head's waves within 448, and not less than the page's (where it holds rows already)
  auto unit_for = [&](float top, float old, int n) {
    top = wave_max(top);
    if constexpr (WPH > 1) {
      if ((threadIdx.x & 63) == 0) tops[n][wv] = top;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < WPH; w++) top = fmaxf(top, tops[n][hw * WPH + w]);
    }
    const float now = power_for(top);
    return r0 > 0 ? fmaxf(now, old) : now;
  };

  if (!keys) {                                       // values: 16 tokens of two columns per lane, which are 16 bytes of each column
    static_assert(UN <= 2, "a lane's 32 values are two units");
    typedef __attribute__((ext_vector_type(2))) T V2;
    const int u = tid, g = u / (dh >> 1), col = 2 * (u - g * (dh >> 1)), t0 = 16 * g;
    V2 raw[2][16];
    float olds[2];
#pragma unroll
    for (int n = 0; n < 2; n++) {
      const int h = h0 + n * HEADS;
      const bool live = n < loop && h < c.Hkv;
      olds[n] = live ? c.vs[cache_block(c, page, h)] : 0.f;
#pragma unroll
      for (int t = 0; t < 16; t++) {
        raw[n][t] = V2{};
        const int r = t0 + t;
        if (live && r >= r0 && r < r1) {
          const T* v = (const T*)a.v + (token0 + r) * a.ldv + (i64)h * dh + col;
          if constexpr (WIDE) raw[n][t] = *(const V2*)v;
          else { raw[n][t][0] = v[0]; raw[n][t][1] = v[1]; }
        }
      }
    }
#pragma unroll
    for (int n = 0; n < 2; n++) {
      if (n >= loop) break;
      const int h = h0 + n * HEADS;
      const bool live = h < c.Hkv;
      const float old = olds[n];
      float x[2][16], top = 0.f;
#pragma unroll
      for (int t = 0; t < 16; t++) {
        x[0][t] = to_f(raw[n][t][0]);
        x[1][t] = to_f(raw[n][t][1]);
        top = larger_finite(larger_finite(top, x[0][t]), x[1][t]);
      }
      const float now = unit_for(top, old, n), inv = 1.f / now, again = old * inv;
      const bool more = r0 > 0 && now > old;
      if (!live || t0 >= P || t0 >= r1) continue;
      const i64 block = cache_block(c, page, h);
      unsigned char* vp = c.v + (block << c.lg) * dh;
      if (tid == 0) c.vs[block] = now;
      if (t0 + 16 <= r0 && !more) continue;
      const bool whole = t0 >= r0 && t0 + 16 <= r1;
#pragma unroll
      for (int k = 0; k < 2; k++) {
        uint4* at = (uint4*)(vp + (i64)(t0 * dh + 16 * (col + k)));
        uint4 held = make_uint4(0, 0, 0, 0);
        if (!whole) held = *at;
        unsigned w[4] = {held.x, held.y, held.z, held.w};
#pragma unroll
        for (int i = 0; i < 4; i++) {
          const float* y = x[k] + 4 * i;
          const unsigned mine = byte_mask(t0 + 4 * i, r0, r1), below = byte_mask(t0 + 4 * i, 0, r0);
          unsigned keep = w[i];
          if (more) keep = (rescaled(keep, again) & below) | (keep & ~below);
          const unsigned fresh = four_e4m3(in_units(y[0], inv), in_units(y[1], inv), in_units(y[2], inv), in_units(y[3], inv));
          w[i] = (fresh & mine) | (keep & ~mine);
        }
        *at = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
    return;
  }

  const int upr = dh >> 4;
  int row[UN], cu[UN];
  bool in[UN];
  Raw8<T> xa[2][UN], xb[2][UN];
  float olds[2];
#pragma unroll
  for (int j = 0; j < UN; j++) {
    const int u = tid + LANES * j, r = u / upr;
    cu[j] = u - r * upr;
    row[j] = r0 + r;
    in[j] = row[j] < r1;
  }
#pragma unroll
  for (int n = 0; n < 2; n++) {
    const int h = h0 + n * HEADS;
    const bool live = n < loop && h < c.Hkv;
    olds[n] = live ? c.ks[cache_block(c, page, h)] : 0.f;
#pragma unroll
    for (int j = 0; j < UN; j++)
      if (live && in[j]) {
        const T* k = (const T*)a.k + (token0 + row[j]) * a.ldk + (i64)h * dh;
        xa[n][j] = load8<T, WIDE>(k + first_half<INTER>(a, cu[j]));
        xb[n][j] = load8<T, WIDE>(k + second_half<INTER>(a, cu[j]));
      }
  }
  double2 cs[UN][8];
#pragma unroll
  for (int j = 0; j < UN; j++)
    if (in[j] && cu[j] < a.dims >> 4) {
      const int pos = a.pos ? a.pos[token0 + row[j]] : at0 + row[j];
#pragma unroll
      for (int i = 0; i < 8; i++) cs[j][i] = angle(a, pos, 8 * cu[j] + i);
    }
#pragma unroll
  for (int n = 0; n < 2; n++) {
    if (n >= loop) break;
    const int h = h0 + n * HEADS;
    const bool live = h < c.Hkv;
    const float old = olds[n];
    float x[UN][16], top = 0.f;
#pragma unroll
    for (int j = 0; j < UN; j++)
      if (live && in[j]) {
        turned<T, INTER>(xa[n][j], xb[n][j], cu[j] < a.dims >> 4, cs[j], x[j]);
#pragma unroll
        for (int i = 0; i < 16; i++) {
          x[j][i] = to_f(from_f<T>(x[j][i]));        // (a key is rounded to float32, to its type, and then to 8 bits)
          top = larger_finite(top, x[j][i]);
        }
      }
    const float now = unit_for(top, old, n), inv = 1.f / now, again = old * inv;
    if (!live) continue;
    const i64 block = cache_block(c, page, h);
    unsigned char* kp = c.k + (block << c.lg) * dh;
    if (tid == 0) c.ks[block] = now;
    if (r0 > 0 && now > old)                         // what the page holds already, in the new unit
      for (int o = tid * 16; o < r0 * dh; o += LANES * 16) {
        uint4 w = *(uint4*)(kp + o);
        w.x = rescaled(w.x, again); w.y = rescaled(w.y, again); w.z = rescaled(w.z, again); w.w = rescaled(w.w, again);
        *(uint4*)(kp + o) = w;
      }
#pragma unroll
    for (int j = 0; j < UN; j++)
      if (in[j]) {
        float* y = x[j];
#pragma unroll
        for (int i = 0; i < 16; i++) y[i] = in_units(y[i], inv);
        *(uint2*)(kp + row[j] * dh + first_half<INTER>(a, cu[j])) = make_uint2(four_e4m3(y[0], y[1], y[2], y[3]), four_e4m3(y[4], y[5], y[6], y[7]));
        *(uint2*)(kp + row[j] * dh + second_half<INTER>(a, cu[j])) = make_uint2(four_e4m3(y[8], y[9], y[10], y[11]), four_e4m3(y[12], y[13], y[14], y[15]));
      }
  }
}

// Waves per head of a page, and what follows from them: a launch's grid
struct AppendShape { int wph, waves, loop, vblocks; i64 visits, grid; };
static AppendShape shape_of(const CacheAppend& a) {
  const CacheView& c = a.c;
  const int units = (c.dh << c.lg) >> 4;
  AppendShape r;
  r.wph = units <= 64 ? 1 : units <= 128 ? 2 : units <= 512 ? 4 : 8;
  r.waves = r.wph > 4 ? r.wph : 4;
  // a sequence's n new rows meet at most (n - 1) / page + 2 pages
  r.visits = c.cu ? ((i64)a.T >> c.lg) + 2 * (i64)(c.n_seqs < a.T ? c.n_seqs : a.T) : (a.T < c.n_seqs ? a.T : c.n_seqs);
  const int heads = r.waves / r.wph;
  r.loop = r.visits * cdiv(c.Hkv, heads) >= 512 ? 2 : 1;
  r.vblocks = cdiv(c.Hkv, heads * r.loop);
  r.grid = r.visits * 2 * r.vblocks + (a.q ? cdiv(a.T, r.waves) : 0);
  return r;
}
bool cache_append_fits(const CacheAppend& a) {
  const AppendShape r = shape_of(a);
  return r.grid * (r.waves * 64) < (i64)1 << 32;
}
template <class T, int UN, int WPH> static void launch(const CacheAppend& a, const AppendShape& r, bool wide, hipStream_t s) {
  const dim3 grid((unsigned)r.grid), block(r.waves * 64);
  const int visits = (int)r.visits;
  if (a.interleaved) {
    if (wide) hipLaunchKernelGGL((cache_append_k<T, UN, WPH, true, true>), grid, block, 0, s, a, visits, r.vblocks, r.loop);
    else hipLaunchKernelGGL((cache_append_k<T, UN, WPH, true, false>), grid, block, 0, s, a, visits, r.vblocks, r.loop);
  } else {
    if (wide) hipLaunchKernelGGL((cache_append_k<T, UN, WPH, false, true>), grid, block, 0, s, a, visits, r.vblocks, r.loop);
    else hipLaunchKernelGGL((cache_append_k<T, UN, WPH, false, false>), grid, block, 0, s, a, visits, r.vblocks, r.loop);
  }
}
template <class T> static void launch(const CacheAppend& a, const AppendShape& r, bool wide, hipStream_t s) {
  switch (r.wph) {
    case 1: launch<T, 1, 1>(a, r, wide, s); break;
    case 2: launch<T, 1, 2>(a, r, wide, s); break;
    case 4: if ((a.c.dh << a.c.lg) >> 4 <= 256) launch<T, 1, 4>(a, r, wide, s); else launch<T, 2, 4>(a, r, wide, s); break;
    default: launch<T, 2, 8>(a, r, wide, s);
  }
}
void launch_cache_append(const CacheAppend& a, hipStream_t s) {
  const AppendShape r = shape_of(a);
  if (r.visits == 0) return;
  const int es = a.dt == 0 ? 4 : 2;
  const i64 strides = a.ldk | a.ldv | (a.q ? a.ldq | a.ldqo : 0);
  const uintptr_t at = (uintptr_t)a.k | (uintptr_t)a.v | (a.q ? (uintptr_t)a.q | (uintptr_t)a.q_out : 0);
  const bool wide = strides * es % 16 == 0 && at % 16 == 0;
  if (a.dt == 0) launch<float>(a, r, wide, s);
  else launch<bf16>(a, r, wide, s);
}
