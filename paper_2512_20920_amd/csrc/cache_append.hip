// New keys and values into the pages of a cache, keys and queries turned to their positions on the way.
//
// A workgroup takes the new rows of one page (a sequence's pages one after the other: find_item) and a share of the heads: the
// angles of its rows stay in registers from head to head.  For a key head it takes the largest value of all its rows' keys and
// of their values, two numbers that meet in LDS, before the first number is written.
#include "cache.h"
#include "rotary.h"

// Eight columns of a row.  WIDE: 16 bytes at a time.
template <class T, bool WIDE> __device__ __forceinline__ void load8(const T* p, float* x) {
  if constexpr (WIDE && sizeof(T) == 2) {
    typedef __attribute__((ext_vector_type(8))) T V;
    const V v = *(const V*)p;
#pragma unroll
    for (int i = 0; i < 8; i++) x[i] = to_f(v[i]);
  } else if constexpr (WIDE) {
    const float4 u = *(const float4*)p, w = *(const float4*)(p + 4);
    x[0] = u.x; x[1] = u.y; x[2] = u.z; x[3] = u.w; x[4] = w.x; x[5] = w.y; x[6] = w.z; x[7] = w.w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++) x[i] = to_f(p[i]);
  }
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

// UN: units of 16 columns per thread that a page's rows of a head make (a page times a head's width is at most 16384)
template <class T, int UN, bool INTER, bool WIDE>
__global__ void __launch_bounds__(256) cache_append_k(CacheAppend a) {
  __shared__ float tops[2][2][4];
  const CacheView& c = a.c;
  const int tid = threadIdx.x, wv = tid >> 6, P = 1 << c.lg, room = cache_room(c), dh = c.dh;
  int s, nth;
  auto pages_of = [&](int s) {
    const int n = cache_rows(c, s, a.T).y, len = cache_len(c, s), first = max(len - n, 0), end = min(len, room);
    return end > first ? ((end - 1) >> c.lg) - (first >> c.lg) + 1 : 0;
  };
  if (!find_item(c.n_seqs, (int)blockIdx.x, pages_of, &s, &nth)) return;
  const int2 rows = cache_rows(c, s, a.T);
  const int len = cache_len(c, s), start = len - rows.y, first = max(start, 0), p = (first >> c.lg) + nth, at0 = p << c.lg;
  const int page = cache_page(c, s, p), r0 = max(first - at0, 0), r1 = min(min(len, room) - at0, P);      // rows r0 .. r1 - 1 of the page
  const i64 token0 = (i64)rows.x + (at0 - start);    // row 0 of the page, as a row of the call (may lie before the first)

  const int upr = dh >> 4, turned = a.dims >> 4;
  int row[UN], ca[UN], cb[UN];
  bool in[UN], turn[UN];
  float2 cs[UN][8];
#pragma unroll
  for (int j = 0; j < UN; j++) {
    const int u = tid + 256 * j, r = u / upr, cu = u - r * upr;
    row[j] = r0 + r;
    in[j] = row[j] < r1;
    turn[j] = cu < turned;
    ca[j] = INTER || !turn[j] ? 16 * cu : 8 * cu;
    cb[j] = INTER || !turn[j] ? 16 * cu + 8 : a.dims / 2 + 8 * cu;
    if (in[j] && turn[j]) {
      const int pos = a.pos ? a.pos[token0 + row[j]] : at0 + row[j];
#pragma unroll
      for (int i = 0; i < 8; i++) cs[j][i] = rotary_turn(a.freq[8 * cu + i], pos, a.mag, 1.f);
    }
  }
  auto load_turned = [&](const T* x, int j, float* v) {
    load8<T, WIDE>(x + ca[j], v);
    load8<T, WIDE>(x + cb[j], v + 8);
    if (turn[j]) {
#pragma unroll
      for (int i = 0; i < 8; i++)
        if constexpr (INTER) rotary_pair(v[2 * i], v[2 * i + 1], cs[j][i]);
        else rotary_pair(v[i], v[8 + i], cs[j][i]);
    }
  };

  const int chunks = gridDim.y, y = blockIdx.y;
  if (page >= 0)
    for (int h = y * c.Hkv / chunks; h < (y + 1) * c.Hkv / chunks; h++) {
      const i64 block = cache_block(c, page, h);
      unsigned char *kp = c.k + (block << c.lg) * dh, *vp = c.v + (block << c.lg) * dh;
      const float old_k = c.ks[block], old_v = c.vs[block];
      float kx[UN][16], top_k = 0.f, top_v = 0.f;
#pragma unroll
      for (int j = 0; j < UN; j++)
        if (in[j]) {
          load_turned((const T*)a.k + (token0 + row[j]) * a.ldk + (i64)h * dh, j, kx[j]);
#pragma unroll
          for (int i = 0; i < 16; i++) {
            kx[j][i] = to_f(from_f<T>(kx[j][i]));    // (a key is what the rotation alone would store, then in 8 bits)
            top_k = larger_finite(top_k, kx[j][i]);
          }
        }
      // values: 16 tokens of two columns per thread, which are 16 bytes of each column
      constexpr int VN = UN > 1 ? UN / 2 : 1;
      float vx[VN][2][16];
#pragma unroll
      for (int j = 0; j < VN; j++) {
        const int u = tid + 256 * j, g = u / (dh >> 1), col = 2 * (u - g * (dh >> 1));
#pragma unroll
        for (int t = 0; t < 16; t++) {
          vx[j][0][t] = vx[j][1][t] = 0.f;
          const int r = 16 * g + t;
          if (r >= r0 && r < r1) {
            const T* x = (const T*)a.v + (token0 + r) * a.ldv + (i64)h * dh + col;
            if constexpr (WIDE) {
              typedef __attribute__((ext_vector_type(2))) T V;
              const V v = *(const V*)x;
              vx[j][0][t] = to_f(v[0]); vx[j][1][t] = to_f(v[1]);
            } else { vx[j][0][t] = to_f(x[0]); vx[j][1][t] = to_f(x[1]); }
            top_v = larger_finite(larger_finite(top_v, vx[j][0][t]), vx[j][1][t]);
          }
        }
      }
      top_k = wave_max(top_k);
      top_v = wave_max(top_v);
      if ((tid & 63) == 0) { tops[h & 1][0][wv] = top_k; tops[h & 1][1][wv] = top_v; }
      __syncthreads();                               // (the next head's go to the other half: one barrier per head is enough)
      float now_k = 0.f, now_v = 0.f;
#pragma unroll
      for (int w = 0; w < 4; w++) { now_k = fmaxf(now_k, tops[h & 1][0][w]); now_v = fmaxf(now_v, tops[h & 1][1][w]); }
      now_k = power_for(now_k);
      now_v = power_for(now_v);
      if (r0 > 0) { now_k = fmaxf(now_k, old_k); now_v = fmaxf(now_v, old_v); }
      const bool more_k = r0 > 0 && now_k > old_k, more_v = r0 > 0 && now_v > old_v;
      const float inv_k = 1.f / now_k, inv_v = 1.f / now_v, again_k = old_k * inv_k, again_v = old_v * inv_v;
      if (tid == 0) { c.ks[block] = now_k; c.vs[block] = now_v; }
      if (more_k)                                    // what the page holds already, in the new unit
        for (int o = tid * 16; o < r0 * dh; o += 4096) {
          uint4 w = *(uint4*)(kp + o);
          w.x = rescaled(w.x, again_k); w.y = rescaled(w.y, again_k); w.z = rescaled(w.z, again_k); w.w = rescaled(w.w, again_k);
          *(uint4*)(kp + o) = w;
        }
#pragma unroll
      for (int j = 0; j < UN; j++)
        if (in[j]) {
          float* x = kx[j];
#pragma unroll
          for (int i = 0; i < 16; i++) x[i] = in_units(x[i], inv_k);
          *(uint2*)(kp + row[j] * dh + ca[j]) = make_uint2(four_e4m3(x[0], x[1], x[2], x[3]), four_e4m3(x[4], x[5], x[6], x[7]));
          *(uint2*)(kp + row[j] * dh + cb[j]) = make_uint2(four_e4m3(x[8], x[9], x[10], x[11]), four_e4m3(x[12], x[13], x[14], x[15]));
        }
#pragma unroll
      for (int j = 0; j < VN; j++) {
        const int u = tid + 256 * j, g = u / (dh >> 1), col = 2 * (u - g * (dh >> 1)), t0 = 16 * g;
        if (t0 >= P || t0 >= r1 || (t0 + 16 <= r0 && !more_v)) continue;
        const bool whole = t0 >= r0 && t0 + 16 <= r1;
#pragma unroll
        for (int k = 0; k < 2; k++) {
          uint4* at = (uint4*)(vp + (i64)(t0 * dh + 16 * (col + k)));
          uint4 held = make_uint4(0, 0, 0, 0);
          if (!whole) held = *at;
          unsigned w[4] = {held.x, held.y, held.z, held.w};
#pragma unroll
          for (int i = 0; i < 4; i++) {
            const float* x = vx[j][k] + 4 * i;
            const unsigned mine = byte_mask(t0 + 4 * i, r0, r1), below = byte_mask(t0 + 4 * i, 0, r0);
            unsigned keep = w[i];
            if (more_v) keep = (rescaled(keep, again_v) & below) | (keep & ~below);
            const unsigned fresh = four_e4m3(in_units(x[0], inv_v), in_units(x[1], inv_v), in_units(x[2], inv_v), in_units(x[3], inv_v));
            w[i] = (fresh & mine) | (keep & ~mine);
          }
          *at = make_uint4(w[0], w[1], w[2], w[3]);
        }
      }
    }
  if (a.q)
    for (int h = y * a.H / chunks; h < (y + 1) * a.H / chunks; h++)
#pragma unroll
      for (int j = 0; j < UN; j++)
        if (in[j]) {
          float v[16];
          load_turned((const T*)a.q + (token0 + row[j]) * a.ldq + (i64)h * dh, j, v);
          T* o = (T*)a.q_out + (token0 + row[j]) * a.ldqo + (i64)h * dh;
          store8<T, WIDE>(o + ca[j], v);
          store8<T, WIDE>(o + cb[j], v + 8);
        }
}

template <class T, int UN, bool INTER> static void launch(const CacheAppend& a, dim3 grid, bool wide, hipStream_t s) {
  if (wide) hipLaunchKernelGGL((cache_append_k<T, UN, INTER, true>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((cache_append_k<T, UN, INTER, false>), grid, dim3(256), 0, s, a);
}
template <class T> static void launch(const CacheAppend& a, dim3 grid, bool wide, hipStream_t s) {
  const int un = cdiv((i64)a.c.dh << a.c.lg, 4096);
  if (a.interleaved) {
    if (un <= 1) launch<T, 1, true>(a, grid, wide, s);
    else if (un <= 2) launch<T, 2, true>(a, grid, wide, s);
    else launch<T, 4, true>(a, grid, wide, s);
  } else {
    if (un <= 1) launch<T, 1, false>(a, grid, wide, s);
    else if (un <= 2) launch<T, 2, false>(a, grid, wide, s);
    else launch<T, 4, false>(a, grid, wide, s);
  }
}
void launch_cache_append(const CacheAppend& a, hipStream_t s) {
  const CacheView& c = a.c;
  // a sequence's n new rows meet at most (n - 1) / page + 2 pages
  const i64 visits = c.cu ? ((i64)a.T >> c.lg) + 2 * (i64)(c.n_seqs < a.T ? c.n_seqs : a.T) : (a.T < c.n_seqs ? a.T : c.n_seqs);
  if (visits == 0) return;
  const int heads = a.q && a.H > c.Hkv ? a.H : c.Hkv;
  i64 chunks = 1024 / visits;
  if (chunks < 1) chunks = 1;
  if (chunks > heads) chunks = heads;
  const int es = a.dt == 0 ? 4 : 2;
  const i64 strides = a.ldk | a.ldv | (a.q ? a.ldq | a.ldqo : 0);
  const uintptr_t at = (uintptr_t)a.k | (uintptr_t)a.v | (a.q ? (uintptr_t)a.q | (uintptr_t)a.q_out : 0);
  const bool wide = strides * es % 16 == 0 && at % 16 == 0;
  const dim3 grid((unsigned)visits, (unsigned)chunks);
  if (a.dt == 0) launch<float>(a, grid, wide, s);
  else launch<bf16>(a, grid, wide, s);
}
