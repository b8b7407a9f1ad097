// Attention over a paged cache of 8-bit numbers (cache.h) on the matrix cores.
//
// Rows are (query, head) pairs that share a key head.  A wave works on transposed scores S^T[key, row] = K Q^T, as the kernels over key ranges do, but
// nothing of the cache goes through LDS: both operands that come from it lie there as a lane needs them, 16 bytes at a time, and turn into bfloat16, their
// power of two included, without a rounding (v_cvt_scalef32_pk_bf16_fp8).  In the form for many rows (32 per wave, tiles of 32 keys, 32x32x16):
//  * K: row m of the operand is the tile's token 16 ((m >> 2) & 1) + 4 (m >> 3) + (m & 3), so that the 16 scores that a lane gets (rows
//    8 (e >> 2) + 4 g + (e & 3) of the result, g = lane >> 5) are tokens 16 g + e, in order.  The head's columns are contracted in the order in which
//    16 bytes of a row hold them: step 2 t takes columns 32 t + 16 g + 0..7, step 2 t + 1 the next eight; Q is loaded alike.
//  * V: a lane's 16 probabilities are those of 16 tokens in a row, which are the 16 bytes of one column that the cache keeps together.
// In the form for few rows (16 per workgroup, whose waves share the keys out in tiles of 64, 16x16x32) the same with g = lane >> 4: four runs of 16 tokens,
// four blocks b of 16 keys whose row m is token 16 (m >> 2) + 4 b + (m & 3).
// Scores, maxima, sums and accumulators are float32.  bfloat16 calls round the probabilities to bfloat16 as operands (results are
// then 1.1 to 1.4 times as far from 64 bits, relative error 0.0023 for a prompt's piece, as with probabilities that would take three products); float32 calls take queries
// and probabilities as three bfloat16 numbers each (24 bits; the cache's numbers need no more than one), so they are float32 throughout.
#include "attn_range_tiles.h"
#include "cache.h"

namespace {

constexpr int FEW_ROWS = 64;             // of a sequence and key head: up to here groups of 16 rows, beyond groups of 1 << lr, 32 for each of the waves

// A row's reference for its exponentials is a maximum that may be this much behind, in units of log2: then results are rescaled in a few tiles instead of
// in more than half of them, and no exponential is past 2^8, of which bfloat16 and float32 hold as many bits as of one below 1.
constexpr float HEADROOM = 8.f;

// What a call does with a sequence.  Keys begin .. end - 1 are seen by some row; cost: tiles of 32 keys for a wave of a workgroup (a group) of rows.
struct SeqWork { int row0, n, start, begin, end, groups, cost; bool few; };
__device__ __forceinline__ SeqWork work_of(const CachedAttn& a, int s) {
  SeqWork w;
  const int2 rows = cache_rows(a.c, s, a.T);
  const int len = cache_len(a.c, s);
  w.row0 = rows.x; w.n = rows.y;
  w.start = len - rows.y;                            // where the first row stands
  w.end = min(len, cache_room(a.c));
  w.begin = a.window ? max(w.start + 1 - a.window, 0) : 0;
  const i64 R = (i64)rows.y * a.G;
  w.few = a.few_only || R <= FEW_ROWS;
  w.groups = (int)(w.few ? (R + 15) >> 4 : (R + (1 << a.lr) - 1) >> a.lr);
  const int tiles = w.end > w.begin ? ((w.end - 1) >> 5) - (w.begin >> 5) + 1 : 0;
  w.cost = w.few ? (tiles + 3) >> 2 : (tiles + (128 >> a.lr) - 1) >> (7 - a.lr);
  return w;
}
// Into how many parts a group's keys go, if `per` tiles per wave are the aim: up to 64
__device__ __forceinline__ int splits_of(const CachedAttn& a, const SeqWork& w, int per) {
  if (a.split == 0 || (!w.few && a.split == 1)) return 1;
  if (!w.few) per = max(per, a.dt == 0 ? 4 : 8);     // (128 rows' parts are work to join; float32 tiles take three times the products: 20.8 -> 18.5 us with 4 at 256 tokens)
  return min(max((w.cost + per - 1) / per, 1), 64);
}
// A call's list of workgroups: sequence by sequence, and in it (split, group, key head), key heads fastest (one stays on one XCD if there are eight).
// Parts of split groups lie in the scratch memory in the same order, in slots of 16 rows: one per workgroup (few) or as many as its rows fill.
// JOIN: the list of four rows each of the split groups instead.
struct Item { int s, at, splits; i64 slot; SeqWork w; };
template <bool JOIN> __device__ __forceinline__ bool find(const CachedAttn& a, int id, Item* x) {
  const int lane = threadIdx.x & 63, n = a.c.n_seqs;
  SeqWork first = {};
  if (lane < n) first = work_of(a, lane);
  int per = 1;                                       // tiles per wave
  if (a.split) {
    // as many as make a.target workgroups of everything: with one more, those and one for each group are always enough.  Rounded up to whole workgroups
    // for each group that may be some too many to be on the CUs together, and then per grows until they are (lists of up to 64 sequences).
    float sum = 0.f, groups = 0.f;
    for (int s0 = 0; s0 < n; s0 += 64) {
      const SeqWork w = s0 == 0 ? first : s0 + lane < n ? work_of(a, s0 + lane) : SeqWork{};
      sum += (float)w.groups * (float)w.cost;
      groups += (float)w.groups;
    }
    const float heads = (float)a.c.Hkv;
    per = (int)fminf(wave_sum(sum) * (heads / (float)a.target), 0x1p30f) + 1;
    if (per > 1 && n <= 64) {
      const float most = fmaxf((float)a.target, wave_sum(groups) * heads);
      for (int i = 0; i < 8; i++) {
        const float all = wave_sum((float)first.groups * (float)splits_of(a, first, per)) * heads;
        if (all <= most) break;
        per = max(per + 1, (int)((float)per * all / most));
      }
    }
  }
  int before = 0;
  i64 slots = 0;
  for (int s0 = 0; s0 < n; s0 += 64) {
    const SeqWork w = s0 == 0 ? first : s0 + lane < n ? work_of(a, s0 + lane) : SeqWork{};
    const int k = splits_of(a, w, per);
    // (first rows that are out of order can ask for more than there are: a sequence has at most all T of them, with T * H < 2^26 no sum of 64 overflows, and
    // whoever is past the scratch memory stays out of it)
    const int groups = w.groups * a.c.Hkv, quads = (int)(((i64)w.n * a.G + 3) >> 2) * a.c.Hkv;
    const int mine = min(JOIN ? (k > 1 ? quads : 0) : groups * k, 1 << 24);
    const int room = min(k > 1 ? groups * k * (w.few ? 1 : 1 << (a.lr - 4)) : 0, 1 << 24);
    const int running = wave_running(mine), all = __builtin_amdgcn_readlane(running, 63), rooms = wave_running(room);
    if (id < before + all) {
      const int l = __builtin_ctzll(__ballot(before + running > id));
      x->s = s0 + l;
      x->at = id - before - (__builtin_amdgcn_readlane(running, l) - __builtin_amdgcn_readlane(mine, l));
      x->slot = slots + __builtin_amdgcn_readlane(rooms, l) - __builtin_amdgcn_readlane(room, l);
      x->splits = __builtin_amdgcn_readlane(k, l);
      x->w.row0 = __builtin_amdgcn_readlane(w.row0, l); x->w.n = __builtin_amdgcn_readlane(w.n, l); x->w.start = __builtin_amdgcn_readlane(w.start, l);
      x->w.begin = __builtin_amdgcn_readlane(w.begin, l); x->w.end = __builtin_amdgcn_readlane(w.end, l);
      x->w.groups = __builtin_amdgcn_readlane(w.groups, l); x->w.cost = __builtin_amdgcn_readlane(w.cost, l); x->w.few = __builtin_amdgcn_readlane((int)w.few, l);
      return true;
    }
    before += all;
    slots += __builtin_amdgcn_readlane(rooms, 63);
  }
  return false;
}

// Keys that the query at `pos` sees
__device__ __forceinline__ int2 seen_from(const CachedAttn& a, int pos, int end) {
  int2 r = make_int2(a.window ? max(pos + 1 - a.window, 0) : 0, a.causal ? min(pos + 1, end) : end);
  if (r.x >= r.y) r = make_int2(0, 0);
  return r;
}

// One row by a wave of its own, which touches only what the row sees: 64 keys at a time, then the columns.  lds: dh floats of this wave's own.
template <class T> __device__ void cached_row(const CachedAttn& a, int s, int i, int h, int pos, int end, float* lds) {
  const CacheView& c = a.c;
  const int lane = threadIdx.x & 63, dh = c.dh, kh = h / a.G, P1 = (1 << c.lg) - 1;
  const int2 r = seen_from(a, pos, end);
  const T* q = (const T*)a.q + (i64)i * a.ldq + (i64)h * dh;
  wave_lds_fence();
  for (int d = lane; d < dh; d += 64) lds[d] = to_f(q[d]);
  wave_lds_fence();
  const float slope = a.slopes ? a.slopes[h] : 0.f;
  float acc[4] = {}, m = -INFINITY, l = 0.f;
  for (int j0 = r.x; j0 < r.y; j0 += 64) {
    const int j = j0 + lane, page = j < r.y ? cache_page(c, s, j >> c.lg) : -1;
    const bool sees = page >= 0;
    const i64 block = cache_block(c, max(page, 0), kh);
    float x = -INFINITY, keep, unit = 0.f;
    if (sees) {
      const unsigned* k = (const unsigned*)(c.k + ((block << c.lg) + (j & P1)) * dh);
      float s0 = 0.f, s1 = 0.f;
      for (int d = 0; d < dh; d += 4) {
        const int w = (int)k[d >> 2];
        s0 = fmaf(__builtin_amdgcn_cvt_f32_fp8(w, 0), lds[d], s0); s1 = fmaf(__builtin_amdgcn_cvt_f32_fp8(w, 1), lds[d + 1], s1);
        s0 = fmaf(__builtin_amdgcn_cvt_f32_fp8(w, 2), lds[d + 2], s0); s1 = fmaf(__builtin_amdgcn_cvt_f32_fp8(w, 3), lds[d + 3], s1);
      }
      x = range_score((s0 + s1) * c.ks[block] * a.scale, a.cap, slope, pos, j, &keep);
      unit = c.vs[block];
    }
    const float mn = fmaxf(m, wave_max(x)), ms = mn == -INFINITY ? 0.f : mn;
    const float p = sees ? expf(x - ms) : 0.f, alpha = expf(m - ms);
    l = l * alpha + wave_sum(p);
#pragma unroll
    for (int u = 0; u < 4; u++) acc[u] *= alpha;
    m = mn;
    unsigned long long live = __ballot(sees);
    while (live) {
      const int b = __builtin_ctzll(live);
      live &= live - 1;
      const float f = __shfl(p * unit, b, WAVE);
      const int jb = (j0 + b) & P1, pg = __shfl(page, b, WAVE);
      const unsigned char* v = c.v + ((cache_block(c, pg, kh) << c.lg) + (jb & ~15)) * dh + (jb & 15);
#pragma unroll
      for (int u = 0; u < 4; u++) if (lane + 64 * u < dh) acc[u] = fmaf(f, e4m3_value(v[(lane + 64 * u) * 16]), acc[u]);
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  T* o = (T*)a.out + (i64)i * a.ldo + (i64)h * dh;
#pragma unroll
  for (int u = 0; u < 4; u++) if (lane + 64 * u < dh) o[lane + 64 * u] = from_f<T>(acc[u] * inv);
  if (lane == 0 && a.lse) a.lse[(i64)h * a.T + i] = l == 0.f ? -INFINITY : m + logf(l);
}

template <class T> __global__ void __launch_bounds__(256) cached_rows_k(CachedAttn a) {
  __shared__ float lds[4][256];
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const i64 id = (i64)blockIdx.x * 4 + wv;
  const int i = (int)(id / a.H), h = (int)(id - (i64)i * a.H);
  if (i >= a.T) return;
  for (int s0 = 0; s0 < a.c.n_seqs; s0 += 64) {
    int2 r = make_int2(0, 0);
    if (s0 + lane < a.c.n_seqs) r = cache_rows(a.c, s0 + lane, a.T);
    const unsigned long long hit = __ballot(i >= r.x && i < r.x + r.y);
    if (hit) {
      const int s = s0 + __builtin_ctzll(hit);
      const SeqWork w = work_of(a, s);
      cached_row<T>(a, s, i, h, w.start + (i - w.row0), w.end, lds[wv]);
      return;
    }
  }
}

__device__ __forceinline__ float lane_f(float v, int l) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), l)); }

// ---- the matrix-core kernel ----
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
// 8 numbers of the cache times a power of two
__device__ __forceinline__ bf16x8 eight(unsigned lo, unsigned hi, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  const uint4 r = make_uint4(__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, b), __builtin_bit_cast(unsigned, c), __builtin_bit_cast(unsigned, d));
  return __builtin_bit_cast(bf16x8, r);
}
__device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
// over the lanes l, l ^ 16, l ^ 32, l ^ 48
__device__ __forceinline__ float quarters_max(float x) {
  const unsigned b = __builtin_bit_cast(unsigned, x);
  const auto r = __builtin_amdgcn_permlane16_swap(b, b, false, false);
  return both_halves_max(fmaxf(__builtin_bit_cast(float, (unsigned)r[0]), __builtin_bit_cast(float, (unsigned)r[1])));
}
__device__ __forceinline__ float quarters_sum(float x) {
  const unsigned b = __builtin_bit_cast(unsigned, x);
  const auto r = __builtin_amdgcn_permlane16_swap(b, b, false, false);
  return both_halves_sum(__builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]));
}
// 16 columns of a row of queries, as Q numbers each (zeros for a row that is not there)
template <class T, int Q> __device__ __forceinline__ void load_q16(const T* q, bool ok, bf16x8 (*f)[2]) {
  float v[16];
#pragma unroll
  for (int u = 0; u < 16; u++) v[u] = 0.f;
  if (ok) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int u = 0; u < 16; u += 4) { const float4 w = *(const float4*)(q + u); v[u] = w.x; v[u + 1] = w.y; v[u + 2] = w.z; v[u + 3] = w.w; }
    } else {
#pragma unroll
      for (int u = 0; u < 16; u += 8) {
        const bf16x8 w = *(const bf16x8*)(q + u);
#pragma unroll
        for (int k = 0; k < 8; k++) v[u + k] = (float)w[k];
      }
    }
  }
#pragma unroll
  for (int p = 0; p < Q; p++)
#pragma unroll
    for (int u = 0; u < 16; u++) {
      const bf16 b = (bf16)v[u];
      f[p][u >> 3][u & 7] = b;
      v[u] -= (float)b;
    }
}
// The scores' final form (MOD), but for a last factor that the exponential takes with it (unit_of), in units of log2; first: distance of the lane's first key
template <int MOD> __device__ __forceinline__ float unit_of(const ScoreForm& sf) { return MOD == 0 ? sf.f : MOD == CAPPED ? sf.cap2 : 1.f; }
template <bool F32, int MOD, class S> __device__ __forceinline__ void final_scores(const CachedAttn& a, const ScoreForm& sf, float first, S& s) {
  if constexpr (F32 && (MOD & CAPPED)) {
#pragma unroll
    for (int e = 0; e < 16; e++) s[e] = tanhf(s[e] * sf.x1);
  } else {
    // The second way of tanh_scores is off by 2^-22 of the CAP: a quarter of a unit at 10^6, in a tile's scores of order one as well.  Past 4096, of which that
    // is 2^-10, only scores of at least 0.66 of the cap go it, so that errors are within 2^-21 of each score.
    tanh_scores<MOD, true, true>(sf, s, a.cap > 4096.f);
  }
  if constexpr (MOD & BIASED) {
    float keep;
#pragma unroll
    for (int e = 0; e < 16; e++) s[e] = final_score<MOD>(sf, s[e], first - (float)e, &keep);
  }
}
__device__ __forceinline__ ScoreForm form_of(const CachedAttn& a, int h, bool ok) {
  ScoreForm sf;
  sf.f = a.scale * LOG2E;
  sf.x1 = a.cap > 0.f ? a.scale / a.cap : 0.f;
  sf.cap2 = a.cap * LOG2E;
  sf.slope2 = a.slopes && ok ? a.slopes[h] * LOG2E : 0.f;
  return sf;
}
// a column's numbers of 16 tokens, of which `keep` are there: what lies behind the last token, or on no page, may be anything
__device__ __forceinline__ uint4 first_tokens(uint4 v, int keep) {
  unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int u = 0; u < 4; u++) { const int b = min(max(keep - 4 * u, 0), 4); w[u] &= b == 4 ? ~0u : (1u << (8 * b)) - 1u; }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// ---- few rows: 16 per workgroup, NW waves share the keys out in tiles of 64, and put their results together in LDS ----
// Bound by reading the cache, where it is long.  A tile's keys are asked for when the last one's have been multiplied, its values likewise, and the
// pages two tiles ahead; the SIMD's other waves (two of them up to 64 columns, one up to 128) hide the rest.  Tiles of 64 keys rather than 32: a wave's
// softmax statistics, reductions over lanes and waits come half as often.
template <int DHP, int NW> constexpr unsigned FEW_SMEM = NW * (DHP * 16 + 32) * 4 + 16;
template <int DHP, bool WHOLE, bool F32, int MOD, int NW>
__device__ __forceinline__ void few_rows(const CachedAttn& a, const Item& x, float* smem) {
  typedef typename std::conditional<F32, float, bf16>::type T;
  constexpr int KT = DHP / 64, DT = DHP / 16, Q = F32 ? 3 : 1;
  const CacheView& c = a.c;
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, col = lane & 15, lg = c.lg, P1 = (1 << lg) - 1;
  const int dh = WHOLE ? DHP : c.dh;
  const int rest = x.at / c.Hkv, kh = x.at - rest * c.Hkv, split = rest / x.w.groups, group = rest - split * x.w.groups;

  const int r = group * 16 + col, qi = r / a.G, i = x.w.row0 + qi, h = kh * a.G + (r - qi * a.G), pos = x.w.start + qi;
  const bool ok = qi < x.w.n;
  int2 sees = ok ? seen_from(a, pos, x.w.end) : make_int2(0, 0);
  if (sees.x == sees.y) sees = make_int2(INT_MAX, 0);
  const int first = wave_imin(sees.x), last = wave_imax(sees.y);
  const int all_from = wave_imax(ok ? sees.x : 0), all_to = wave_imin(ok ? sees.y : INT_MAX);
  // this wave's tiles: t0, t0 + NW, .. below t1 (of 64 keys, counted from the sequence's first)
  int t0 = 0, t1 = 0;
  if (first < last) {
    const int a0 = first >> 6, n = ((last - 1) >> 6) - a0 + 1, per = (n + x.splits - 1) / x.splits;
    t0 = a0 + min(split * per, n);
    t1 = min(t0 + per, a0 + n);
  }
  t0 += wv;

  // where a lane's keys and values of a tile lie: token 16 gk + .. of the keys, 16 g + .. of the values
  const int gk = col >> 2;
  // (of any t; what lies behind the last token is no page, whatever its unit may be)
  auto page_of = [&](int t, int group) { const int j = t * 64 + group * 16, p = cache_page(c, x.s, j >> lg); return j < x.w.end ? p : -1; };
  int pk = page_of(t0, gk), pv = page_of(t0, g);
  uint4 k[4][KT], v[DT];
  float ks, vs;
  auto fetch_k = [&](int t, int page) {
    const i64 block = cache_block(c, max(page, 0), kh);
    ks = c.ks[block];
    const unsigned char* p = c.k + ((block << lg) + ((t * 64 + gk * 16) & P1) + (col & 3)) * dh;
    // (columns past the width read others, which meet zeros of q)
#pragma unroll
    for (int b = 0; b < 4; b++)
#pragma unroll
      for (int u = 0; u < KT; u++) k[b][u] = *(const uint4*)(p + 4 * b * dh + (WHOLE || 64 * u + 16 * g < dh ? 64 * u + 16 * g : 0));
  };
  auto fetch_v = [&](int t, int page) {
    const i64 block = cache_block(c, max(page, 0), kh);
    vs = c.vs[block];
    const unsigned char* p = c.v + ((block << lg) + ((t * 64 + g * 16) & P1)) * dh;
#pragma unroll
    for (int d = 0; d < DT; d++) v[d] = *(const uint4*)(p + 16 * (WHOLE || 16 * d + col < dh ? 16 * d + col : 0));
  };
  bf16x8 qf[KT][Q][2];
#pragma unroll
  for (int t = 0; t < KT; t++) load_q16<T, Q>((const T*)a.q + (i64)i * a.ldq + (i64)h * dh + 64 * t + 16 * g, ok && (WHOLE || 64 * t + 16 * g < dh), qf[t]);
  const ScoreForm sf = form_of(a, h, ok);
  const float unit = unit_of<MOD>(sf);

  f32x4 acc[DT];
#pragma unroll
  for (int d = 0; d < DT; d++) acc[d] = f32x4{};
  float m = -INFINITY, l = 0.f;
  if (t0 < t1) { fetch_k(t0, pk); fetch_v(t0, pv); }
  int nk = page_of(t0 + NW, gk), nv = page_of(t0 + NW, g);
  for (int t = t0; t < t1; t += NW) {
    const int kv = t * 64;
    f32x16 s;
#pragma unroll
    for (int b = 0; b < 4; b++) {
      f32x4 z = {};
#pragma unroll
      for (int u = 0; u < KT; u++) {
        const bf16x8 k0 = eight(k[b][u].x, k[b][u].y, ks), k1 = eight(k[b][u].z, k[b][u].w, ks);
#pragma unroll
        for (int p = 0; p < Q; p++) { z = mfma16(k0, qf[u][p][0], z); z = mfma16(k1, qf[u][p][1], z); }
      }
#pragma unroll
      for (int e = 0; e < 4; e++) s[4 * b + e] = z[e];
    }
    const bool more = t + NW < t1;
    const int vp = pv;
    if (more) fetch_k(t + NW, nk);
    final_scores<F32, MOD>(a, sf, (float)(pos - kv - 16 * g), s);
    const bool bad = vp < 0, any_bad = __any(bad);
    if (kv < all_from || kv + 64 > all_to || any_bad) {
      const int lo = max(sees.x, kv) - kv - 16 * g;
      const unsigned n = (unsigned)max(min(sees.y, kv + 64) - max(sees.x, kv), 0);
#pragma unroll
      for (int e = 0; e < 16; e++) if ((unsigned)(e - lo) >= n || bad) s[e] = -INFINITY;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int e = 0; e < 16; e += 2) mx = fmaxf(fmaxf(mx, s[e]), s[e + 1]);
    const float top = quarters_max(mx) * unit;
    if (__any(top > m + HEADROOM)) {
      const float mn = fmaxf(m, top), alpha = fast_exp2(m - (mn == -INFINITY ? 0.f : mn));
      l *= alpha;
#pragma unroll
      for (int d = 0; d < DT; d++) acc[d] *= alpha;
      m = mn;
    }
    const float ms = m == -INFINITY ? 0.f : m;
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 16; e++) { s[e] = fast_exp2(MOD & BIASED ? s[e] - ms : fmaf(s[e], unit, -ms)); sum += s[e]; }
    l += sum;
    bf16x8 pf[Q][2];
#pragma unroll
    for (int p = 0; p < Q; p++) {
      pf[p][0] = acc_to_frag(s, 0);
      pf[p][1] = acc_to_frag(s, 1);
#pragma unroll
      for (int e = 0; e < 16; e++) s[e] -= (float)pf[p][e >> 3][e & 7];
    }
    if (kv + 64 > x.w.end || any_bad) {
      const int keep = bad ? 0 : x.w.end - kv - 16 * g;
      vs = bad ? 1.f : vs;
#pragma unroll
      for (int d = 0; d < DT; d++) v[d] = first_tokens(v[d], keep);
    }
#pragma unroll
    for (int d = 0; d < DT; d++) {
      const bf16x8 v0 = eight(v[d].x, v[d].y, vs), v1 = eight(v[d].z, v[d].w, vs);
#pragma unroll
      for (int p = 0; p < Q; p++) { acc[d] = mfma16(v0, pf[p][0], acc[d]); acc[d] = mfma16(v1, pf[p][1], acc[d]); }
    }
    if (more) fetch_v(t + NW, nv);
    pv = nv;
    nk = page_of(t + 2 * NW, gk);
    nv = page_of(t + 2 * NW, g);
  }
  l = quarters_sum(l);

  // the waves' maxima and sums, then their results in units of the common maximum: [wave][16 columns' block][lane]
  float* ml = smem + NW * DHP * 16;                  // [wave][maximum, sum][16 rows]
  unsigned* odd = (unsigned*)(ml + NW * 32);
  if (lane < 16) { ml[wv * 32 + lane] = m; ml[wv * 32 + 16 + lane] = l; }
  if (threadIdx.x == 0) *odd = 0;
  __syncthreads();
  float M = -INFINITY, tot = 0.f;
#pragma unroll
  for (int w = 0; w < NW; w++) M = fmaxf(M, ml[w * 32 + col]);
  const float Ms = M == -INFINITY ? 0.f : M, mine = fast_exp2(m - Ms);
#pragma unroll
  for (int w = 0; w < NW; w++) tot = fmaf(fast_exp2(ml[w * 32 + col] - Ms), ml[w * 32 + 16 + col], tot);
  float4* part = (float4*)smem;
#pragma unroll
  for (int d = 0; d < DT; d++) part[(wv * DT + d) * 64 + lane] = make_float4(acc[d][0] * mine, acc[d][1] * mine, acc[d][2] * mine, acc[d][3] * mine);
  __syncthreads();
  const float inv = tot == 0.f ? 0.f : 1.f / tot;
  const i64 slot = x.slot + x.at;
  bool bad = false;
#pragma unroll
  for (int d = wv; d < DT; d += NW) {                // (a thread's row is its lane's)
    float4 z = part[d * 64 + lane];
#pragma unroll
    for (int w = 1; w < NW; w++) { const float4 y = part[(w * DT + d) * 64 + lane]; z.x += y.x; z.y += y.y; z.z += y.z; z.w += y.w; }
    const int at = 16 * d + 4 * g;
    if (x.splits > 1) {
      if (ok && slot < a.slots) *(float4*)(a.parts + (slot * 16 + col) * DHP + at) = z;
    } else if (ok && (WHOLE || at < dh)) {
      bad = bad || !(fmaf(z.x, 0.f, fmaf(z.y, 0.f, fmaf(z.z, 0.f, z.w * 0.f))) == 0.f);
      typedef __attribute__((ext_vector_type(4))) T V4;
      V4 o;
      o[0] = from_f<T>(z.x * inv); o[1] = from_f<T>(z.y * inv); o[2] = from_f<T>(z.z * inv); o[3] = from_f<T>(z.w * inv);
      *(V4*)((T*)a.out + (i64)i * a.ldo + (i64)h * dh + at) = o;
    }
  }
  if (x.splits > 1) {
    if (threadIdx.x < 16 && ok && slot < a.slots) a.stats[slot * 16 + col] = make_float2(M, tot);
    return;
  }
  if (threadIdx.x < 16 && ok && a.lse) a.lse[(i64)h * a.T + i] = tot == 0.f ? -INFINITY : (M + log2f(tot)) * LN2;
  // a value that is not finite: seen by its row, or only multiplied by zero in a tile that it sees a part of?
  unsigned long long b = __ballot(bad);
  if (b) { b |= b >> 32; b |= b >> 16; if (lane == 0) atomicOr(odd, (unsigned)b & 0xffffu); }
  __syncthreads();
  const unsigned again = *odd;
  if (again)
    for (int n = wv; n < 16; n += NW)
      if ((again >> n) & 1) {
        const int rr = group * 16 + n, qr = rr / a.G;
        cached_row<T>(a, x.s, x.w.row0 + qr, kh * a.G + (rr - qr * a.G), x.w.start + qr, x.w.end, smem + wv * DHP);
      }
}

// ---- many rows: 32 per wave, tiles of 32 keys ----
// Bound by the vector instructions of the softmax and the conversions, and by how many waves a SIMD has to take them from: two at 128 columns (195
// registers), three at 64.  4096 rows of 32 heads to 8 of 128 columns behind 4096 tokens: 486 to 499 us, 0.85 to 0.83 PFLOP/s.  Each wave converts its tiles for itself: converted
// once for the workgroup, in LDS, 553 us, with the reads a tile ahead 510; queries in LDS, which leaves registers for three waves, 547 us (502 with two):
// more waves find less of each other's tiles in the L1 cache.  A tile's registers are filled again as soon as they are used up; with a second set 525.
// LDS: the parts of three waves, then a row of floats for each
template <int DHP> constexpr int ROWS_AT = 3 * 64 * (DHP / 2 + 2);
template <int DHP> constexpr unsigned MANY_SMEM = (ROWS_AT<DHP> + 4 * DHP) * 4;
// DHP: head width rounded up to 64, 128 or 256.  WHOLE: it is the width.  F32: float32 queries and results.
template <int DHP, bool WHOLE, bool F32, int MOD>
__device__ __forceinline__ void many_rows(const CachedAttn& a, const Item& x, float* smem) {
  typedef typename std::conditional<F32, float, bf16>::type T;
  constexpr int KT = DHP / 32, DT = DHP / 32, Q = F32 ? 3 : 1;
  const CacheView& c = a.c;
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 5, col = lane & 31, lg = c.lg, P1 = (1 << lg) - 1;
  const int dh = WHOLE ? DHP : c.dh;
  const int rest = x.at / c.Hkv, kh = x.at - rest * c.Hkv, split = rest / x.w.groups;
  const int group = x.w.groups - 1 - (rest - split * x.w.groups);      // (late rows see most)
  // of the workgroup's waves those of one block of 32 rows share its keys out
  const int nb = a.lr - 5, kparts = 4 >> nb, kp = wv >> nb, blk = (group << nb) + (wv & ((1 << nb) - 1));

  // this lane's row
  const int r = blk * 32 + col, qi = r / a.G, i = x.w.row0 + qi, h = kh * a.G + (r - qi * a.G), pos = x.w.start + qi;
  const bool ok = qi < x.w.n;
  bf16x8 qf[KT][Q][2];
#pragma unroll
  for (int t = 0; t < KT; t++) load_q16<T, Q>((const T*)a.q + (i64)i * a.ldq + (i64)h * dh + 32 * t + 16 * g, ok && (WHOLE || 32 * t + 16 * g < dh), qf[t]);
  int2 sees = ok ? seen_from(a, pos, x.w.end) : make_int2(0, 0);
  if (sees.x == sees.y) sees = make_int2(INT_MAX, 0);
  const int first = wave_imin(sees.x), last = wave_imax(sees.y);
  const int all_from = wave_imax(ok ? sees.x : 0), all_to = wave_imin(ok ? sees.y : INT_MAX);
  // this wave's tiles: t0 .. t1 - 1 (of 32 keys, counted from the sequence's first)
  int t0 = 0, t1 = 0;
  if (first < last) {
    const int a0 = first >> 5, n = ((last - 1) >> 5) - a0 + 1, all = x.splits * kparts, per = (n + all - 1) / all;
    t0 = a0 + min((split * kparts + kp) * per, n);
    t1 = min(t0 + per, a0 + n);
  }
  const int count = max(t1 - t0, 0);
  const ScoreForm sf = form_of(a, h, ok);
  const float unit = unit_of<MOD>(sf);

  // pages and scales of 64 tiles at a time, one tile per lane: of its first 16 tokens and of its second
  int page0 = 0, page1 = 0;
  float ks0 = 0.f, ks1 = 0.f, vs0 = 0.f, vs1 = 0.f;
  auto look_up = [&](int n) {
    const int kv = (t0 + n + lane) * 32;
    const bool there = n + lane < count;
    page0 = there ? cache_page(c, x.s, kv >> lg) : -1;
    page1 = there && kv + 16 < x.w.end ? cache_page(c, x.s, (kv + 16) >> lg) : -1;      // (behind the last token there is none)
    const i64 b0 = cache_block(c, max(page0, 0), kh), b1 = cache_block(c, max(page1, 0), kh);
    ks0 = c.ks[b0]; ks1 = c.ks[b1]; vs0 = c.vs[b0]; vs1 = c.vs[b1];
  };
  const int tok = 16 * ((col >> 2) & 1) + 4 * (col >> 3) + (col & 3);
  uint4 k[KT], v[DT];
  float ks, vs;
  bool bad;
  // the n-th tile's keys, values; its pages have been looked up.  (Read by all lanes before any chooses: in a branch, a lane that is not in it may be the one
  // that is read.)
  auto fetch_k = [&](int n) {
    const int l = n & 63, kv = (t0 + n) * 32;
    const int p0 = __builtin_amdgcn_readlane(page0, l), p1 = __builtin_amdgcn_readlane(page1, l);
    const float k0 = lane_f(ks0, l), k1 = lane_f(ks1, l);
    const i64 s0 = (cache_block(c, max(p0, 0), kh) << lg) + (kv & P1), s1 = (cache_block(c, max(p1, 0), kh) << lg) + ((kv + 16) & P1);
    ks = tok & 16 ? k1 : k0;
    const unsigned char* p = c.k + ((tok & 16 ? s1 : s0) + (tok & 15)) * dh;
    // (columns past the width read others, which meet zeros of q)
#pragma unroll
    for (int u = 0; u < KT; u++) k[u] = *(const uint4*)(p + (WHOLE || 32 * u + 16 * g < dh ? 32 * u + 16 * g : 0));
  };
  auto fetch_v = [&](int n) {
    const int l = n & 63, kv = (t0 + n) * 32;
    const int p0 = __builtin_amdgcn_readlane(page0, l), p1 = __builtin_amdgcn_readlane(page1, l);
    const float v0 = lane_f(vs0, l), v1 = lane_f(vs1, l);
    const i64 s0 = (cache_block(c, max(p0, 0), kh) << lg) + (kv & P1), s1 = (cache_block(c, max(p1, 0), kh) << lg) + ((kv + 16) & P1);
    bad = g ? p1 < 0 : p0 < 0;
    vs = g ? v1 : v0;
    const unsigned char* p = c.v + (g ? s1 : s0) * dh;
#pragma unroll
    for (int u = 0; u < DT; u++) v[u] = *(const uint4*)(p + 16 * (WHOLE || 32 * u + col < dh ? 32 * u + col : 0));
  };

  f32x16 acc[DT];
#pragma unroll
  for (int d = 0; d < DT; d++) acc[d] = f32x16{};
  float m = -INFINITY, l = 0.f;
  if (count > 0) {
    look_up(0);
    fetch_k(0);
    fetch_v(0);
  }
  for (int n = 0; n < count; n++) {
    const int kv = (t0 + n) * 32;
    f32x16 s = {};
#pragma unroll
    for (int t = 0; t < KT; t++) {
      const bf16x8 k0 = eight(k[t].x, k[t].y, ks), k1 = eight(k[t].z, k[t].w, ks);
#pragma unroll
      for (int p = 0; p < Q; p++) { s = mfma(k0, qf[t][p][0], s); s = mfma(k1, qf[t][p][1], s); }
    }
    // (a 64th tile's pages are looked up when its keys are asked for: its values come behind them, this tile's are here already)
    if (n + 1 < count) {
      if (((n + 1) & 63) == 0) look_up(n + 1);
      fetch_k(n + 1);
    }
    final_scores<F32, MOD>(a, sf, (float)(pos - kv - 16 * g), s);
    const bool any_bad = __any(bad);
    if (kv < all_from || kv + 32 > all_to || any_bad) {
      const int lo = max(sees.x, kv) - kv - 16 * g;
      const unsigned cnt = (unsigned)max(min(sees.y, kv + 32) - max(sees.x, kv), 0);
#pragma unroll
      for (int e = 0; e < 16; e++) if ((unsigned)(e - lo) >= cnt || bad) s[e] = -INFINITY;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int e = 0; e < 16; e += 2) mx = fmaxf(fmaxf(mx, s[e]), s[e + 1]);
    const float top = both_halves_max(mx) * unit;
    if (__any(top > m + HEADROOM)) {
      const float mn = fmaxf(m, top), alpha = fast_exp2(m - (mn == -INFINITY ? 0.f : mn));
      l *= alpha;
#pragma unroll
      for (int d = 0; d < DT; d++) acc[d] *= alpha;
      m = mn;
    }
    const float ms = m == -INFINITY ? 0.f : m;
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 16; e++) { s[e] = fast_exp2(MOD & BIASED ? s[e] - ms : fmaf(s[e], unit, -ms)); sum += s[e]; }
    l += sum;
    bf16x8 pf[Q][2];
#pragma unroll
    for (int p = 0; p < Q; p++) {
      pf[p][0] = acc_to_frag(s, 0);
      pf[p][1] = acc_to_frag(s, 1);
#pragma unroll
      for (int e = 0; e < 16; e++) s[e] -= (float)pf[p][e >> 3][e & 7];
    }
    if (kv + 32 > x.w.end || any_bad) {
      const int keep = bad ? 0 : x.w.end - kv - 16 * g;
      vs = bad ? 1.f : vs;
#pragma unroll
      for (int d = 0; d < DT; d++) v[d] = first_tokens(v[d], keep);
    }
#pragma unroll
    for (int d = 0; d < DT; d++) {
      const bf16x8 v0 = eight(v[d].x, v[d].y, vs), v1 = eight(v[d].z, v[d].w, vs);
#pragma unroll
      for (int p = 0; p < Q; p++) { acc[d] = mfma(v0, pf[p][0], acc[d]); acc[d] = mfma(v1, pf[p][1], acc[d]); }
    }
    if (n + 1 < count) fetch_v(n + 1);
  }
  l = both_halves_sum(l);

  if (kparts > 1) {
    // the waves of a block put their results together
    constexpr int P = DT * 16 + 2;
    float* mine = smem + (wv - (1 << nb)) * (P * 64) + lane;
    if (kp) {
#pragma unroll
      for (int d = 0; d < DT; d++)
#pragma unroll
        for (int e = 0; e < 16; e++) mine[(d * 16 + e) * 64] = acc[d][e];
      mine[(P - 2) * 64] = m;
      mine[(P - 1) * 64] = l;
    }
    __syncthreads();
    if (kp) return;
    for (int k = 1; k < kparts; k++) {
      const float* p = smem + (((k - 1) << nb) + wv) * (P * 64) + lane;
      const float m1 = p[(P - 2) * 64], mn = fmaxf(m, m1), ms = mn == -INFINITY ? 0.f : mn, f0 = fast_exp2(m - ms), f1 = fast_exp2(m1 - ms);
      l = l * f0 + p[(P - 1) * 64] * f1;
      m = mn;
#pragma unroll
      for (int d = 0; d < DT; d++)
#pragma unroll
        for (int e = 0; e < 16; e++) acc[d][e] = fmaf(p[(d * 16 + e) * 64], f1, acc[d][e] * f0);
    }
  }
  if (x.splits > 1) {
    const i64 slot = x.slot + ((i64)x.at << (a.lr - 4)) + wv * 2;                 // (two of 16 rows each, one behind the other)
    if (!ok || slot + 1 >= a.slots) return;
    if (g == 0) a.stats[slot * 16 + col] = make_float2(m, l);
    float* p = a.parts + (slot * 16 + col) * DHP;
#pragma unroll
    for (int d = 0; d < DT; d++)
#pragma unroll
      for (int e = 0; e < 16; e += 4)
        *(float4*)(p + d * 32 + 2 * e + 4 * g) = make_float4(acc[d][e], acc[d][e + 1], acc[d][e + 2], acc[d][e + 3]);
    return;
  }
  // a value that is not finite: seen by its row, or only multiplied by zero in a tile that it sees a part of?
  float z = 0.f;
#pragma unroll
  for (int d = 0; d < DT; d++)
#pragma unroll
    for (int e = 0; e < 16; e++) z = fmaf(acc[d][e], 0.f, z);
  unsigned long long odd = __ballot(ok && z != 0.f);
  const unsigned again = (unsigned)odd | (unsigned)(odd >> 32);
  const float inv = l == 0.f ? 0.f : 1.f / l;
  if (ok) {
    T* o = (T*)a.out + (i64)i * a.ldo + (i64)h * dh;
#pragma unroll
    for (int d = 0; d < DT; d++)
#pragma unroll
      for (int e = 0; e < 16; e += 4)
        if (WHOLE || d * 32 + 2 * e + 4 * g < dh) {
          typedef __attribute__((ext_vector_type(4))) T V4;
          V4 v;
#pragma unroll
          for (int u = 0; u < 4; u++) v[u] = from_f<T>(acc[d][e + u] * inv);
          *(V4*)(o + d * 32 + 2 * e + 4 * g) = v;
        }
    if (g == 0 && a.lse) a.lse[(i64)h * a.T + i] = l == 0.f ? -INFINITY : (m + log2f(l)) * LN2;
  }
  if (again)
    for (int b = 0; b < 32; b++)
      if ((again >> b) & 1) {
        const int rr = blk * 32 + b, qr = rr / a.G;
        cached_row<T>(a, x.s, x.w.row0 + qr, kh * a.G + (rr - qr * a.G), x.w.start + qr, x.w.end, smem + ROWS_AT<DHP> + wv * DHP);
      }
}

template <int DHP, bool WHOLE, bool F32, int MOD>
__global__ void __launch_bounds__(256, DHP == 256 || F32 ? 1 : DHP == 128 ? 2 : 3) cached_attn_k(CachedAttn a) {
  extern __shared__ __attribute__((aligned(16))) float smem[];
  Item x;
  if (!find<false>(a, (int)blockIdx.x, &x)) return;
  if (x.w.few) few_rows<DHP, WHOLE, F32, MOD, 4>(a, x, smem);
  else many_rows<DHP, WHOLE, F32, MOD>(a, x, smem);
}
template <int DHP, bool WHOLE, bool F32, int MOD, int NW>
__global__ void __launch_bounds__(NW * 64, DHP == 256 || F32 ? 1 : DHP == 64 ? 3 : 2) cached_few_k(CachedAttn a) {
  extern __shared__ __attribute__((aligned(16))) float smem[];
  Item x;
  if (find<false>(a, (int)blockIdx.x, &x)) few_rows<DHP, WHOLE, F32, MOD, NW>(a, x, smem);
}

// Joins the parts of split groups, a wave per row
template <class T, int DHP> __global__ void __launch_bounds__(256) cached_join_k(CachedAttn a) {
  __shared__ float lds[4][DHP];
  constexpr int C = DHP / 64;
  Item x;
  if (!find<true>(a, (int)blockIdx.x, &x)) return;
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), Hkv = a.c.Hkv, dh = a.c.dh;
  const int quad = x.at / Hkv, kh = x.at - quad * Hkv, rr = quad * 4 + wv, qi = rr / a.G;
  if (qi >= x.w.n) return;
  // of the list of workgroups that made the parts: the row's group, and which of its slots and rows
  const int lrows = x.w.few ? 4 : a.lr, slots = 1 << (lrows - 4), g0 = rr >> lrows, group = x.w.few ? g0 : x.w.groups - 1 - g0, in = rr & ((1 << lrows) - 1);
  if (x.slot + (i64)x.splits * x.w.groups * Hkv * slots > a.slots) return;
  const int i = x.w.row0 + qi, h = kh * a.G + (rr - qi * a.G);
  {
    auto part = [&](int split) {
      const i64 at = ((i64)split * x.w.groups + group) * Hkv + kh;
      return (x.slot + at * slots) * 16 + in;
    };
    const float2 st = lane < x.splits ? a.stats[part(lane)] : make_float2(-INFINITY, 0.f);
    float p[16][C];
    auto load = [&](int k0) {
#pragma unroll
      for (int k = 0; k < 16; k++)
#pragma unroll
        for (int u = 0; u < C; u++) p[k][u] = k0 + k < x.splits ? a.parts[part(k0 + k) * DHP + lane * C + u] : 0.f;
    };
    load(0);                                         // (on their way with the statistics)
    const float M = wave_max(st.x), Ms = M == -INFINITY ? 0.f : M;
    const float w = st.y == 0.f ? 0.f : exp2f(st.x - Ms);
    const float tot = wave_sum(w * st.y);
    float v[C] = {};
    for (int k0 = 0; k0 < x.splits; k0 += 16) {
      if (k0) load(k0);
#pragma unroll
      for (int k = 0; k < 16; k++) {
        const float f = lane_f(w, (k0 + k) & 63);    // (0 behind the last)
#pragma unroll
        for (int u = 0; u < C; u++) v[u] = fmaf(f, p[k][u], v[u]);
      }
    }
    float z = 0.f;
#pragma unroll
    for (int u = 0; u < C; u++) z = fmaf(v[u], 0.f, z);
    if (!__all(z == 0.f)) {
      cached_row<T>(a, x.s, i, h, x.w.start + qi, x.w.end, lds[wv]);
      return;
    }
    const float inv = tot == 0.f ? 0.f : 1.f / tot;
    T* o = (T*)a.out + (i64)i * a.ldo + (i64)h * dh;
#pragma unroll
    for (int u = 0; u < C; u++) if (lane * C + u < dh) o[lane * C + u] = from_f<T>(v[u] * inv);
    if (lane == 0 && a.lse) a.lse[(i64)h * a.T + i] = tot == 0.f ? -INFINITY : (M + log2f(tot)) * LN2;
  }
}

// Most groups that a call can have
i64 most_groups(const CachedAttn& a) {
  const i64 rows = (i64)a.T * a.G, seqs = a.c.n_seqs < a.T ? a.c.n_seqs : a.T;
  const i64 by_row = rows / 16 + seqs, by_seq = (rows >> a.lr) + (FEW_ROWS / 16) * seqs;
  return a.few_only || by_row < by_seq ? by_row : by_seq;
}
int padded(int dh) { return dh <= 64 ? 64 : dh <= 128 ? 128 : 256; }
i64 most_slots(const CachedAttn& a) {
  return a.split ? (most_groups(a) * a.c.Hkv + a.target) * (a.split == 2 && !a.few_only ? 1 << (a.lr - 4) : 1) : 0;
}

template <class K> void launch(K kernel, std::atomic<unsigned long long>& attr_mask, i64 grid, int block, unsigned smem, const CachedAttn& a, hipStream_t s) {
  if (smem > 65536 && attr_needed(attr_mask)) {
    (void)hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    attr_done(attr_mask);
  }
  hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(block), smem, s, a);
}
template <int DHP, bool WHOLE, bool F32, int MOD> void go(const CachedAttn& a, hipStream_t s) {
  static std::atomic<unsigned long long> mask[3];
  const i64 grid = most_groups(a) * a.c.Hkv + (a.split ? a.target : 0);
  if (!a.few_only) launch(cached_attn_k<DHP, WHOLE, F32, MOD>, mask[0], grid, 256, MANY_SMEM<DHP>, a, s);      // (more than the form for few rows takes)
  else {
    // eight waves where nothing is split, if their registers allow it
    constexpr int NW = DHP == 256 || F32 ? 4 : 8;
    if (a.split || most_groups(a) * a.c.Hkv >= 256) launch(cached_few_k<DHP, WHOLE, F32, MOD, 4>, mask[1], grid, 256, FEW_SMEM<DHP, 4>, a, s);
    else launch(cached_few_k<DHP, WHOLE, F32, MOD, NW>, mask[2], grid, NW * 64, FEW_SMEM<DHP, NW>, a, s);
  }
  if (!a.split) return;
  const i64 rows = (i64)a.T * a.G, seqs = a.c.n_seqs < a.T ? a.c.n_seqs : a.T, few = (i64)FEW_ROWS * seqs;
  const i64 joined = a.few_only || a.split == 2 || rows < few ? rows : few;      // rows that may have been split
  typedef typename std::conditional<F32, float, bf16>::type T;
  hipLaunchKernelGGL((cached_join_k<T, DHP>), dim3((unsigned)((joined / 4 + seqs) * a.c.Hkv)), dim3(256), 0, s, a);
}
template <int DHP, bool F32> void go(const CachedAttn& a, hipStream_t s) {
  // (without a part of the score's form its kernel has no instructions of it; a scale that is not positive is multiplied, not put into the exponential)
  const int mod = (a.cap > 0.f ? CAPPED : 0) | (a.slopes || !(a.scale > 0.f) ? BIASED : 0);
  auto pick = [&](auto whole) {
    constexpr bool WHOLE = decltype(whole)::value;
    if (mod == 0) go<DHP, WHOLE, F32, 0>(a, s);
    else if (mod == CAPPED) go<DHP, WHOLE, F32, CAPPED>(a, s);
    else if (mod == BIASED) go<DHP, WHOLE, F32, BIASED>(a, s);
    else go<DHP, WHOLE, F32, CAPPED | BIASED>(a, s);
  };
  if (a.c.dh == DHP) pick(std::true_type{}); else pick(std::false_type{});
}

}  // namespace

// What the sizes alone say.  One row per sequence, or few in all: the form for few rows throughout.  Splitting its keys takes a second launch (4 us and
// more), and gives work to CUs that have none: a workgroup with a CU to itself takes 3 us for 512 tokens.  Without, with, 8 sequences of 4 key heads of 128, us:
// 512 tokens 8.2, 10.6; 1024 10.9, 10.1; 2048 17.8, 12.5.  Where there is a workgroup for every CU anyway it only evens out lengths.  Prompts' keys are split
// where there are fewer.
// A prompt's workgroup takes 32, 64 or 128 rows, and its four waves a quarter, half or all of their keys each: the fewer rows there are, the more workgroups
// they make.  32 heads of 128 over 8, 32, 64, 128 rows, us: 512 tokens 15.8, 16.3, 31.1; 512 behind 3000 46.8, 53.7, 63.5; 2048 behind 3000 184, 173, 182;
// 4096 behind 3000 426, 404, 396.  The same of 64: 11.5, 13.4, 24.9; 34.3, 46.4, 51.1; 109, 111, 131; 249, 241, 258.
void cached_attn_plan(CachedAttn* a) {
  // the workgroups that bfloat16's form for few rows has on the CUs together: four, two, one on each.  (Of those with fewer, three for
  // most for many rows at 64 columns, in float32 half as many, some wait for others to end.)
  a->target = a->c.dh <= 64 ? 1024 : a->c.dh <= 128 ? 512 : 256;
  const i64 blocks = ((i64)a->T * a->H) >> 7;        // workgroups of 128 rows
  a->lr = 4 * blocks <= a->target ? 5 : 2 * blocks <= 3 * (i64)a->target ? 6 : 7;
  a->few_only = (i64)a->T * a->G <= FEW_ROWS || a->T <= a->c.n_seqs;
  const i64 room = (i64)a->c.max_pages << a->c.lg, groups = most_groups(*a) * a->c.Hkv;
  a->split = a->few_only && room <= (groups < 256 ? 768 : 2048) ? 0 : groups < 256 ? 2 : 1;
}
size_t cached_attn_bytes(const CachedAttn& a) { return (size_t)most_slots(a) * 16 * (padded(a.c.dh) * 4 + 8); }
bool cached_attn_takes(const CachedAttn& a) {
  const int es = a.dt == 0 ? 4 : 2;
  return (a.dt == 1 || a.c.dh <= 128) && (a.ldq | a.ldo) * es % 16 == 0 && ((uintptr_t)a.q | (uintptr_t)a.out) % 16 == 0;
}
void launch_cached_attn(CachedAttn a, void* work, bool rows, hipStream_t s) {
  if (a.T < 1 || a.c.n_seqs < 1) return;
  if (rows) {
    const dim3 grid((unsigned)cdiv((i64)a.T * a.H, 4));
    if (a.dt == 0) hipLaunchKernelGGL((cached_rows_k<float>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((cached_rows_k<bf16>), grid, dim3(256), 0, s, a);
    return;
  }
  a.slots = most_slots(a);
  a.parts = (float*)work;
  a.stats = (float2*)(a.parts + a.slots * 16 * padded(a.c.dh));
  const int w = padded(a.c.dh);
  if (a.dt == 0) { if (w == 64) go<64, true>(a, s); else go<128, true>(a, s); }
  else { if (w == 64) go<64, false>(a, s); else if (w == 128) go<128, false>(a, s); else go<256, false>(a, s); }
}
