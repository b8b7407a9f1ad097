// Attention over key ranges on the matrix cores: bf16, heads of up to 128 columns (a multiple of 8).
// Rounding.  Scores, maxima, sums and accumulators are float32.  Probabilities (P) and score gradients (dS) are rounded to bf16 where they become
// operands of the second products, which is what the matrix cores take at full rate; two numbers per value, 16 bits, would double those products (dq with a
// bias does it, see range_bwd_dq_k).  Root mean square errors against 64 bits as multiples of a single rounding's: o 1.2, gradients 1.4 (short documents
// 1.5); row by row, with P and dS in float32, 1.0 and 1.1 to 1.25.
#include "attn_range_tiles.h"
#include "attn_range_few.h"

// Two workgroups fit on a CU: where the whole grid is resident at once, workgroups i and i + 256 share one, so the second 256 take the
// tiles in the other order, and a long tile shares its CU with a short one.
__device__ __forceinline__ int paired(int tile, int tiles, int per_tile) {
  const int first = 256 / per_tile;
  return (int)gridDim.x <= 512 && tile >= first ? tiles - 1 - (tile - first) : tile;
}
// Which tile a workgroup takes (1-D grid of tiles x heads).  Heads are the fastest index, and those that share a key head follow each
// other 8 apart where there are 8 key heads or more, so that they run on the same XCD (id & 7) and find its keys in that L2.
__device__ __forceinline__ void place(const RangeAttn& a, int* tile, int* h) {
  const int row = (int)blockIdx.x / a.H, r = (int)blockIdx.x - row * a.H;
  *tile = paired(row, (a.Tq + 127) / 128, a.H);
  *h = (r % a.Hkv) * a.G + r / a.Hkv;
}

// The keys that 128 queries see: from the first to the last, and whether there may be keys between that none sees (neighbouring
// queries' ranges that don't touch, or a query without any)
struct QueryRanges { int first, end; bool gaps; };
struct TwoRanges { int2 r0, r1; };                  // of queries q0 + lane, q0 + 64 + lane (none: lo = INT_MAX, hi = 0)
__device__ __forceinline__ TwoRanges two_ranges(const RangeAttn& a, int q0, int rows, int keys) {
  const int lane = (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
  TwoRanges t;
  const int2 none = make_int2(INT_MAX, 0), s0 = stored_range(a, q0 + lane), s1 = stored_range(a, q0 + 64 + lane);
  t.r0 = q0 + lane < rows ? clamped(s0, keys) : none;
  t.r1 = q0 + 64 + lane < rows ? clamped(s1, keys) : none;
  if (t.r0.x == t.r0.y) t.r0 = none;
  if (t.r1.x == t.r1.y) t.r1 = none;
  return t;
}
__device__ __forceinline__ QueryRanges query_ranges(const TwoRanges& t, int q0, int rows, int lane) {
  QueryRanges q;
  q.first = wave_imin(min(t.r0.x, t.r1.x));
  q.end = wave_imax(max(t.r0.y, t.r1.y));
  auto apart = [](int2 u, int2 v) { return max(u.x, v.x) > min(u.y, v.y); };
  const int2 over = make_int2(__builtin_amdgcn_readfirstlane(t.r1.x), __builtin_amdgcn_readfirstlane(t.r1.y));
  int2 n0 = make_int2(__shfl_down(t.r0.x, 1, WAVE), __shfl_down(t.r0.y, 1, WAVE)), n1 = make_int2(__shfl_down(t.r1.x, 1, WAVE), __shfl_down(t.r1.y, 1, WAVE));
  if (lane == 63) n0 = over;
  q.gaps = __any((q0 + lane + 1 < rows && apart(t.r0, n0)) || (lane < 63 && q0 + 64 + lane + 1 < rows && apart(t.r1, n1)));
  return q;
}
// where the first tile of 64 keys starts, at or after kv, that some query sees; `end`: there is none.  (The ranges are read again: they are
// not worth four registers in the loops.)
__device__ __forceinline__ int live_from(const QueryRanges& q, int kv, int q0, int rows, int keys) {
  if (kv >= q.end) return q.end;
  if (!q.gaps) return kv;
  const TwoRanges t = two_ranges(args_again(), q0, rows, keys);
  if (__any((t.r0.x < kv + 64 && t.r0.y > kv) || (t.r1.x < kv + 64 && t.r1.y > kv))) return kv;
  return min(wave_imin(min(t.r0.y > kv ? t.r0.x : INT_MAX, t.r1.y > kv ? t.r1.x : INT_MAX)), q.end);
}

// ------------------------------------------------------------------------------------
// Forward.  Workgroup = 128 queries of one head, wave = 32 queries; keys and values streamed in tiles of 64 from the first key
// that some query sees to the last, tiles that none sees left out; K two tiles ahead and V one.  An iteration is two phases with a
// barrier behind each: in the first a wave takes the maximum and half of the exponentials and reads the next tile's key
// fragments, in the second it multiplies those and P V of this tile, with the other half of the exponentials between.
// Bound by the matrix pipe and the exponentials by turns, 1.2 us per tile of 128 x 64 on a full CU, 1.8 alone: one document of 8192 rows, 16
// heads of 128: 303 us, 0.9 PFLOP/s; 16 documents of 512: 56 us.
// ------------------------------------------------------------------------------------
template <int DHP, int MOD>
__global__ void __launch_bounds__(256, 2) range_fwd_k(RangeAttn a) {
  typedef Tiles<DHP> T;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem_raw[];      // K, V, K, V
  int qt, h;
  place(a, &qt, &h);
  qt = (a.Tq + 127) / 128 - 1 - qt;                 // late query tiles tend to be the long ones
  const int rows = rows_in_use(a), keys = keys_in_use(a), q0 = qt * 128;
  if (q0 >= rows) return;
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 5;
  const int myq = q0 + wv * 32 + (lane & 31), kh = h / a.G;
  const QueryRanges qr = query_ranges(two_ranges(a, q0, rows, keys), q0, rows, lane);
  const int2 mine = myq < rows ? key_range(a, myq, keys) : make_int2(INT_MIN, INT_MAX);    // (a row that is not there needs no mask)
  const int all_from = wave_imax(mine.x), all_to = wave_imin(mine.y);                      // every query sees the keys between
  const ScoreForm sf = score_form(a, h);
  const int at = MOD & BIASED ? (a.at ? a.at[min(myq, rows - 1)] : myq) : 0;

  bf16x8 qf[T::KK];
  T::load_frags((const bf16*)a.q + (i64)myq * a.ldq + (i64)h * a.dh, myq < rows, a.dh, g, qf);
  const HeadRows rk = {(const unsigned char*)a.k + (i64)kh * a.dh * 2, a.ldk * 2, a.dh * 2}, rv = {(const unsigned char*)a.v + (i64)kh * a.dh * 2, a.ldv * 2, a.dh * 2};
  const unsigned lds0 = lds_address(smem_raw) + (unsigned)wv * (T::BYTES / 4);
  auto issue = [&](const HeadRows& r, int kv, unsigned stage) {             // 16 of the tile's rows
    T::load16(rows_buffer(r, kv, min(64, qr.end - kv)), (unsigned)r.ldb, r.width, wv * 16, lds0 + stage * T::BYTES);
  };
  const unsigned rbase = T::row_base(lane), cbase = T::col_base(lane);
  f32x16 oacc[T::DT] = {}, s[2];
  bf16x8 kf[2 * T::KK], pf[4];
  float m = -INFINITY, l = 0.f;
  bool partly = false;                              // some tile was not seen whole: what the rest of it holds was multiplied by zero
  auto read_k = [&](unsigned stage, int from) {     // half of K of a tile
    const unsigned char* cK = smem_raw + stage * T::BYTES;
#pragma unroll
    for (int kk = from; kk < from + T::KK / 2; kk++)
#pragma unroll
      for (int j = 0; j < 2; j++) kf[kk * 2 + j] = *(const bf16x8*)(cK + j * 32 * T::ROW + (rbase ^ (unsigned)(kk * 32)));
  };
  auto times_q = [&]() {
    s[0] = f32x16{};
    s[1] = f32x16{};
#pragma unroll
    for (int kk = 0; kk < T::KK; kk++)
#pragma unroll
      for (int j = 0; j < 2; j++) s[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[kk * 2 + j], qf[kk], s[j], 0, 0, 0);
  };
  // scores to their final form in units of log2 (MOD), and those of keys that are not seen to -infinity
  auto finish = [&](int kv) {
    if constexpr (MOD != 0) {
      const float d0 = (float)(at - kv - g * 4);
      float keep;
      tanh_scores<MOD, true>(sf, s[0]);
      tanh_scores<MOD, true>(sf, s[1]);
#pragma unroll
      for (int j = 0; j < 2; j++)
#pragma unroll
        for (int e = 0; e < 16; e++) s[j][e] = final_score<MOD>(sf, s[j][e], d0 - (float)(j * 32 + (e >> 2) * 8 + (e & 3)), &keep);
    }
    if (kv < all_from || kv + 64 > all_to) {
      partly = true;
      const int lo = max(mine.x, kv) - kv - g * 4;
      const unsigned n = (unsigned)max(min(mine.y, kv + 64) - max(mine.x, kv), 0);
#pragma unroll
      for (int j = 0; j < 2; j++)
#pragma unroll
        for (int e = 0; e < 16; e++)
          if ((unsigned)(j * 32 + (e >> 2) * 8 + (e & 3) - lo) >= n) s[j][e] = -INFINITY;
    }
  };
  const float unit = MOD != 0 ? 1.f : sf.f;              // (without MOD the scale is positive and goes into the exponential)
  float ms = 0.f;
  auto exponentials = [&](f32x16 x, int half) {
    float rs[2] = {};
#pragma unroll
    for (int e = 0; e < 16; e++) {
      x[e] = fast_exp2(MOD != 0 ? x[e] - ms : fmaf(x[e], unit, -ms));
      rs[e & 1] += x[e];
    }
    l += rs[0] + rs[1];
    pf[half * 2] = acc_to_frag(x, 0);
    pf[half * 2 + 1] = acc_to_frag(x, 1);
  };
  if (qr.first < qr.end) {
    int kv = qr.first, kv1 = live_from(qr, kv + 64, q0, rows, keys), kv2;                    // this tile, the next one, the one after
    issue(rk, kv, 0); issue(rk, kv1, 2); issue(rv, kv, 1);
    T::arrived(qf);
    wait_vmcnt<2 * T::LOADS>();                     // the first keys
    phase_end();
    read_k(0, 0);
    read_k(0, T::KK / 2);
    times_q();
    wait_vmcnt<T::LOADS>();                         // K of the next tile is there, V of this one may be on its way
    phase_end();
    // the keys read in the phase before and the values just read make room
    auto softmax = [&](unsigned st) {
      kv2 = live_from(qr, kv1 + 64, q0, rows, keys);
      issue(rk, kv2, st);
      issue(rv, kv1, st ^ 2u ^ 1u);
      read_k(st ^ 2u, 0);
      finish(kv);
      float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
      for (int e = 0; e < 32; e += 2) mx[(e >> 1) & 3] = fmaxf(fmaxf(mx[(e >> 1) & 3], s[e >> 4][e & 15]), s[e >> 4][(e & 15) + 1]);
      const float mn = fmaxf(m, both_halves_max(fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]))) * unit);
      if (__any(mn > m)) {                          // the accumulator is rescaled only when some query of the wave has raised its maximum
        const float alpha = fast_exp2(m - (mn == -INFINITY ? 0.f : mn));
        l *= alpha;
#pragma unroll
        for (int d = 0; d < T::DT; d++) oacc[d] *= alpha;
        m = mn;
      }
      read_k(st ^ 2u, T::KK / 2);
      ms = m == -INFINITY ? 0.f : m;
      exponentials(s[0], 0);
      wait_vmcnt<2 * T::LOADS>();                   // V of this tile is there
      phase_end();
    };
    unsigned st = 0;
    while (kv1 < qr.end) {
      softmax(st);
      __builtin_amdgcn_s_setprio(1);
      const f32x16 rest = s[1];
      const unsigned char* cV = smem_raw + (st + 1) * T::BYTES;
      bf16x8 vf[T::DT];
      times_q();
      exponentials(rest, 1);
      T::read_cols(vf, cV, cbase, 0);
      if constexpr (DHP == 128) {
        __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
#pragma unroll
        for (int j = 0; j < 14; j++) {
          __builtin_amdgcn_sched_group_barrier(0x002, 5, 0);
          if (j >= 6) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      T::template cols_times<64>(oacc, cV, cbase, pf, vf);                  // O^T[dh, q] += V^T[dh, kv] P^T[kv, q]
      __builtin_amdgcn_s_setprio(0);
      wait_vmcnt<T::LOADS>();                       // K of the tile after the next is there
      phase_end();
      st ^= 2u;
      kv = kv1;
      kv1 = kv2;
    }
    softmax(st);
    exponentials(s[1], 1);
    const unsigned char* cV = smem_raw + (st + 1) * T::BYTES;
    bf16x8 vf[T::DT];
    T::read_cols(vf, cV, cbase, 0);
    T::template cols_times<64>(oacc, cV, cbase, pf, vf);
    wait_vmcnt<0>();                                // the zero-filled loads past the last tile
    phase_end();
  }
  if (partly && !T::finite(oacc)) {                 // a value that is not finite: seen, or only in a tile with seen ones?
    for (int r = 0; r < 32 && q0 + wv * 32 + r < rows; r++) range_row_fwd<bf16>(args_again(), q0 + wv * 32 + r, h, keys, (float*)smem_raw + wv * 2 * DHP);
    return;
  }
  l = both_halves_sum(l);
  if (myq < rows) {
    const RangeAttn b = args_again();
    T::store((bf16*)b.out + (i64)myq * b.ldo + (i64)h * b.dh, oacc, l == 0.f ? 0.f : 1.0f / l, b.dh, g);
    if (g == 0 && b.lse) b.lse[(i64)h * b.Tq + myq] = l == 0.f ? -INFINITY : (m + __log2f(l)) * LN2;
  }
}

// ------------------------------------------------------------------------------------
// Forward for few rows: 32 rows per workgroup, tiles of 32 keys shared out to the waves, each in LDS of its own that no other wave
// touches, so nothing waits at a barrier until the partial results meet.  A single token's query against a long run of keys
// reads every key and value once, for all heads that share them: that reading bounds it (92800 keys of five sequences, 8 key heads of
// 128: 70 us, 5.4 TB/s, and 4.8 to join).
// Heads of 64 fit four waves to a SIMD if the registers are kept to 128: 4000 rows x 12 heads 65.0 us, 57.2 with four; 128 columns
// have LDS for two only.
// ------------------------------------------------------------------------------------
// a wave's result to its part of LDS, [column][32 rows]
template <int DT> __device__ __forceinline__ void put_partial(float* mine, const f32x16 (&acc)[DT], int lane) {
#pragma unroll
  for (int d = 0; d < DT; d++)
#pragma unroll
    for (int e = 0; e < 16; e++) mine[(d * 32 + (e >> 2) * 8 + (lane >> 5) * 4 + (e & 3)) * 32 + (lane & 31)] = acc[d][e];
}
template <int DHP> constexpr unsigned FEW_SMEM = 4 * Tiles<DHP>::BYTES + 4 * 256;       // the waves' K and V (then their results), statistics
template <int DHP, int MOD>
__global__ void __launch_bounds__(256, DHP == 64 ? 4 : 2) range_fwd_few_k(RangeAttn a, FewShape f) {
  typedef Tiles<DHP> T;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem_raw[];
  int tile, split, head, t0;
  few_place(a, f, (int)blockIdx.x, &tile, &split, &head);
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 5, kh = head % a.Hkv;
  FewRow row = few_row(a, f, tile, head, lane & 31, a.Tq);
  const int2 stored = stored_range(a, row.i);
  const int at = (MOD & BIASED) && row.ok ? (a.at ? a.at[row.i] : row.i) : 0;
  bf16x8 qf[T::KK];
  T::load_frags((const bf16*)a.q + (i64)row.i * a.ldq + (i64)row.h * a.dh, row.ok, a.dh, g, qf);
  const int rows = rows_in_use(a), keys = keys_in_use(a);
  if (tile * f.qpt >= rows) return;
  row.ok = row.ok && row.i < rows;
  const FewKeys fk = few_keys(f, row, stored, split, keys, &t0);
  const ScoreForm sf = score_form(a, row.h);
  const HeadRows rk = {(const unsigned char*)a.k + (i64)kh * a.dh * 2, a.ldk * 2, a.dh * 2}, rv = {(const unsigned char*)a.v + (i64)kh * a.dh * 2, a.ldv * 2, a.dh * 2};
  unsigned char* tK = smem_raw + wv * T::BYTES;      // 32 rows of K, 32 of V
  const unsigned aK = lds_address(smem_raw) + (unsigned)wv * T::BYTES, aV = aK + T::BYTES / 2;
  auto issue = [&](const HeadRows& r, int t, unsigned dst) {
    const int kv = t < fk.t1 ? fk.first + t * 32 : 0, n = t < fk.t1 ? min(32, fk.end - kv) : 0;
    const __amdgpu_buffer_rsrc_t rs = rows_buffer(r, kv, n);
    T::load16(rs, (unsigned)r.ldb, r.width, 0, dst);
    T::load16(rs, (unsigned)r.ldb, r.width, 16, dst + 16 * T::ROW);
  };
  int t = fk.live_from(t0 + wv, 4);
  issue(rk, t, aK);
  issue(rv, t, aV);
  T::arrived(qf);
  const unsigned rbase = T::row_base(lane), cbase = T::col_base(lane);
  f32x16 acc[T::DT] = {};
  float m = -INFINITY, l = 0.f;
  wait_vmcnt<0>();
  while (t < fk.t1) {
    const int kv = fk.first + t * 32, next = fk.live_from(t + 4, 4);
    wait_vmcnt<2 * T::LOADS>();                     // K; V may be on its way
    bf16x8 x[T::KK];
#pragma unroll
    for (int kk = 0; kk < T::KK; kk++) x[kk] = *(const bf16x8*)(tK + (rbase ^ (unsigned)(kk * 32)));
    __builtin_amdgcn_sched_barrier(0);
    f32x16 s = {};
#pragma unroll
    for (int kk = 0; kk < T::KK; kk++) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[kk], qf[kk], s, 0, 0, 0);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    issue(rk, next, aK);
    const float d0 = (float)(at - kv - g * 4);
    const int lo = max(fk.r.x, kv) - kv - g * 4;
    const unsigned n = (unsigned)max(min(fk.r.y, kv + 32) - max(fk.r.x, kv), 0);
    float mx = -INFINITY, keep;
    if constexpr (MOD != 0) {
      tanh_scores<MOD, true>(sf, s);
#pragma unroll
      for (int e = 0; e < 16; e++) s[e] = final_score<MOD>(sf, s[e], d0 - (float)((e >> 2) * 8 + (e & 3)), &keep);
    }
    if (!__all(!row.ok || (fk.r.x <= kv && fk.r.y >= kv + 32))) {
#pragma unroll
      for (int e = 0; e < 16; e++) if ((unsigned)((e >> 2) * 8 + (e & 3) - lo) >= n) s[e] = -INFINITY;
    }
#pragma unroll
    for (int e = 0; e < 16; e += 2) mx = fmaxf(fmaxf(mx, s[e]), s[e + 1]);
    const float unit = MOD != 0 ? 1.f : sf.f;       // (without MOD the scale is positive and goes into the exponential)
    const float mn = fmaxf(m, both_halves_max(mx) * unit), ms = mn == -INFINITY ? 0.f : mn;
    float rs = 0.f;
#pragma unroll
    for (int e = 0; e < 16; e++) { s[e] = fast_exp2(MOD != 0 ? s[e] - ms : fmaf(s[e], unit, -ms)); rs += s[e]; }
    if (__any(mn > m)) {
      const float alpha = fast_exp2(m - ms);
      l *= alpha;
#pragma unroll
      for (int d = 0; d < T::DT; d++) acc[d] *= alpha;
    }
    l += rs;
    m = mn;
    bf16x8 pf[2], vf[T::DT];
    pf[0] = acc_to_frag(s, 0);
    pf[1] = acc_to_frag(s, 1);
    wait_vmcnt<2 * T::LOADS>();                     // V; the next K may be on its way
    T::read_cols(vf, tK + T::BYTES / 2, cbase, 0);
    T::template cols_times<32>(acc, tK + T::BYTES / 2, cbase, pf, vf);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    issue(rv, next, aV);
    t = next;
  }
  wait_vmcnt<0>();                                  // the zero-filled loads past the last tile
  l = both_halves_sum(l);
  float *stats = (float*)(smem_raw + 4 * T::BYTES), *mine = (float*)tK;
  put_partial<T::DT>(mine, acc, lane);
  if (g == 0) { stats[wv * 64 + lane] = m; stats[wv * 64 + 32 + lane] = l; }
  __syncthreads();
  few_finish<bf16, DHP, 4>(a, f, tile, split, head, rows, keys, (const float*)smem_raw, stats, (float*)smem_raw);
}

// ------------------------------------------------------------------------------------
// Backward, part 1: dQ, D = <o, dO> of the rows, and per block of 64 queries which keys some and all of them see, for part 2.
//   S^T = K Q^T,  P^T = exp(S^T - lse),  dP^T = V dO^T,  dS^T = P^T (dP^T - D),  dQ^T += K^T dS^T,  times scale at the end.
// The forward kernel's tiles and phases; the keys of a tile are read once more in the phase after, so they have three stages.
// One document of 8192 rows, 16 heads of 128: 378 us, 1.1 PFLOP/s, the matrix pipe 65 % busy.
// ------------------------------------------------------------------------------------
template <int DHP, int MOD>
__global__ void __launch_bounds__(256, 2) range_bwd_dq_k(RangeAttn a, BlockSeen* __restrict__ blocks) {
  typedef Tiles<DHP> T;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem_raw[];      // K, K, K, V, V
  int qt, h;
  place(a, &qt, &h);
  qt = (a.Tq + 127) / 128 - 1 - qt;
  const int rows = rows_in_use(a), keys = keys_in_use(a), q0 = qt * 128;
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 5;
  const QueryRanges qr = query_ranges(two_ranges(a, q0, rows, keys), q0, rows, lane);
  if (h == 0 && wv < 2) {
    const BlockSeen b = block_seen(a, qt * 2 + wv, rows, keys, lane);
    if (lane == 0 && q0 + wv * 64 < a.Tq) blocks[qt * 2 + wv] = b;
  }
  if (q0 >= rows) return;
  const int myq = q0 + wv * 32 + (lane & 31), kh = h / a.G;
  const int2 mine = myq < rows ? key_range(a, myq, keys) : make_int2(INT_MIN, INT_MAX);
  const int all_from = wave_imax(mine.x), all_to = wave_imin(mine.y);
  const ScoreForm sf = score_form(a, h);
  const int at = MOD & BIASED ? (a.at ? a.at[min(myq, rows - 1)] : myq) : 0;

  bf16x8 qf[T::KK], dof[T::KK];
  T::load_frags((const bf16*)a.q + (i64)myq * a.ldq + (i64)h * a.dh, myq < rows, a.dh, g, qf);
  T::load_frags((const bf16*)a.d_o + (i64)myq * a.ldo + (i64)h * a.dh, myq < rows, a.dh, g, dof);
  float mylse = myq < rows ? a.lse[(i64)h * a.Tq + myq] * LOG2E : 0.f;
  // no sum: it sees nothing, or every score is -infinity, from keys that may hold infinities themselves (times a zero probability)
  bool partly = __any(mylse == -INFINITY && mine.x < mine.y);
  if (mylse == -INFINITY) mylse = 0.f;
  float myD = 0.f;
  {
    bf16x8 of[T::KK];
    T::load_frags((const bf16*)a.o + (i64)myq * a.ldo + (i64)h * a.dh, myq < rows, a.dh, g, of);
#pragma unroll
    for (int kk = 0; kk < T::KK; kk++)
#pragma unroll
      for (int u = 0; u < 8; u++) myD = fmaf((float)of[kk][u], (float)dof[kk][u], myD);
    myD = both_halves_sum(myD);
  }
  const HeadRows rk = {(const unsigned char*)a.k + (i64)kh * a.dh * 2, a.ldk * 2, a.dh * 2}, rv = {(const unsigned char*)a.v + (i64)kh * a.dh * 2, a.ldv * 2, a.dh * 2};
  const unsigned lds0 = lds_address(smem_raw) + (unsigned)wv * (T::BYTES / 4);
  auto issue = [&](const HeadRows& r, int kv, unsigned stage) {
    T::load16(rows_buffer(r, kv, min(64, qr.end - kv)), (unsigned)r.ldb, r.width, wv * 16, lds0 + stage * T::BYTES);
  };
  const unsigned rbase = T::row_base(lane), cbase = T::col_base(lane);
  f32x16 acc[T::DT] = {}, s[2], dp[2];
  bf16x8 dsf[4], first[T::DT];
  bf16x8 fr[2][4];
  auto read_kv = [&](bf16x8 (&f)[4], unsigned sk, unsigned sv, int kk) {
    const unsigned char *cK = smem_raw + sk * T::BYTES, *cV = smem_raw + sv * T::BYTES;
    const unsigned w = rbase ^ (unsigned)(kk * 32);
    f[0] = *(const bf16x8*)(cK + w);
    f[1] = *(const bf16x8*)(cV + w);
    f[2] = *(const bf16x8*)(cK + 32 * T::ROW + w);
    f[3] = *(const bf16x8*)(cV + 32 * T::ROW + w);
  };
  auto times_q = [&](unsigned sk, unsigned sv) {    // (after read_kv(fr[0], .., 0))
#pragma unroll
    for (int j = 0; j < 2; j++) { s[j] = f32x16{}; dp[j] = f32x16{}; }
#pragma unroll
    for (int kk = 0; kk < T::KK; kk++) {
      if (kk < T::KK - 1) read_kv(fr[(kk + 1) & 1], sk, sv, kk + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < 2; j++) {
        s[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[kk & 1][j * 2], qf[kk], s[j], 0, 0, 0);
        dp[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[kk & 1][j * 2 + 1], dof[kk], dp[j], 0, 0, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // With a bias that falls with the distance every query has few keys of weight, and D's error is as large as all roundings together
  // in every row.  There dS keeps 16 bits (a fourth product), and part 2 gets D with what the row's dS, which should add up to nothing,
  // add up to: dq's and dk's errors 1.6 times that of a gradient rounded once -> 1.3, 1.4.
  float rest = 0.f;
  // dS in place of S.  D = <o, dO> carries the rounding of o, which for a query of few keys counts as much as all other roundings: where
  // one tile holds all keys of a query, its D is summed from the tile's own products instead, D = sum P dP.
  auto gradients = [&](int kv) {
    const bool masked = kv < all_from || kv + 64 > all_to, alone = mine.x >= kv && mine.y <= kv + 64;
    if (masked) partly = true;
    tanh_scores<MOD, false>(sf, s[0]);
    tanh_scores<MOD, false>(sf, s[1]);
    float d0 = (float)(at - kv - g * 4);
    int lo = max(mine.x, kv) - kv - g * 4;
    const unsigned n = (unsigned)max(min(mine.y, kv + 64) - max(mine.x, kv), 0);
    auto prob = [&](int j, int e, float* keep) {
      if constexpr (MOD != 0) return fast_exp2(final_score<MOD>(sf, s[j][e], d0 - (float)(j * 32 + (e >> 2) * 8 + (e & 3)), keep) - mylse);
      *keep = 1.f;
      return fast_exp2(fmaf(s[j][e], sf.f, -mylse));
    };
    auto seen = [&](int j, int e) { return (unsigned)(j * 32 + (e >> 2) * 8 + (e & 3) - lo) < n; };
    if (__any(alone)) {
      float sum = 0.f, keep;
#pragma unroll
      for (int j = 0; j < 2; j++)
#pragma unroll
        for (int e = 0; e < 16; e++) sum += seen(j, e) ? prob(j, e, &keep) * dp[j][e] : 0.f;
      sum = both_halves_sum(sum);
      if (alone) myD = sum;                         // (the probabilities are worked out twice, not kept)
      asm volatile("" : "+v"(mylse), "+v"(lo), "+v"(d0));
    }
#pragma unroll
    for (int j = 0; j < 2; j++)
#pragma unroll
      for (int e = 0; e < 16; e++) {
        float keep;
        const float p = prob(j, e, &keep);
        float x = p * (dp[j][e] - myD);
        if constexpr (MOD & BIASED) {
          if (masked && !seen(j, e)) x = 0.f;
          rest += x;
        }
        s[j][e] = x * keep;
      }
    if (masked) {
#pragma unroll
      for (int j = 0; j < 2; j++)
#pragma unroll
        for (int e = 0; e < 16; e++)
          if (!seen(j, e)) s[j][e] = 0.f;
    }
    if constexpr (!(MOD & BIASED)) {
#pragma unroll
      for (int c = 0; c < 4; c++) dsf[c] = acc_to_frag(s[c >> 1], c & 1);
    }
  };
  auto times_k = [&](const unsigned char* tile) {   // dQ^T += K^T dS^T
    if constexpr (MOD & BIASED) T::template cols_times_split<64>(acc, tile, cbase, s, first);
    else T::template cols_times<64>(acc, tile, cbase, dsf, first);
  };
  if (qr.first < qr.end) {
    int kv = qr.first, kv1 = live_from(qr, kv + 64, q0, rows, keys), kv2;
    issue(rk, kv, 0); issue(rv, kv, 3); issue(rk, kv1, 1); issue(rv, kv1, 4);
    T::arrived(qf);
    T::arrived(dof);
    asm volatile("" : "+v"(mylse), "+v"(myD));
    wait_vmcnt<2 * T::LOADS>();
    phase_end();
    unsigned before = 2, now = 0, sv = 3;           // places of K of the last tile and this one, of V of this one
    read_kv(fr[0], 0, 3, 0);
    times_q(0, 3);
    phase_end();
    // the values just read and the keys read for the second time make room
    auto probabilities = [&]() {
      kv2 = live_from(qr, kv1 + 64, q0, rows, keys);
      issue(rk, kv2, before);
      issue(rv, kv2, sv);
      gradients(kv);
      T::read_cols(first, smem_raw + now * T::BYTES, cbase, 0);
      const unsigned next = 3u - before - now;
      before = now;
      now = next;
      sv = 7u - sv;
      wait_vmcnt<2 * T::LOADS>();                   // K and V of the next tile are there
      phase_end();
    };
    while (kv1 < qr.end) {
      probabilities();
      __builtin_amdgcn_s_setprio(1);
      read_kv(fr[0], now, sv, 0);
      times_k(smem_raw + before * T::BYTES);
      times_q(now, sv);
      __builtin_amdgcn_s_setprio(0);
      phase_end();
      kv = kv1;
      kv1 = kv2;
    }
    probabilities();
    times_k(smem_raw + before * T::BYTES);
    wait_vmcnt<0>();                                // the zero-filled loads past the last tile
    phase_end();
  }
  const RangeAttn b = args_again();
  if constexpr (MOD & BIASED) myD += both_halves_sum(rest);
  if (g == 0 && myq < rows) b.dvec[(i64)h * b.Tq + myq] = myD;
  if (partly && !T::finite(acc)) {
    for (int r = 0; r < 32 && q0 + wv * 32 + r < rows; r++) range_row_dq<bf16>(args_again(), q0 + wv * 32 + r, h, keys, (float*)smem_raw + wv * 2 * DHP);
    return;
  }
  if (myq < rows) T::store((bf16*)b.dq + (i64)myq * b.ldq + (i64)h * b.dh, acc, b.scale, b.dh, g);
}

// ------------------------------------------------------------------------------------
// Backward, part 2: dK and dV.  Workgroup = 128 keys of one key head, wave = 32 keys (one per lane column).  It goes over the blocks of
// 64 queries that see some of its keys, and in each over the query heads that share the key head:
//   S = Q K^T,  P = exp(S - lse),  dP = dO V^T,  dS = P (dP - D),  dV^T += dO^T P,  dK^T += Q^T dS, times scale at the end.
// parts > 1: workgroup `part` of a tile takes every parts-th of those (block, head) pairs and leaves its sums in float32 for a second
// launch.  One document of 8192 rows, 16 heads of 128 to 4, 1, 2, 4 parts: 1258 us, 761 + 17, 612 + 28 (0.9 PFLOP/s); the longest chains
// of (block, head) pairs bound the first, registers (two waves per SIMD) the last.
// ------------------------------------------------------------------------------------
template <int DHP> constexpr unsigned DKV_STAGE = 2 * Tiles<DHP>::BYTES + 5 * 256;      // Q, dO, lse, D, lo, hi, at
template <int DHP, int MOD>
__global__ void __launch_bounds__(256, 2) range_bwd_dkv_k(RangeAttn a, const BlockSeen* __restrict__ blocks, float* __restrict__ sums, int parts) {
  typedef Tiles<DHP> T;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem_raw[];      // 2 stages
  const int per = a.Hkv * parts, row = (int)blockIdx.x / per, r0 = (int)blockIdx.x - row * per, kt = paired(row, (a.Tk + 127) / 128, per), kh = r0 % a.Hkv, part = r0 / a.Hkv;
  const int rows = rows_in_use(a), keys = keys_in_use(a), k0 = kt * 128;
  if (k0 >= keys) return;
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 5;
  const int kw = k0 + wv * 32, mykv = kw + (lane & 31);

  bf16x8 kf[T::KK], vf[T::KK];
  T::load_frags((const bf16*)a.k + (i64)mykv * a.ldk + (i64)kh * a.dh, mykv < keys, a.dh, g, kf);
  T::load_frags((const bf16*)a.v + (i64)mykv * a.ldv + (i64)kh * a.dh, mykv < keys, a.dh, g, vf);
  // blocks that see some of the workgroup's keys, from the first to the last
  const int nb = (rows + 63) / 64;
  const int2* seen2 = (const int2*)blocks;
  int b0 = INT_MAX, b1 = -1;
#pragma unroll 4
  for (int b = lane; b < nb; b += 64) {
    const int2 t = seen2[2 * (i64)b];
    if (t.x < k0 + 128 && t.y > k0) { b0 = min(b0, b); b1 = b; }
  }
  b0 = wave_imin(b0);
  b1 = wave_imax(b1);
  unsigned long long live = 0;
  int base = b0 - 64, blk = -1, hg = part - parts;  // hg: head of the pairs of block blk
  bool first = true;
  auto next = [&]() {                               // the next (block, head) of this part; blk = -1: none
    hg += parts;
    while (first || hg >= a.G) {
      while (!live) {
        base += 64;
        if (base > b1 || b1 < 0) { blk = -1; return; }
        const int b = base + lane_now();
        const int2 t = b <= b1 ? seen2[2 * (i64)b] : make_int2(INT_MAX, 0);
        live = __ballot(t.x < k0 + 128 && t.y > k0);
      }
      if (!first) hg -= a.G;
      first = false;
      blk = base + __builtin_ctzll(live);
      live &= live - 1;
    }
  };
  f32x16 dkacc[T::DT] = {}, dvacc[T::DT] = {};
  const unsigned lds0 = lds_address(smem_raw);
  auto issue = [&](int b, int head, int stage) {
    const unsigned dst = lds0 + (unsigned)stage * DKV_STAGE<DHP>;
    const int h = kh * a.G + head, n = min(64, rows - b * 64);
    const HeadRows rq = {(const unsigned char*)a.q + (i64)h * a.dh * 2, a.ldq * 2, a.dh * 2}, ro = {(const unsigned char*)a.d_o + (i64)h * a.dh * 2, a.ldo * 2, a.dh * 2};
    T::load16(rows_buffer(rq, b * 64, n), (unsigned)rq.ldb, rq.width, wv * 16, dst + wv * (T::BYTES / 4));
    T::load16(rows_buffer(ro, b * 64, n), (unsigned)ro.ldb, ro.width, wv * 16, dst + T::BYTES + wv * (T::BYTES / 4));
    const unsigned words = dst + 2 * T::BYTES, off = (unsigned)lane_now() * 4u;
    if (wv == 0) load_lds_b32(words_buffer(a.lse + (i64)h * a.Tq, b * 64, n), words, off);
    if (wv == 1) load_lds_b32(words_buffer(a.dvec + (i64)h * a.Tq, b * 64, n), words + 256u, off);
    if (wv == 2) load_lds_b32(words_buffer(a.lo, b * 64, n), words + 512u, off);
    if (wv == 3) load_lds_b32(words_buffer(a.hi, b * 64, n), words + 768u, off);
    if constexpr (MOD & BIASED) {
      if (wv == 0 && a.at) load_lds_b32(words_buffer(a.at, b * 64, n), words + 1024u, off);
      if (wv == 0 && !a.at) ((int*)(smem_raw + (unsigned)stage * DKV_STAGE<DHP> + 2 * T::BYTES + 1024u))[off / 4] = b * 64 + (int)off / 4;
    }
  };
  bool partly = false;
  next();
  if (blk >= 0) issue(blk, hg, 0);
  T::arrived(kf);
  T::arrived(vf);
  wait_vmcnt<0>();
  __syncthreads();
  int cur = 0;
  while (blk >= 0) {
    const int b = blk, h = kh * a.G + hg;
    const int4 seen = blocks[b];
    next();
    if (blk >= 0) issue(blk, hg, cur ^ 1);
    if (seen.x < kw + 32 && seen.y > kw) {          // some query of the block sees some key of this wave
      const bool whole = seen.z <= kw && seen.w >= kw + 32;
      const ScoreForm sf = score_form(a, h);
      const unsigned char *cQ = smem_raw + cur * DKV_STAGE<DHP>, *cO = cQ + T::BYTES;
      const float *cL = (const float*)(cO + T::BYTES), *cD = cL + 64;
      if (!whole || __any(cL[lane_now()] == -INFINITY)) partly = true;      // (a query whose scores are all -infinity: exp(-inf + inf) here)
      const int *cLo = (const int*)(cD + 64), *cHi = cLo + 64, *cAt = cHi + 64;
#pragma unroll 1
      for (int j = 0; j < 2; j++) {
        const int lane = lane_now(), g = lane >> 5, mykv = kw + (lane & 31);
        const unsigned rb = T::row_base(lane) + (unsigned)(j * 32 * T::ROW), cb = T::col_base(lane);
        f32x16 s = {}, dp = {};
        bf16x8 f[2][2];
        auto read_rows = [&](bf16x8 (&x)[2], int kk) {
          x[0] = *(const bf16x8*)(cQ + (rb ^ (unsigned)(kk * 32)));
          x[1] = *(const bf16x8*)(cO + (rb ^ (unsigned)(kk * 32)));
        };
        read_rows(f[0], 0);
#pragma unroll
        for (int kk = 0; kk < T::KK; kk++) {
          if (kk < T::KK - 1) read_rows(f[(kk + 1) & 1], kk + 1);
          __builtin_amdgcn_sched_barrier(0);
          s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[kk & 1][0], kf[kk], s, 0, 0, 0);
          dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[kk & 1][1], vf[kk], dp, 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        }
        tanh_scores<MOD, false>(sf, s);
        // element e is query j * 32 + (e >> 2) * 8 + g * 4 + (e & 3) of the block
#pragma unroll
        for (int eb = 0; eb < 4; eb++) {
          const int q4 = j * 32 + eb * 8 + g * 4;
          if constexpr (DHP == 128) __builtin_amdgcn_sched_barrier(0);      // (all reads at once would cost the registers that are short here)
          const float4 l4 = *(const float4*)(cL + q4), d4 = *(const float4*)(cD + q4);
          const float lv[4] = {l4.x, l4.y, l4.z, l4.w}, dv[4] = {d4.x, d4.y, d4.z, d4.w};
          int av[4];
          if constexpr (MOD & BIASED) {
            const int4 a4 = *(const int4*)(cAt + q4);
            av[0] = a4.x; av[1] = a4.y; av[2] = a4.z; av[3] = a4.w;
          }
#pragma unroll
          for (int i = 0; i < 4; i++) {
            const int e = eb * 4 + i;
            float x, keep = 1.f;
            if constexpr (MOD != 0) x = fmaf(lv[i], -LOG2E, final_score<MOD>(sf, s[e], MOD & BIASED ? (float)(av[i] - mykv) : 0.f, &keep));
            else x = fmaf(s[e], sf.f, -lv[i] * LOG2E);
            s[e] = fast_exp2(x);
            dp[e] = s[e] * (dp[e] - dv[i]) * keep;
          }
        }
        if (!whole) {
#pragma unroll
          for (int eb = 0; eb < 4; eb++) {
            const int q4 = j * 32 + eb * 8 + g * 4;
            if constexpr (DHP == 128) __builtin_amdgcn_sched_barrier(0);
            const int4 l4 = *(const int4*)(cLo + q4), h4 = *(const int4*)(cHi + q4);
            const int lo[4] = {l4.x, l4.y, l4.z, l4.w}, hi[4] = {h4.x, h4.y, h4.z, h4.w};
#pragma unroll
            for (int i = 0; i < 4; i++)
              if (mykv < lo[i] || mykv >= hi[i]) s[eb * 4 + i] = dp[eb * 4 + i] = 0.f;
          }
        }
        bf16x8 pf[2], dsf[2];
#pragma unroll
        for (int c = 0; c < 2; c++) { pf[c] = acc_to_frag(s, c); dsf[c] = acc_to_frag(dp, c); }
        // dO^T P and Q^T dS by turns, 16 queries each, the next fragments read while these are multiplied
        bf16x8 x[2][T::DT];
        T::read_cols(x[0], cO + j * 32 * T::ROW, cb, 0);
#pragma unroll
        for (int c = 0; c < 4; c++) {
          if (c < 3) T::read_cols(x[(c + 1) & 1], (c & 1 ? cO : cQ) + j * 32 * T::ROW, cb, (c + 1) >> 1);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int d = 0; d < T::DT; d++) {
            if (c & 1) dkacc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[c & 1][d], dsf[c >> 1], dkacc[d], 0, 0, 0);
            else dvacc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[c & 1][d], pf[c >> 1], dvacc[d], 0, 0, 0);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
    // this wave's part of the next tile has landed, and its reads of this one have returned
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __syncthreads();
    cur ^= 1;
  }
  if (parts > 1) {
    if (mykv >= keys) return;
    float* out = sums + ((((i64)part * 2) * a.Tk + mykv) * a.Hkv + kh) * DHP;
    const i64 dv = (i64)a.Tk * a.Hkv * DHP;
#pragma unroll
    for (int d = 0; d < T::DT; d++)
#pragma unroll
      for (int e = 0; e < 4; e++) {
        const int c = d * 32 + e * 8 + g * 4;
        *(float4*)(out + c) = make_float4(dkacc[d][e * 4], dkacc[d][e * 4 + 1], dkacc[d][e * 4 + 2], dkacc[d][e * 4 + 3]);
        *(float4*)(out + dv + c) = make_float4(dvacc[d][e * 4], dvacc[d][e * 4 + 1], dvacc[d][e * 4 + 2], dvacc[d][e * 4 + 3]);
      }
    return;
  }
  if (partly && (!T::finite(dkacc) || !T::finite(dvacc))) {
    for (int r = 0; r < 32 && kw + r < keys; r++) range_row_dkv<bf16>(args_again(), kw + r, kh, rows, keys, (float*)smem_raw + wv * 2 * DHP);
    return;
  }
  if (mykv < keys) {
    const RangeAttn b = args_again();
    T::store((bf16*)b.dk + (i64)mykv * b.ldk + (i64)kh * b.dh, dkacc, b.scale, b.dh, g);
    T::store((bf16*)b.dv + (i64)mykv * b.ldv + (i64)kh * b.dh, dvacc, 1.0f, b.dh, g);
  }
}
// ------------------------------------------------------------------------------------
// Backward for few rows: dQ of 32 rows, then dK/dV of 32 keys per workgroup, the keys (the blocks of 32 queries and the heads that share the
// key head) shared out to the waves, each with tiles of its own in LDS.  A workgroup's first loads and last sums are half of its time where
// documents are short (2048 rows x 16 heads of 128, longest 730: 33 and 39 us).
// ------------------------------------------------------------------------------------
// a^T[row, lane] = tile a's rows x fa, the same for b; the next fragments are read while these are multiplied
template <int DHP> __device__ __forceinline__ void rows_times2(f32x16& a, f32x16& b, const unsigned char* ta, const unsigned char* tb, unsigned rbase,
                                                               const bf16x8 (&fa)[DHP / 16], const bf16x8 (&fb)[DHP / 16]) {
  bf16x8 x[2][2];
  auto read = [&](bf16x8 (&y)[2], int kk) {
    y[0] = *(const bf16x8*)(ta + (rbase ^ (unsigned)(kk * 32)));
    y[1] = *(const bf16x8*)(tb + (rbase ^ (unsigned)(kk * 32)));
  };
  a = f32x16{};
  b = f32x16{};
  read(x[0], 0);
#pragma unroll
  for (int kk = 0; kk < DHP / 16; kk++) {
    if (kk < DHP / 16 - 1) read(x[(kk + 1) & 1], kk + 1);
    __builtin_amdgcn_sched_barrier(0);
    a = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[kk & 1][0], fa[kk], a, 0, 0, 0);
    b = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[kk & 1][1], fb[kk], b, 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
  }
}
// The last workgroups of the launch (from `tiles` on) note which keys the blocks of 64 queries see, a wave per block.
template <int DHP, int MOD>
__global__ void __launch_bounds__(256, 2) range_dq_few_k(RangeAttn a, FewShape f, int tiles, BlockSeen* __restrict__ blocks) {
  typedef Tiles<DHP> T;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem_raw[];
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 5;
  if ((int)blockIdx.x >= tiles) {
    const int b = ((int)blockIdx.x - tiles) * 4 + wv;
    const BlockSeen r = block_seen(a, b, rows_in_use(a), keys_in_use(a), lane);
    if (lane == 0 && b * 64 < a.Tq) blocks[b] = r;
    return;
  }
  int tile, split, head, t0;
  few_place(a, f, (int)blockIdx.x, &tile, &split, &head);
  const int kh = head % a.Hkv;
  FewRow row = few_row(a, f, tile, head, lane & 31, a.Tq);
  const int2 stored = stored_range(a, row.i);
  const int at = (MOD & BIASED) && row.ok ? (a.at ? a.at[row.i] : row.i) : 0;
  const i64 orow = (i64)row.i * a.ldo + (i64)row.h * a.dh, srow = (i64)row.h * a.Tq + row.i;
  bf16x8 qf[T::KK], dof[T::KK], of[T::KK];
  float L = row.ok ? a.lse[srow] * LOG2E : 0.f, D = 0.f;
  T::load_frags((const bf16*)a.d_o + orow, row.ok, a.dh, g, dof);
  T::load_frags((const bf16*)a.o + orow, row.ok, a.dh, g, of);
  T::load_frags((const bf16*)a.q + (i64)row.i * a.ldq + (i64)row.h * a.dh, row.ok, a.dh, g, qf);
  const int rows = rows_in_use(a), keys = keys_in_use(a);
  if (tile * f.qpt >= rows) return;
  row.ok = row.ok && row.i < rows;
  const FewKeys fk = few_keys(f, row, stored, 0, keys, &t0);
  const ScoreForm sf = score_form(a, row.h);
  const HeadRows rk = {(const unsigned char*)a.k + (i64)kh * a.dh * 2, a.ldk * 2, a.dh * 2}, rv = {(const unsigned char*)a.v + (i64)kh * a.dh * 2, a.ldv * 2, a.dh * 2};
  unsigned char* tK = smem_raw + wv * T::BYTES;      // 32 rows of K, 32 of V
  const unsigned aK = lds_address(smem_raw) + (unsigned)wv * T::BYTES, aV = aK + T::BYTES / 2;
  auto issue = [&](const HeadRows& r, int t, unsigned dst) {
    const int kv = fk.first + t * 32;
    const __amdgpu_buffer_rsrc_t rs = rows_buffer(r, kv, min(32, fk.end - kv));
    T::load16(rs, (unsigned)r.ldb, r.width, 0, dst);
    T::load16(rs, (unsigned)r.ldb, r.width, 16, dst + 16 * T::ROW);
  };
  int t = fk.live_from(t0 + wv, 4);
  if (t < fk.t1) {
    issue(rv, t, aV);
    issue(rk, t, aK);
  }
#pragma unroll
  for (int kk = 0; kk < T::KK; kk++)
#pragma unroll
    for (int u = 0; u < 8; u++) D = fmaf((float)of[kk][u], (float)dof[kk][u], D);
  D = both_halves_sum(D);
  if (L == -INFINITY) L = 0.f;
  T::arrived(qf);
  T::arrived(dof);
  asm volatile("" : "+v"(L), "+v"(D));
  const unsigned rbase = T::row_base(lane), cbase = T::col_base(lane);
  f32x16 acc[T::DT] = {};
  bool own = wv == 0;                               // this wave has the row's D
  float rest = 0.f;
  while (t < fk.t1) {
    const int kv = fk.first + t * 32, next = fk.live_from(t + 4, 4);
    wait_vmcnt<0>();
    f32x16 dp, s;
    rows_times2<DHP>(dp, s, tK + T::BYTES / 2, tK, rbase, dof, qf);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    if (next < fk.t1) issue(rv, next, aV);
    const float d0 = (float)(at - kv - g * 4);
    const int lo = max(fk.r.x, kv) - kv - g * 4;
    const unsigned n = (unsigned)max(min(fk.r.y, kv + 32) - max(fk.r.x, kv), 0);
    float keep[16];
    tanh_scores<MOD, false>(sf, s);
#pragma unroll
    for (int e = 0; e < 16; e++) {
      if constexpr (MOD != 0) s[e] = fast_exp2(final_score<MOD>(sf, s[e], d0 - (float)((e >> 2) * 8 + (e & 3)), &keep[e]) - L);
      else { s[e] = fast_exp2(fmaf(s[e], sf.f, -L)); keep[e] = 1.f; }
    }
    const bool masked = !__all(!row.ok || (fk.r.x <= kv && fk.r.y >= kv + 32));
    if (masked) {
#pragma unroll
      for (int e = 0; e < 16; e++) if ((unsigned)((e >> 2) * 8 + (e & 3) - lo) >= n) s[e] = dp[e] = 0.f;
    }
    // (as in the other form: D of a row whose keys are all in this tile)
    const bool alone = fk.r.x >= kv && fk.r.y <= kv + 32 && fk.r.x < fk.r.y;
    if (__any(alone)) {
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 16; e++) sum = fmaf(s[e], dp[e], sum);
      sum = both_halves_sum(sum);
      if (alone) { D = sum; own = true; }
    }
#pragma unroll
    for (int e = 0; e < 16; e++) s[e] *= dp[e] - D;
    if (masked) {                                   // (D may be no number)
#pragma unroll
      for (int e = 0; e < 16; e++) if ((unsigned)((e >> 2) * 8 + (e & 3) - lo) >= n) s[e] = 0.f;
    }
    if constexpr (MOD & BIASED) {                   // (as in the other form)
#pragma unroll
      for (int e = 0; e < 16; e++) rest += s[e];
    }
#pragma unroll
    for (int e = 0; e < 16; e++) s[e] *= keep[e];
    bf16x8 first[T::DT];
    T::read_cols(first, tK, cbase, 0);
    if constexpr (MOD & BIASED) T::template cols_times_split<32>(acc, tK, cbase, &s, first);
    else {
      const bf16x8 ds[2] = {acc_to_frag(s, 0), acc_to_frag(s, 1)};
      T::template cols_times<32>(acc, tK, cbase, ds, first);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    if (next < fk.t1) issue(rk, next, aK);
    t = next;
  }
  float4* found = (float4*)(smem_raw + 4 * T::BYTES);      // [wave][row]: D, whether it is the one, the sum of dS
  rest = both_halves_sum(rest);
  if (g == 0) found[wv * 32 + lane] = make_float4(D, own ? 1.f : 0.f, rest, 0.f);
  put_partial<T::DT>((float*)tK, acc, lane);
  __syncthreads();
  const FewRow mine = few_row(a, f, tile, head, threadIdx.x & 31, rows);
  if (threadIdx.x < 32 && mine.ok) {
    float d = found[threadIdx.x].x;
#pragma unroll
    for (int w = 1; w < 4; w++) if (found[w * 32 + threadIdx.x].y != 0.f) d = found[w * 32 + threadIdx.x].x;
    if constexpr (MOD & BIASED) {
#pragma unroll
      for (int w = 0; w < 4; w++) d += found[w * 32 + threadIdx.x].z;
    }
    a.dvec[(i64)mine.h * a.Tq + mine.i] = d;
  }
  const bool fine = few_store<bf16, DHP, 4>((const float*)smem_raw, (bf16*)a.dq + (i64)mine.i * a.ldq + (i64)mine.h * a.dh, mine.ok, a.dh, a.scale);
  if (__syncthreads_or(!fine))
    for (int x = wv; x < 32; x += 4) {
      const FewRow again = few_row(a, f, tile, head, x, rows);
      if (again.ok) range_row_dq<bf16>(args_again(), again.i, again.h, keys, (float*)smem_raw + wv * 2 * DHP);
    }
}
template <int DHP, int MOD>
__global__ void __launch_bounds__(256, 2) range_dkv_few_k(RangeAttn a, const BlockSeen* __restrict__ blocks, float* __restrict__ sums, int parts) {
  typedef Tiles<DHP> T;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem_raw[];
  const int per = a.Hkv * parts, kt = (int)blockIdx.x / per, r0 = (int)blockIdx.x - kt * per, kh = r0 % a.Hkv, part = r0 / a.Hkv;
  const int k0 = kt * 32;                           // early keys are seen by the most queries
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 5, mykv = k0 + (lane & 31);
  // (first loads: see stored_range)
  bf16x8 kf[T::KK], vf[T::KK];
  const int2 nobody = make_int2(INT_MAX, 0);
  int2 seen0 = lane * 64 < a.Tq ? *(const int2*)(blocks + lane) : nobody;
  T::load_frags((const bf16*)a.k + (i64)mykv * a.ldk + (i64)kh * a.dh, mykv < a.Tk, a.dh, g, kf);
  T::load_frags((const bf16*)a.v + (i64)mykv * a.ldv + (i64)kh * a.dh, mykv < a.Tk, a.dh, g, vf);
  const int rows = rows_in_use(a), keys = keys_in_use(a);
  if (k0 >= keys) return;
  unsigned char* tQ = smem_raw + wv * T::BYTES;      // 32 rows of Q, 32 of dO
  const unsigned aQ = lds_address(smem_raw) + (unsigned)wv * T::BYTES, aS = lds_address(smem_raw) + 4 * T::BYTES + (unsigned)wv * 1280u;
  const float* st = (const float*)(smem_raw + 4 * T::BYTES + wv * 1280);      // lse, D, lo, hi, at: 64 words each, of which 32 are used
  // the pairs of a block of 32 queries, in a block of 64 that sees some of the keys, and a head, dealt out to the waves of all parts
  const int nb = (rows + 63) / 64;
  unsigned long long live = __ballot(lane < nb && seen0.x < k0 + 32 && seen0.y > k0);
  int base = 0, blk = -1, n = part * 4 + wv, q0 = -1, h = 0;      // n: of the pairs of block blk, 2 G to a block
  auto next = [&]() {                               // q0 = -1: none
    do {
      while (blk < 0 || n >= 2 * a.G) {
        while (!live) {
          base += 64;
          if (base >= nb) { q0 = -1; return; }
          const int b = base + lane_now();
          const int2 r = b < nb ? *(const int2*)(blocks + b) : make_int2(INT_MAX, 0);
          live = __ballot(r.x < k0 + 32 && r.y > k0);
        }
        if (blk >= 0) n -= 2 * a.G;
        blk = base + __builtin_ctzll(live);
        live &= live - 1;
      }
      q0 = blk * 64 + (n & 1) * 32;
      h = kh * a.G + (n >> 1);
      n += 4 * parts;
    } while (q0 >= rows);
  };
  auto issue = [&]() {
    const int m = min(32, rows - q0);
    const HeadRows rq = {(const unsigned char*)a.q + (i64)h * a.dh * 2, a.ldq * 2, a.dh * 2}, ro = {(const unsigned char*)a.d_o + (i64)h * a.dh * 2, a.ldo * 2, a.dh * 2};
    const __amdgpu_buffer_rsrc_t bq = rows_buffer(rq, q0, m), bo = rows_buffer(ro, q0, m);
    T::load16(bq, (unsigned)rq.ldb, rq.width, 0, aQ);
    T::load16(bq, (unsigned)rq.ldb, rq.width, 16, aQ + 16 * T::ROW);
    T::load16(bo, (unsigned)ro.ldb, ro.width, 0, aQ + T::BYTES / 2);
    T::load16(bo, (unsigned)ro.ldb, ro.width, 16, aQ + T::BYTES / 2 + 16 * T::ROW);
    const unsigned off = (unsigned)lane_now() * 4u;
    load_lds_b32(words_buffer(a.lse + (i64)h * a.Tq, q0, m), aS, off);
    load_lds_b32(words_buffer(a.dvec + (i64)h * a.Tq, q0, m), aS + 256u, off);
    load_lds_b32(words_buffer(a.lo, q0, m), aS + 512u, off);
    load_lds_b32(words_buffer(a.hi, q0, m), aS + 768u, off);
    if constexpr (MOD & BIASED) {
      if (a.at) load_lds_b32(words_buffer(a.at, q0, m), aS + 1024u, off);
      else ((int*)st)[256 + off / 4] = q0 + (int)off / 4;
    }
  };
  next();
  if (q0 >= 0) issue();
  T::arrived(kf);
  T::arrived(vf);
  f32x16 dka[T::DT] = {}, dva[T::DT] = {};
  while (q0 >= 0) {
    const ScoreForm sf = score_form(a, h);
    wait_vmcnt<0>();
    const int lane = lane_now(), g = lane >> 5, mykv = k0 + (lane & 31);
    const unsigned rbase = T::row_base(lane), cbase = T::col_base(lane);
    f32x16 s, dp;
    rows_times2<DHP>(s, dp, tQ, tQ + T::BYTES / 2, rbase, kf, vf);
    tanh_scores<MOD, false>(sf, s);
    const int2 lo_hi = make_int2(((const int*)st)[128 + (lane & 31)], ((const int*)st)[192 + (lane & 31)]);
#pragma unroll
    for (int eb = 0; eb < 4; eb++) {
      const int r0 = eb * 8 + g * 4;
      __builtin_amdgcn_sched_barrier(0);            // (all reads at once would cost the registers that are short here)
      const float4 l4 = *(const float4*)(st + r0), d4 = *(const float4*)(st + 64 + r0);
      const float lv[4] = {l4.x, l4.y, l4.z, l4.w}, dv[4] = {d4.x, d4.y, d4.z, d4.w};
      int av[4] = {0, 0, 0, 0};
      if constexpr (MOD & BIASED) {
        const int4 a4 = *(const int4*)(st + 256 + r0);
        av[0] = a4.x; av[1] = a4.y; av[2] = a4.z; av[3] = a4.w;
      }
#pragma unroll
      for (int i = 0; i < 4; i++) {
        const int e = eb * 4 + i;
        float x, keep = 1.f;
        if constexpr (MOD != 0) x = fmaf(lv[i], -LOG2E, final_score<MOD>(sf, s[e], MOD & BIASED ? (float)(av[i] - mykv) : 0.f, &keep));
        else x = fmaf(s[e], sf.f, -lv[i] * LOG2E);
        s[e] = fast_exp2(x);
        dp[e] = s[e] * (dp[e] - dv[i]) * keep;
      }
    }
    if (!__all(lo_hi.x <= k0 && lo_hi.y >= k0 + 32)) {
#pragma unroll
      for (int eb = 0; eb < 4; eb++) {
        const int r0 = eb * 8 + g * 4;
        __builtin_amdgcn_sched_barrier(0);
        const int4 lo4 = *(const int4*)(st + 128 + r0), hi4 = *(const int4*)(st + 192 + r0);
        const int lo[4] = {lo4.x, lo4.y, lo4.z, lo4.w}, hi[4] = {hi4.x, hi4.y, hi4.z, hi4.w};
#pragma unroll
        for (int i = 0; i < 4; i++)
          if (mykv < lo[i] || mykv >= hi[i]) s[eb * 4 + i] = dp[eb * 4 + i] = 0.f;
      }
    }
    bf16x8 pf[2], dsf[2];
#pragma unroll
    for (int c = 0; c < 2; c++) { pf[c] = acc_to_frag(s, c); dsf[c] = acc_to_frag(dp, c); }
    const unsigned char* tO = tQ + T::BYTES / 2;
    bf16x8 x[2][T::DT];
    T::read_cols(x[0], tO, cbase, 0);
#pragma unroll
    for (int c = 0; c < 4; c++) {
      if (c < 3) T::read_cols(x[(c + 1) & 1], c & 1 ? tO : tQ, cbase, (c + 1) >> 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int d = 0; d < T::DT; d++) {
        if (c & 1) dka[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[c & 1][d], dsf[c >> 1], dka[d], 0, 0, 0);
        else dva[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[c & 1][d], pf[c >> 1], dva[d], 0, 0, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    next();
    if (q0 >= 0) issue();
  }
  const RangeAttn b = args_again();
  const int r = k0 + (int)(threadIdx.x & 31);
  if (parts > 1) {
    float* row = sums + ((((i64)part * 2) * b.Tk + r) * b.Hkv + kh) * DHP;
    put_partial<T::DT>((float*)tQ, dka, lane);
    __syncthreads();
    (void)few_store<float, DHP, 4>((const float*)smem_raw, row, r < keys, DHP, 1.f);
    __syncthreads();
    put_partial<T::DT>((float*)tQ, dva, lane);
    __syncthreads();
    (void)few_store<float, DHP, 4>((const float*)smem_raw, row + (i64)b.Tk * b.Hkv * DHP, r < keys, DHP, 1.f);
    return;
  }
  put_partial<T::DT>((float*)tQ, dka, lane);
  __syncthreads();
  bool fine = few_store<bf16, DHP, 4>((const float*)smem_raw, (bf16*)b.dk + (i64)r * b.ldk + (i64)kh * b.dh, r < keys, b.dh, b.scale);
  __syncthreads();
  put_partial<T::DT>((float*)tQ, dva, lane);
  __syncthreads();
  fine &= few_store<bf16, DHP, 4>((const float*)smem_raw, (bf16*)b.dv + (i64)r * b.ldv + (i64)kh * b.dh, r < keys, b.dh, 1.f);
  if (__syncthreads_or(!fine))
    for (int x = wv; x < 32 && k0 + x < keys; x += 4) range_row_dkv<bf16>(b, k0 + x, kh, rows, keys, (float*)smem_raw + wv * 2 * DHP);
}

// ---- launchers ----
static bool takes(const RangeAttn& a, bool back) {
  // (the tanh of these kernels is off by up to 2^-22 where a wave has large scores, a capped score by that of the cap: 2^-10 at most here)
  if (a.dt != 1 || a.dh > 128 || a.dh % 8 || a.cap > 4096.f) return false;
  uintptr_t p = (uintptr_t)a.q | (uintptr_t)a.k | (uintptr_t)a.v;
  p |= back ? (uintptr_t)a.o | (uintptr_t)a.d_o | (uintptr_t)a.dq | (uintptr_t)a.dk | (uintptr_t)a.dv : (uintptr_t)a.out;
  const i64 l = a.ldq | a.ldk | a.ldv | a.ldo;
  // 64 rows of a tile are addressed with 31-bit byte offsets
  return !(p & 15) && !(l & 7) && a.ldq < (1 << 24) && a.ldk < (1 << 24) && a.ldv < (1 << 24) && a.ldo < (1 << 24);
}
bool range_flash_takes(const RangeAttn& a, bool back) { return takes(a, back); }
// what a kernel has to have; a negative scale needs scores in their final form before the maximum, as a bias does
static int parts_of_score(const RangeAttn& a) {
  const int m = (a.cap > 0.f ? CAPPED : 0) | (a.slopes ? BIASED : 0);
  return m == 0 && a.scale < 0.f ? BIASED : m;
}
#define BY_FORM(call)                                                              \
  do {                                                                             \
    const int m = parts_of_score(a);                                               \
    if (a.dh <= 64) { if (m == 0) call(64, 0); else if (m == 1) call(64, 1); else if (m == 2) call(64, 2); else call(64, 3); } \
    else if (m == 0) call(128, 0);                                                 \
    else if (m == 1) call(128, 1);                                                 \
    else if (m == 2) call(128, 2);                                                 \
    else call(128, 3);                                                             \
  } while (0)

template <class K> static void set_lds(std::atomic<unsigned long long>& mask, K kernel, unsigned bytes) {
  if (attr_needed(mask)) {
    (void)hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    attr_done(mask);
  }
}
// Parts of a key tile's (query block, head) pairs in dK/dV, for 128 keys per workgroup and for 32: workgroups enough to fill the chip twice, where
// several heads that share a key head make the pairs many (and the float32 sums that a part costs few).  For 1 to 8 parts: see range_bwd_dkv_k.
static int dkv_parts(const RangeAttn& a) {
  const i64 workgroups = (i64)cdiv(a.Tk, 128) * a.Hkv;
  int n = 1;
  while (a.G > 1 && n < 8 && n < 2 * a.G && workgroups * n < 1024) n *= 2;
  return n;
}
static int dkv_parts_few(const RangeAttn& a) {
  const i64 workgroups = (i64)cdiv(a.Tk, 32) * a.Hkv;
  int n = 1;
  while (n < 8 && n < a.G && workgroups * n < 1024) n *= 2;
  return n;
}
size_t range_flash_sum_floats(const RangeAttn& a) {
  const int n = dkv_parts(a) > dkv_parts_few(a) ? dkv_parts(a) : dkv_parts_few(a);
  return n > 1 ? (size_t)n * 2 * a.Tk * a.Hkv * (a.dh <= 64 ? 64 : 128) : 0;
}
// Which form each kernel takes; form: 0 by the rules, 1 for few rows, 2 for many.  The lengths of the documents, which the host does not know, count as
// much as the sizes: documents of 512 are at home in tiles of 128 at half of a line, long ones only above it.  The lines lie where the geometric mean over
// three kinds of batch crosses 1: many / few (above 1: few rows are faster), documents of 30 to 730 rows, one document, documents of 512, heads of 128
//   forward  1024 x 32 rows x heads 1.08 1.12 0.92   2304 x 16 1.12 1.16 0.81   5000 x 8 1.00 1.23 0.82   2560 x 16 1.02 1.10 0.84   1400 x 32 1.00 0.92 0.75
//   dQ                              1.04 1.04 0.85             1.05 1.14 0.79            1.00 1.19 0.81             0.97 1.08 0.84             0.97 0.89 0.77
//   dK/dV    1400 x 32 1.16 1.08 0.87   3300 x 16 1.21 1.07 0.87   6500 x 8 1.09 1.15 0.84   3700 x 16 1.07 1.02 0.85   2048 x 32 0.96 0.88 0.72
// and of 64
//   forward  3300 x 16 1.00 1.22 0.89   2048 x 32 1.10 0.99 0.82   4096 x 16 1.08 1.06 0.77   5400 x 16 1.18 0.91 0.90   8192 x 16 0.96 0.73 0.78
//   dQ                 1.00 1.10 0.84             0.94 0.92 0.74             0.99 0.99 0.70             1.05 0.86 0.84             0.91 0.74 0.75
//   (capped, the documents of 30 to 730 rows: 4095 x 16 1.33, dQ 1.20; 5400 x 16 1.45, 1.28)
//   dK/dV    5000 x 8 1.46 1.60 0.98    2048 x 32 1.15 1.06 0.83   4096 x 16 1.18 1.13 0.79   5400 x 16 1.07 0.98 0.87   8192 x 16 0.90 0.77 0.79
// dK/dV with heads that share a key head (128, then 64): query rows x heads / key heads
//   2048 x 16/8 1.17 1.05 1.04, 1.14 1.10 0.95   3300 x 16/8 1.13 0.85 1.04, 1.01 0.92 1.05   4096 x 16/8 1.57 0.99, 1.28 0.92   8192 x 16/8 of 64 1.32 0.82
//   2048 x 16/4 1.19 1.05 1.04, 1.19 1.13 1.01   1024 x 32/8 1.07 1.00, 1.04 0.98   1400 x 32/8 1.03 0.93 1.04, 1.17 0.95 1.06   6000 x 8/2 1.13 0.80, 1.14 0.86
//   4096 x 16/1 1.66 1.70, 1.65 2.04   6000 x 16/1 1.31 1.27 1.04, 1.38 1.39 1.13   8192 x 16/1 0.94 0.94 0.75, 0.96 1.03 0.81
static bool few_queries(const RangeAttn& a, int form) { return form ? form == 1 : (i64)a.Tq * a.H <= (a.dh <= 64 ? 64 : 36) * 1024; }
static bool few_dkv(const RangeAttn& a, int form) {
  if (form) return form == 1;
  const i64 rows = (i64)a.Tk * a.H;
  if (a.G <= 2) return rows <= (a.G == 2 || a.dh <= 64 ? 64 : 48) * 1024;
  return (i64)a.Tk * a.Hkv <= 8 * 1024 && rows <= 96 * 1024;
}

template <int DHP, int MOD> static void bwd(const RangeAttn& a, void* blocks, float* sums, int form, hipStream_t s) {
  const bool fq = few_queries(a, form), fkv = few_dkv(a, form);
  if (a.Tq > 0 && fq) {
    static std::atomic<unsigned long long> mask{0};
    constexpr unsigned smem = 4 * Tiles<DHP>::BYTES + 4 * 512;
    set_lds(mask, range_dq_few_k<DHP, MOD>, smem);
    FewShape f = few_shape(a, nullptr);
    f.splits = 1;
    const int tiles = f.tiles * a.Hkv * f.hb;
    hipLaunchKernelGGL((range_dq_few_k<DHP, MOD>), dim3((unsigned)(tiles + cdiv(a.Tq, 64 * 4))), dim3(256), smem, s, a, f, tiles, (BlockSeen*)blocks);
  } else if (a.Tq > 0) {
    static std::atomic<unsigned long long> mask{0};
    constexpr unsigned smem = 5 * Tiles<DHP>::BYTES;
    set_lds(mask, range_bwd_dq_k<DHP, MOD>, smem);
    hipLaunchKernelGGL((range_bwd_dq_k<DHP, MOD>), dim3((unsigned)((i64)cdiv(a.Tq, 128) * a.H)), dim3(256), smem, s, a, (BlockSeen*)blocks);
  }
  if (a.Tk <= 0) return;
  const int parts = fkv ? dkv_parts_few(a) : dkv_parts(a);
  if (fkv) {
    static std::atomic<unsigned long long> mask{0};
    constexpr unsigned smem = 4 * Tiles<DHP>::BYTES + 4 * 1280;
    set_lds(mask, range_dkv_few_k<DHP, MOD>, smem);
    hipLaunchKernelGGL((range_dkv_few_k<DHP, MOD>), dim3((unsigned)((i64)cdiv(a.Tk, 32) * a.Hkv * parts)), dim3(256), smem, s, a, (const BlockSeen*)blocks, sums, parts);
  } else {
    static std::atomic<unsigned long long> mask{0};
    constexpr unsigned smem = 2 * DKV_STAGE<DHP>;
    set_lds(mask, range_bwd_dkv_k<DHP, MOD>, smem);
    hipLaunchKernelGGL((range_bwd_dkv_k<DHP, MOD>), dim3((unsigned)((i64)cdiv(a.Tk, 128) * a.Hkv * parts)), dim3(256), smem, s, a, (const BlockSeen*)blocks, sums, parts);
  }
  sum_parts<bf16, DHP>(a, sums, parts, s);
}
template <int DHP, int MOD> static void fwd(const RangeAttn& a, float* work, int form, hipStream_t s) {
  static std::atomic<unsigned long long> mask{0};
  if (few_queries(a, form)) {
    set_lds(mask, range_fwd_few_k<DHP, MOD>, FEW_SMEM<DHP>);
    const FewShape f = few_shape(a, work);
    hipLaunchKernelGGL((range_fwd_few_k<DHP, MOD>), dim3((unsigned)((i64)f.tiles * f.splits * a.Hkv * f.hb)), dim3(256), FEW_SMEM<DHP>, s, a, f);
    join_splits<bf16, DHP>(a, f, s);
    return;
  }
  static std::atomic<unsigned long long> mask_many{0};
  constexpr unsigned smem = 4 * Tiles<DHP>::BYTES;
  set_lds(mask_many, range_fwd_k<DHP, MOD>, smem);
  hipLaunchKernelGGL((range_fwd_k<DHP, MOD>), dim3((unsigned)((i64)cdiv(a.Tq, 128) * a.H)), dim3(256), smem, s, a);
}
size_t range_few_floats(const RangeAttn& a) { return few_floats(a); }
void launch_range_fwd_flash(const RangeAttn& a, float* work, int form, hipStream_t s) {
  if (a.Tq <= 0) return;
#define FWD(W, M) fwd<W, M>(a, work, form, s)
  BY_FORM(FWD);
}
void launch_range_bwd_flash(const RangeAttn& a, void* blocks, float* sums, int form, hipStream_t s) {
#define BWD(W, M) bwd<W, M>(a, blocks, sums, form, s)
  BY_FORM(BWD);
}
