// C entry points of the operators for attention layers: attention over key ranges, rotary positions, layer norm.  They check
// their arguments, lay out the caller's scratch memory and enqueue; nothing here allocates or waits.
#include "kernels.h"
#include "../../include/revffn.h"
#include <math.h>
#include <initializer_list>

#define TRY(x) do { int e_ = (x); if (e_) return e_; } while (0)

namespace {

// a launch's grid times its 256 threads has to stay below 2^32
bool grid_fits(i64 workgroups) { return workgroups < ((i64)1 << 24); }

struct Scratch { float *parts, *dvec; void* blocks; float* sums; size_t bytes; };
Scratch lay_out(const RangeAttn& a, bool backward, void* work) {
  Scratch w = {nullptr, nullptr, nullptr, nullptr, 0};
  auto take = [&](size_t n) { void* p = work ? (char*)work + w.bytes : nullptr; w.bytes += (n + 255) / 256 * 256; return p; };
  if (backward) {
    w.dvec = (float*)take((size_t)a.H * a.Tq * 4);
    w.blocks = take(((size_t)a.Tq + 63) / 64 * 16);
    if (a.dh <= 128) w.sums = (float*)take((a.dt == 1 ? range_flash_sum_floats(a) : range_f32_sum_floats(a)) * 4);
  } else if (a.dh <= 128) w.parts = (float*)take(range_few_floats(a) * 4);
  return w;
}

int check_desc(const revffn_attn_desc* d, RangeAttn* a) {
  if (!d) return REVFFN_ENULL;
  if ((d->dtype != 0 && d->dtype != 1) || d->kernel_mode < 0 || (d->kernel_mode & 0xff) > 2 || d->kernel_mode >> 8 > 2 || d->H < 1 || d->Hkv < 1 || d->H % d->Hkv ||
      d->H > 65536 || d->dh < 1 || d->dh > 512 || d->Tq < 0 || d->Tk < 0 || !(fabsf(d->scale) < INFINITY) || !(d->softcap >= 0.f) ||
      !(d->softcap < INFINITY))
    return REVFFN_EINVAL;
  const i64 wq = (i64)d->H * d->dh, wk = (i64)d->Hkv * d->dh;
  *a = RangeAttn{};
  a->dt = d->dtype; a->H = d->H; a->Hkv = d->Hkv; a->G = d->H / d->Hkv; a->dh = d->dh; a->Tq = d->Tq; a->Tk = d->Tk;
  a->ldq = d->ldq ? d->ldq : wq; a->ldk = d->ldk ? d->ldk : wk; a->ldv = d->ldv ? d->ldv : wk; a->ldo = d->ldo ? d->ldo : wq;
  if (a->ldq < wq || a->ldo < wq || a->ldk < wk || a->ldv < wk) return REVFFN_ESHAPE;
  if (!grid_fits(((i64)d->Tq + 3) / 4 * d->H) || !grid_fits(((i64)d->Tk + 3) / 4 * d->Hkv)) return REVFFN_ESHAPE;
  a->scale = d->scale != 0.f ? d->scale : 1.0f / sqrtf((float)d->dh);
  a->cap = d->softcap;
  if (a->cap > 0.f && !(fabsf(a->scale) / a->cap < 1e30f)) return REVFFN_EINVAL;      // (q.k scale / cap would overflow)
  a->slopes = d->slopes;
  return 0;
}
int check_mask(const revffn_attn_mask* m, RangeAttn* a) {
  if (!m || (a->Tq > 0 && (!m->lo || !m->hi))) return REVFFN_ENULL;
  a->lo = m->lo; a->hi = m->hi; a->at = m->at; a->used = m->used;
  return 0;
}
// whether a result starts where an input or another result does (results first, rows > 0 of them)
bool same_place(std::initializer_list<const void*> results, std::initializer_list<const void*> inputs) {
  for (auto r = results.begin(); r != results.end(); r++) {
    for (auto other = r + 1; other != results.end(); other++) if (*r && *r == *other) return true;
    for (const void* in : inputs) if (*r && *r == in) return true;
  }
  return false;
}
int frequencies(const revffn_rotary* r, double* f) {
  if (!r || !f) return REVFFN_ENULL;
  if (r->dims < 2 || r->dims > ROTARY_MAX_DIMS || r->dims % 2 || (r->interleaved != 0 && r->interleaved != 1) || r->scaling < 0 || r->scaling > 3 ||
      !(r->theta > 0.f) || !(r->theta < INFINITY) || !(fabsf(r->magnitude) < INFINITY))
    return REVFFN_EINVAL;
  if (r->scaling && (!(r->factor > 0.f) || !(r->factor < INFINITY))) return REVFFN_EINVAL;
  if (r->scaling == 2 && r->dims == 2) return REVFFN_EINVAL;
  if (r->scaling == 3 && (r->original < 1 || !(r->few_turns >= 0.f) || !(r->many_turns > r->few_turns) || !(r->many_turns < INFINITY)))
    return REVFFN_EINVAL;
  const int n = r->dims;
  double theta = r->theta;
  if (r->scaling == 2) theta *= pow((double)r->factor, (double)n / (n - 2));
  // (every call works them out: by products, off by n / 2 half steps of 64 bits at the last, whose angles are the smallest)
  const double ratio = pow(theta, -2.0 / n);
  double next = 1.0;
  for (int i = 0; i < n / 2; i++) {
    double v = next;
    next *= ratio;
    if (r->scaling == 1) v /= r->factor;
    if (r->scaling == 3) {
      double g = (r->original * v / (2 * M_PI) - r->few_turns) / ((double)r->many_turns - r->few_turns);
      g = g < 0 ? 0 : g > 1 ? 1 : g;
      v = g * v + (1 - g) * v / r->factor;
    }
    f[i] = v;
  }
  return 0;
}

}  // namespace

extern "C" {

int revffn_op_attention_ranges(const int32_t* cu_q, const int32_t* cu_k, const int32_t* prefix, int32_t n_docs, int32_t causal,
                               int32_t window, int32_t Tq, int32_t Tk, int32_t* lo, int32_t* hi, int32_t* at, int32_t* used, void* stream) {
  if (Tq > 0 && (!lo || !hi)) return REVFFN_ENULL;
  if (n_docs < 1 || n_docs == INT32_MAX || (causal != 0 && causal != 1) || window < 0 || Tq < 0 || Tk < 0 || (prefix && window) || (!causal && (prefix || window)))
    return REVFFN_EINVAL;
  if ((!cu_q && Tq % n_docs) || (!cu_q && !cu_k && Tk % n_docs)) return REVFFN_ESHAPE;
  if (Tq > 0 || used) launch_attn_ranges(cu_q, cu_k, prefix, n_docs, causal, window, Tq, Tk, lo, hi, at, used, (hipStream_t)stream);
  return 0;
}

size_t revffn_op_attention_masked_workspace(const revffn_attn_desc* desc, int32_t backward) {
  RangeAttn a;
  if (check_desc(desc, &a)) return 0;
  const size_t f = lay_out(a, false, nullptr).bytes, b = backward ? lay_out(a, true, nullptr).bytes : 0;
  return f > b ? f : b;
}

int revffn_op_attention_masked_fwd(const revffn_attn_desc* desc, const revffn_attn_mask* mask, const void* q, const void* k, const void* v,
                                   void* o, float* lse, void* work, size_t work_bytes, void* stream) {
  RangeAttn a;
  TRY(check_desc(desc, &a));
  TRY(check_mask(mask, &a));
  if ((a.Tq > 0 && (!q || !o)) || (a.Tk > 0 && (!k || !v))) return REVFFN_ENULL;
  const Scratch w = lay_out(a, false, work);
  if (w.bytes && !work) return REVFFN_ENULL;
  if (w.bytes > work_bytes || ((uintptr_t)work & 15)) return REVFFN_EINVAL;
  a.q = q; a.k = k; a.v = v; a.out = o; a.lse = lse;
  const int mode = desc->kernel_mode & 0xff, form = desc->kernel_mode >> 8;
  const bool flash = mode != 1 && range_flash_takes(a, false), f32 = mode != 1 && range_f32_takes(a, false);
  if (mode == 2 && !flash && !f32) return REVFFN_EUNSUPPORTED;
  if (a.Tq > 0 && same_place({o, lse}, {q, k, v})) return REVFFN_EINVAL;
  if (flash) launch_range_fwd_flash(a, w.parts, form, (hipStream_t)stream);
  else if (f32) launch_range_fwd_f32(a, w.parts, (hipStream_t)stream);
  else launch_range_fwd_rows(a, (hipStream_t)stream);
  return 0;
}

int revffn_op_attention_masked_bwd(const revffn_attn_desc* desc, const revffn_attn_mask* mask, const void* q, const void* k, const void* v,
                                   const void* o, const void* d_o, const float* lse, void* dq, void* dk, void* dv, void* work,
                                   size_t work_bytes, void* stream) {
  RangeAttn a;
  TRY(check_desc(desc, &a));
  TRY(check_mask(mask, &a));
  if ((a.Tq > 0 && (!q || !o || !d_o || !lse || !dq)) || (a.Tk > 0 && (!k || !v || !dk || !dv))) return REVFFN_ENULL;
  const Scratch w = lay_out(a, true, work);
  if (w.bytes && !work) return REVFFN_ENULL;
  if (w.bytes > work_bytes || ((uintptr_t)work & 15)) return REVFFN_EINVAL;
  a.q = q; a.k = k; a.v = v; a.o = o; a.d_o = d_o; a.lse = (float*)lse; a.dq = dq; a.dk = dk; a.dv = dv; a.dvec = w.dvec;
  const int mode = desc->kernel_mode & 0xff, form = desc->kernel_mode >> 8;
  const bool flash = mode != 1 && range_flash_takes(a, true), f32 = mode != 1 && range_f32_takes(a, true);
  if (mode == 2 && !flash && !f32) return REVFFN_EUNSUPPORTED;
  // (dk and dv are worked out after dq, from q, o's D, d_o and lse)
  if (same_place({a.Tq > 0 ? dq : nullptr, a.Tk > 0 ? dk : nullptr, a.Tk > 0 ? dv : nullptr}, {q, k, v, o, d_o, lse})) return REVFFN_EINVAL;
  if (flash) launch_range_bwd_flash(a, w.blocks, w.sums, form, (hipStream_t)stream);
  else if (f32) launch_range_bwd_f32(a, w.blocks, w.sums, (hipStream_t)stream);
  else launch_range_bwd_rows(a, (hipStream_t)stream);
  return 0;
}

int revffn_op_rotary_frequencies(const revffn_rotary* r, double* freqs) { return frequencies(r, freqs); }

int revffn_op_rotary(int32_t dtype, const revffn_rotary* r, const void* x, void* y, const int32_t* pos, int32_t T, int32_t S, int32_t H,
                     int32_t dh, int64_t ldx, int64_t ldy, int32_t transposed, void* stream) {
  RotaryArgs a;
  if (!r || (T > 0 && (!x || !y))) return REVFFN_ENULL;
  if ((dtype != 0 && dtype != 1) || T < 0 || (!pos && S < 1) || H < 1 || dh < 2 || dh > 1024 || H > 65536 || (transposed != 0 && transposed != 1))
    return REVFFN_EINVAL;
  TRY(frequencies(r, a.freq));
  if (r->dims > dh) return REVFFN_EINVAL;
  // (the kernel's division of a row into heads is exact up to 2^22 columns)
  if (ldx < (i64)H * dh || ldy < (i64)H * dh || (i64)H * dh > (1 << 22) || !grid_fits(T) || (x == y && ldx != ldy)) return REVFFN_ESHAPE;
  if (T == 0) return 0;
  a.x = x; a.y = y; a.pos = pos; a.dt = dtype; a.T = T; a.S = S < 1 ? 1 : S; a.H = H; a.dh = dh; a.dims = r->dims; a.interleaved = r->interleaved;
  a.ldx = ldx; a.ldy = ldy;
  a.mag = r->magnitude != 0.f ? r->magnitude : 1.f;
  a.sign = transposed ? -1.f : 1.f;
  for (int i = 0; i < r->dims / 2; i++) a.freq[i] /= 2 * M_PI;
  launch_rotary(a, (hipStream_t)stream);
  return 0;
}

size_t revffn_op_layernorm_workspace(int32_t rows, int32_t cols) {
  return rows < 0 || cols < 1 ? 0 : layernorm_partial_floats(rows, cols) * 4;
}

int revffn_op_layernorm_fwd(int32_t dtype, const void* x, const void* gain, const void* bias, void* y, float* mean, float* rstd, int32_t rows,
                            int32_t cols, int64_t ldx, int64_t ldy, float eps, void* stream) {
  if (rows > 0 && (!x || !y)) return REVFFN_ENULL;
  if ((dtype != 0 && dtype != 1) || rows < 0 || cols < 1 || cols > (1 << 24) || !(eps >= 0.f) || !(eps < INFINITY)) return REVFFN_EINVAL;
  if (ldx < cols || ldy < cols || (x == y && ldx != ldy) || !grid_fits(4 * (i64)rows)) return REVFFN_ESHAPE;
  LayerNorm a = {};
  a.x = x; a.gain = gain; a.bias = bias; a.y = y; a.mean = mean; a.rstd = rstd; a.dt = dtype; a.rows = rows; a.cols = cols; a.ldx = ldx; a.ldy = ldy;
  a.eps = eps;
  launch_layernorm_fwd(a, (hipStream_t)stream);
  return 0;
}

int revffn_op_layernorm_bwd(int32_t dtype, const void* dy, const void* x, const void* gain, const float* mean, const float* rstd, void* dx,
                            void* dgain, void* dbias, int32_t rows, int32_t cols, int64_t lddy, int64_t ldx, int64_t lddx, int32_t grads_f32,
                            void* work, size_t work_bytes, void* stream) {
  if (rows > 0 && (!dy || !x || !mean || !rstd || !dx)) return REVFFN_ENULL;
  if ((dtype != 0 && dtype != 1) || rows < 0 || cols < 1 || cols > (1 << 24) || (grads_f32 != 0 && grads_f32 != 1)) return REVFFN_EINVAL;
  if (ldx < cols || lddy < cols || lddx < cols || (dy == dx && lddy != lddx) || !grid_fits(4 * (i64)rows)) return REVFFN_ESHAPE;
  if (rows > 0 && dx == x) return REVFFN_EINVAL;                // (x is read again for the sums)
  if (dgain || dbias) {
    if (!work) return REVFFN_ENULL;
    if (work_bytes < revffn_op_layernorm_workspace(rows, cols) || ((uintptr_t)work & 15)) return REVFFN_EINVAL;
  }
  LayerNorm a = {};
  a.dy = dy; a.x = x; a.gain = gain; a.mean = (float*)mean; a.rstd = (float*)rstd; a.dx = dx; a.dgain = dgain; a.dbias = dbias; a.dt = dtype;
  a.rows = rows; a.cols = cols; a.lddy = lddy; a.ldx = ldx; a.lddx = lddx; a.grads_f32 = grads_f32; a.partial = (float*)work;
  launch_layernorm_bwd(a, (hipStream_t)stream);
  return 0;
}

}  // extern "C"
