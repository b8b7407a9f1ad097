// LayerNorm forward and backward.  A row's values stay in registers between the passes over it (mean, variance about that mean,
// result), so memory is read once and written once, which is what bounds it.
//   y = (x - mean) rstd g + b;    dx = rstd (d - mean(d) - xh mean(d xh)) with d = dy g, xh = (x - mean) rstd;
//   dg = sum over rows of dy xh, db = of dy: every wave (workgroup) keeps the sums of the rows it works on in registers; one
//   partial sum per workgroup goes to memory, and a second launch adds those in order.
// bf16, 8192 rows of 2048: forward 14 us (4.8 TB/s), backward 25 (4.0) and 4.8 for the sums.
// Columns of a thread: chunks of 8 neighbours, chunk n at column 8 (thread + n threads): the same whatever the alignment, so the
// result does not depend on where the rows lie; rows are read 16 bytes at a time wherever they start, the last
// few columns of an odd row one by one.
#include "kernels.h"

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_v;
typedef __attribute__((ext_vector_type(8))) float f32x8_v;
// the same, at any element's address (the hardware takes unaligned 16-byte accesses)
typedef bf16x8_v bf16x8_any __attribute__((aligned(2)));
typedef f32x8_v f32x8_any __attribute__((aligned(4)));
typedef f32x8_v f32x8_16 __attribute__((aligned(16)));
template <class T, bool ALIGNED> struct Vec8;
template <> struct Vec8<bf16, true> { typedef bf16x8_v type; };
template <> struct Vec8<bf16, false> { typedef bf16x8_any type; };
template <> struct Vec8<float, true> { typedef f32x8_16 type; };
template <> struct Vec8<float, false> { typedef f32x8_any type; };

// 8 columns, of which `left` are there (the others read as 0)
template <bool ALIGNED, class T> __device__ __forceinline__ void load8(const T* p, int left, float (&r)[8]) {
  if (ALIGNED || left >= 8) {
    const auto v = *(const typename Vec8<T, ALIGNED>::type*)p;
#pragma unroll
    for (int i = 0; i < 8; i++) r[i] = (float)v[i];
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++) r[i] = i < left ? (float)p[i] : 0.f;
  }
}
template <bool ALIGNED, class T> __device__ __forceinline__ void store8(T* p, int left, const float (&r)[8]) {
  if (ALIGNED || left >= 8) {
    typename Vec8<T, ALIGNED>::type v;
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = (T)r[i];
    *(typename Vec8<T, ALIGNED>::type*)p = v;
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++) if (i < left) p[i] = (T)r[i];
  }
}
// the same as they are in memory: the next row's are on their way while a row is worked on
template <class T, bool ALIGNED> struct Raw8 {
  typename Vec8<T, true>::type v;
  __device__ __forceinline__ void load(const T* p, int left) {
    if (ALIGNED || left >= 8) v = *(const typename Vec8<T, ALIGNED>::type*)p;
    else {
#pragma unroll
      for (int i = 0; i < 8; i++) v[i] = i < left ? p[i] : (T)0.f;
    }
  }
  __device__ __forceinline__ void get(float (&r)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; i++) r[i] = (float)v[i];
  }
};

// the sum over the WAVES waves that work on a row, in every thread of them; red: 2 * WAVES floats, which two sums use by turns
template <int WAVES> __device__ __forceinline__ float row_sum(float v, float* red) {
  v = wave_sum(v);
  if constexpr (WAVES == 1) return v;
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  float s = 0.f;
#pragma unroll
  for (int w = 0; w < WAVES; w++) s += red[w];
  return s;
}

// WAVES waves per row, CH chunks of 8 columns per thread in registers.  CH = 0: rows longer than that, read once per pass.
template <class T, bool ALIGNED, int WAVES, int CH>
__global__ void __launch_bounds__(WAVES == 1 ? 256 : WAVES * 64) layernorm_fwd_k(LayerNorm a) {
  constexpr int NT = WAVES * 64, ROWS = WAVES == 1 ? 4 : 1;
  __shared__ float red[3][WAVES];
  const int row = (int)blockIdx.x * ROWS + (ROWS == 4 ? (int)(threadIdx.x >> 6) : 0), tid = ROWS == 4 ? threadIdx.x & 63 : threadIdx.x;
  if (row >= a.rows) return;
  const T* x = (const T*)a.x + (i64)row * a.ldx;
  T* y = (T*)a.y + (i64)row * a.ldy;
  const T *g = (const T*)a.gain, *b = (const T*)a.bias;
  const int cols = a.cols;
  const float n = (float)cols;
  float mean, rstd;
  auto write = [&](int c, const float (&v)[8]) {
    float gv[8], bv[8], o[8];
    if (g) load8<ALIGNED>(g + c, cols - c, gv);
    if (b) load8<ALIGNED>(b + c, cols - c, bv);
#pragma unroll
    for (int i = 0; i < 8; i++) {
      o[i] = (v[i] - mean) * rstd;
      if (g) o[i] *= gv[i];
      if (b) o[i] += bv[i];
    }
    store8<ALIGNED>(y + c, cols - c, o);
  };
  if constexpr (CH > 0) {
    float v[CH][8];
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < CH; k++) {
      const int c = (tid + k * NT) * 8;
      if (c < cols) load8<ALIGNED>(x + c, cols - c, v[k]);
      else {
#pragma unroll
        for (int i = 0; i < 8; i++) v[k][i] = 0.f;
      }
#pragma unroll
      for (int i = 0; i < 8; i++) s += v[k][i];
    }
    mean = row_sum<WAVES>(s, red[0]) / n;
    float q = 0.f;
#pragma unroll
    for (int k = 0; k < CH; k++) {
      const int c = (tid + k * NT) * 8;
#pragma unroll
      for (int i = 0; i < 8; i++) if (ALIGNED ? c < cols : c + i < cols) q += (v[k][i] - mean) * (v[k][i] - mean);
    }
    rstd = 1.0f / sqrtf(row_sum<WAVES>(q, red[1]) / n + a.eps);
#pragma unroll
    for (int k = 0; k < CH; k++) {
      const int c = (tid + k * NT) * 8;
      if (c < cols) write(c, v[k]);
    }
  } else {
    float s = 0.f, q = 0.f, v[8];
    for (int c = tid * 8; c < cols; c += NT * 8) {
      load8<ALIGNED>(x + c, cols - c, v);
#pragma unroll
      for (int i = 0; i < 8; i++) s += v[i];
    }
    mean = row_sum<WAVES>(s, red[0]) / n;
    for (int c = tid * 8; c < cols; c += NT * 8) {
      load8<ALIGNED>(x + c, cols - c, v);
#pragma unroll
      for (int i = 0; i < 8; i++) if (ALIGNED || c + i < cols) q += (v[i] - mean) * (v[i] - mean);
    }
    rstd = 1.0f / sqrtf(row_sum<WAVES>(q, red[1]) / n + a.eps);
    for (int c = tid * 8; c < cols; c += NT * 8) {
      load8<ALIGNED>(x + c, cols - c, v);
      write(c, v);
    }
  }
  if (tid == 0) {
    if (a.mean) a.mean[row] = mean;
    if (a.rstd) a.rstd[row] = rstd;
  }
}

// Row r of workgroup w: w, w + grid, ..  PARAMS: partial sums of dg and db, [workgroup][2][columns].  CH = 0: rows longer than the registers hold;
// dg and db then come from a kernel of their own.
template <class T, bool ALIGNED, int WAVES, int CH, bool PARAMS>
__global__ void __launch_bounds__(WAVES == 1 ? 256 : WAVES * 64) layernorm_bwd_k(LayerNorm a) {
  constexpr int NT = WAVES * 64, ROWS = WAVES == 1 ? 4 : 1, C = CH > 0 ? CH : 1;
  __shared__ float red[4][WAVES];
  extern __shared__ float sums[];                    // WAVES == 1: [4][C * 512]
  const int wv = threadIdx.x >> 6, tid = ROWS == 4 ? threadIdx.x & 63 : threadIdx.x;
  const T* g = (const T*)a.gain;
  const int cols = a.cols;
  const float n = (float)cols;
  float dg[C][8] = {}, db[C][8] = {};
  int turn = 0;
  i64 row = (i64)blockIdx.x * ROWS + (ROWS == 4 ? wv : 0);
  const i64 step = (i64)gridDim.x * ROWS;
  Raw8<T, ALIGNED> rx[C], rd[C];
  float mean_next = 0.f, rstd_next = 0.f;
  auto fetch = [&](i64 r) {
    if (r >= a.rows) return;
    mean_next = a.mean[r];
    rstd_next = a.rstd[r];
    if constexpr (CH > 0) {
      const T *x = (const T*)a.x + r * a.ldx, *dy = (const T*)a.dy + r * a.lddy;
#pragma unroll
      for (int k = 0; k < C; k++) {
        const int c = (tid + k * NT) * 8;
        if (c < cols) {
          rx[k].load(x + c, cols - c);
          rd[k].load(dy + c, cols - c);
        }
      }
    }
  };
  fetch(row);
  for (; row < a.rows; row += step) {
    const T *x = (const T*)a.x + row * a.ldx, *dy = (const T*)a.dy + row * a.lddy;
    T* dx = (T*)a.dx + row * a.lddx;
    const float mean = mean_next, rstd = rstd_next;
    float s = 0.f, q = 0.f;
    if constexpr (CH > 0) {
      float xh[CH][8], d[CH][8];
#pragma unroll
      for (int k = 0; k < CH; k++) {
        const int c = (tid + k * NT) * 8;
        if (c < cols) {
          rx[k].get(xh[k]);
          rd[k].get(d[k]);
        }
      }
      fetch(row + step);
#pragma unroll
      for (int k = 0; k < CH; k++) {
        const int c = (tid + k * NT) * 8;
        if (c < cols) {
          float gv[8];
          if (g) load8<ALIGNED>(g + c, cols - c, gv);
#pragma unroll
          for (int i = 0; i < 8; i++) {
            xh[k][i] = (xh[k][i] - mean) * rstd;
            if (!ALIGNED && c + i >= cols) xh[k][i] = 0.f;
            if (PARAMS) { dg[k][i] = fmaf(d[k][i], xh[k][i], dg[k][i]); db[k][i] += d[k][i]; }
            if (g) d[k][i] *= gv[i];
            s += d[k][i];
            q = fmaf(d[k][i], xh[k][i], q);
          }
        }
      }
      s = row_sum<WAVES>(s, red[turn]) / n;
      q = row_sum<WAVES>(q, red[turn + 1]) / n;
#pragma unroll
      for (int k = 0; k < CH; k++) {
        const int c = (tid + k * NT) * 8;
        if (c < cols) {
          float o[8];
#pragma unroll
          for (int i = 0; i < 8; i++) o[i] = rstd * (d[k][i] - s - xh[k][i] * q);
          store8<ALIGNED>(dx + c, cols - c, o);
        }
      }
    } else {
      float v[8], d[8], gv[8];
      auto part = [&](int c) {
        load8<ALIGNED>(x + c, cols - c, v);
        load8<ALIGNED>(dy + c, cols - c, d);
        if (g) load8<ALIGNED>(g + c, cols - c, gv);
#pragma unroll
        for (int i = 0; i < 8; i++) {
          v[i] = (v[i] - mean) * rstd;
          if (!ALIGNED && c + i >= cols) v[i] = 0.f;
          if (g) d[i] *= gv[i];
        }
      };
      for (int c = tid * 8; c < cols; c += NT * 8) {
        part(c);
#pragma unroll
        for (int i = 0; i < 8; i++) { s += d[i]; q = fmaf(d[i], v[i], q); }
      }
      s = row_sum<WAVES>(s, red[turn]) / n;
      q = row_sum<WAVES>(q, red[turn + 1]) / n;
      for (int c = tid * 8; c < cols; c += NT * 8) {
        part(c);
#pragma unroll
        for (int i = 0; i < 8; i++) d[i] = rstd * (d[i] - s - v[i] * q);
        store8<ALIGNED>(dx + c, cols - c, d);
      }
      fetch(row + step);
    }
    turn ^= 2;                                       // (a slow wave may still read the last row's sums)
  }
  if constexpr (PARAMS && CH > 0) {
    // In the threads' own order, value i of chunk k at (8 k + i) NT + thread: whole lines to LDS and to memory; the last kernel knows
    // which column that is.
    float* out = a.partial + (i64)blockIdx.x * 2 * (C * 8 * NT);
    if constexpr (ROWS == 4) {                       // the four waves' sums, in wave order
#pragma unroll
      for (int w = 0; w < 2; w++) {
        __syncthreads();
#pragma unroll
        for (int k = 0; k < C; k++)
#pragma unroll
          for (int i = 0; i < 8; i++) sums[(wv * C * 8 + k * 8 + i) * 64 + tid] = w ? db[k][i] : dg[k][i];
        __syncthreads();
#pragma unroll
        for (int p = 0; p < C * 2; p++) {
          const int at = p * 256 + (int)threadIdx.x;
          out[w * C * 512 + at] = (sums[at] + sums[C * 512 + at]) + (sums[2 * C * 512 + at] + sums[3 * C * 512 + at]);
        }
      }
    } else {
#pragma unroll
      for (int k = 0; k < C; k++)
#pragma unroll
        for (int i = 0; i < 8; i++) { out[(k * 8 + i) * NT + tid] = dg[k][i]; out[(C * 8 + k * 8 + i) * NT + tid] = db[k][i]; }
    }
  }
}
// the same partial sums for rows that are longer than the registers hold: 64 columns and a share of the rows per workgroup
template <class T> __global__ void __launch_bounds__(256) layernorm_params_k(LayerNorm a) {
  __shared__ float part[2][4][64];
  const int c = (int)blockIdx.x * 64 + (threadIdx.x & 63), w = threadIdx.x >> 6;
  float dg = 0.f, db = 0.f;
  if (c < a.cols)
    for (i64 row = (i64)blockIdx.y * 4 + w; row < a.rows; row += (i64)gridDim.y * 4) {
      const float d = to_f(((const T*)a.dy)[row * a.lddy + c]);
      dg = fmaf(d, (to_f(((const T*)a.x)[row * a.ldx + c]) - a.mean[row]) * a.rstd[row], dg);
      db += d;
    }
  part[0][w][threadIdx.x & 63] = dg;
  part[1][w][threadIdx.x & 63] = db;
  __syncthreads();
  if (w > 1 || c >= a.cols) return;
  const float* p = &part[w][0][threadIdx.x & 63];
  a.partial[((i64)blockIdx.y * 2 + w) * a.cols + c] = (p[0] + p[64]) + (p[128] + p[192]);
}
// 16 values of one of the two sums per workgroup, 16 threads to a value, each every 16th of the partial sums.  threads: of the
// kernel that left them in its threads' order, `padded` values of each; 0: in the order of the columns
template <class T> __global__ void __launch_bounds__(256) layernorm_reduce_k(const float* __restrict__ partial, int n, int cols, int padded, int threads, T* dgain, T* dbias) {
  __shared__ float part[16][17];
  const int tc = threadIdx.x & 15, w = threadIdx.x >> 4, at = (int)blockIdx.x * 16 + tc;
  T* out = blockIdx.y ? dbias : dgain;
  if (!out) return;
  int c = at;
  if (threads) {
    const int v = at / threads, t = at - v * threads;
    c = (t + (v >> 3) * threads) * 8 + (v & 7);
  }
  float s = 0.f;
  if (at < padded && c < cols) {
    const float* p = partial + (i64)blockIdx.y * padded + at;
#pragma unroll 8
    for (int i = w; i < n; i += 16) s += p[(i64)i * 2 * padded];
  }
  part[w][tc] = s;
  __syncthreads();
  if (w == 0 && at < padded && c < cols) {
#pragma unroll
    for (int i = 1; i < 16; i++) s += part[i][tc];
    out[c] = from_f<T>(s);
  }
}

// Waves per row, 8-column chunks per thread and (backward) workgroups, each of which leaves partial sums of whole rows: more of them keep
// more rows in flight, but the sums cost each 4 KiB per wave of a row and chunk of traffic twice and a few microseconds at its end.  Backward with its sums, us,
// by workgroups (bf16 unless said; w4: with four waves to a row instead, w16: sixteen):
//   8192 x 512   256, 512, 1024, 2048: 14.0 13.3 14.9 19.2, w4 20.7   32768 x 256: 45.9 31.4 24.8 29.8, w4 52.9
//   8192 x 1024  256, 512, 1024: 21.0 19.6 20.7, w4 33.0 and more     2000 x 1024: 11.3 13.2 13.2
//   8192 x 2048  128, 256, 512: 48.7 32.8 31.1, w4 33.0               2000 x 2048: 16.1 14.5 17.6   float32 67.5 49.2 51.0, w4 45.7
//   8192 x 4096  256, 512, 1024: 82.8 60.0 56.8, w16 68.4             2000 x 4096: 27.6 23.9 29.1   float32 98.8 86.8 98.3
//   8192 x 8192  256, 512, 1024: 135.5 102.0 116.6, w16 109.3         2000 x 8192: 43.2 40.6 55.5   float32 184.4 174.1 199.2, w16 164.1
//   2000 x 16384 128, 256, 512: 73.4 59.9 78.9, from memory for every pass 90.5                     float32 152.8 114.4 130.4
// Longer rows, which are read for every pass: 1000 x 32768 forward 38.8 (3.4 TB/s), backward 98.7; float32 84, 160.
struct Shape { int waves, chunks, parts; };
static Shape shape_of(int cols) {
  if (cols <= 512) return {1, 1, 1024};
  if (cols <= 1024) return {1, 2, 512};
  if (cols <= 2048) return {1, 4, 256};
  if (cols <= 4096) return {4, 2, 512};
  if (cols <= 8192) return {4, 4, 512};
  if (cols <= 16384) return {16, 2, 256};
  return {16, 0, 32};
}
static int padded_columns(int cols) { const Shape f = shape_of(cols); return f.chunks ? f.waves * f.chunks * 512 : cols; }
size_t layernorm_partial_floats(int rows, int cols) {
  const int n = shape_of(cols).parts;
  return (size_t)(rows < 1 ? 1 : rows < n ? rows : n) * 2 * padded_columns(cols);
}

static bool aligned(const LayerNorm& a, bool back) {
  const uintptr_t p = (uintptr_t)a.x | (uintptr_t)a.gain | (back ? (uintptr_t)a.dy | (uintptr_t)a.dx : (uintptr_t)a.y | (uintptr_t)a.bias);
  const i64 l = a.cols | a.ldx | (back ? a.lddy | a.lddx : a.ldy);
  return (p & 15) == 0 && (l & 7) == 0;
}
#define BY_COLS(call)                                   \
  do {                                                  \
    const Shape f = shape_of(a.cols);                   \
    if (f.waves == 1) { if (f.chunks == 1) call(1, 1); else if (f.chunks == 2) call(1, 2); else call(1, 4); } \
    else if (f.waves == 4) { if (f.chunks == 2) call(4, 2); else call(4, 4); } \
    else if (f.chunks) call(16, 2);                     \
    else call(16, 0);                                   \
  } while (0)

template <class T, bool AL> static void fwd(const LayerNorm& a, hipStream_t s) {
#define FWD(W, CH) hipLaunchKernelGGL((layernorm_fwd_k<T, AL, W, CH>), dim3(cdiv(a.rows, W == 1 ? 4 : 1)), dim3(W == 1 ? 256 : W * 64), 0, s, a)
  BY_COLS(FWD);
}
void launch_layernorm_fwd(const LayerNorm& a, hipStream_t s) {
  if (a.rows <= 0) return;
  const bool al = aligned(a, false);
  if (a.dt == 0) { if (al) fwd<float, true>(a, s); else fwd<float, false>(a, s); }
  else if (al) fwd<bf16, true>(a, s);
  else fwd<bf16, false>(a, s);
}
template <class T, bool AL, int W, int CH> static int bwd_one(const LayerNorm& a, bool params, hipStream_t s) {
  constexpr int ROWS = W == 1 ? 4 : 1;
  const dim3 block(W == 1 ? 256 : W * 64);
  int grid = cdiv(a.rows, ROWS);
  if constexpr (CH > 0) {
    if (params) {
      if (grid > shape_of(a.cols).parts) grid = shape_of(a.cols).parts;
      hipLaunchKernelGGL((layernorm_bwd_k<T, AL, W, CH, true>), dim3(grid), block, W == 1 ? (size_t)4 * CH * 512 * 4 : 0, s, a);
      return grid;
    }
  }
  const int n = a.rows < 4 * 32 ? cdiv(a.rows, 4) : 32;
  if (params) hipLaunchKernelGGL(layernorm_params_k<T>, dim3(cdiv(a.cols, 64), n), dim3(256), 0, s, a);      // (first: dx may be dy)
  hipLaunchKernelGGL((layernorm_bwd_k<T, AL, W, CH, false>), dim3(grid), block, 0, s, a);
  return params ? n : 0;
}
template <class T, bool AL> static int bwd(const LayerNorm& a, bool params, hipStream_t s) {
#define BWD(W, CH) return bwd_one<T, AL, W, CH>(a, params, s)
  BY_COLS(BWD);
}
void launch_layernorm_bwd(const LayerNorm& a, hipStream_t s) {
  const bool al = aligned(a, true), params = a.dgain || a.dbias;
  int n = 0;
  if (a.rows > 0) {
    if (a.dt == 0) n = al ? bwd<float, true>(a, params, s) : bwd<float, false>(a, params, s);
    else n = al ? bwd<bf16, true>(a, params, s) : bwd<bf16, false>(a, params, s);
  }
  if (!params) return;
  const Shape f = shape_of(a.cols);
  const int padded = padded_columns(a.cols), threads = f.chunks ? f.waves * 64 : 0;
  const dim3 grid(cdiv(padded, 16), 2);
  if (a.dt == 0 || a.grads_f32) hipLaunchKernelGGL(layernorm_reduce_k<float>, grid, dim3(256), 0, s, a.partial, n, a.cols, padded, threads, (float*)a.dgain, (float*)a.dbias);
  else hipLaunchKernelGGL(layernorm_reduce_k<bf16>, grid, dim3(256), 0, s, a.partial, n, a.cols, padded, threads, (bf16*)a.dgain, (bf16*)a.dbias);
}
