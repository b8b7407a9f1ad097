// LayerNorm forward and backward.  A row's values stay in registers between the passes over it (mean, variance about that mean,
// result), so memory is read once and written once, which is what bounds it.
//   y = (x - mean) rstd g + b;    dx = rstd (d - mean(d) - xh mean(d xh)) with d = dy g, xh = (x - mean) rstd;
//   dg = sum over rows of dy xh, db = of dy: every wave (workgroup) keeps the sums of the rows it works on in registers; one
//   partial sum per workgroup goes to memory, and a second launch adds those in order.
// Columns of a thread: chunks of 8 neighbours, chunk n at column 8 (thread + n threads): the same whatever the alignment, so the
// result does not depend on where the rows lie; aligned rows are read 16 bytes at a time, others element by element.
#include "kernels.h"

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_v;

template <bool ALIGNED> __device__ __forceinline__ void load8(const bf16* p, int left, float (&r)[8]) {
  if constexpr (ALIGNED) {
    const bf16x8_v v = *(const bf16x8_v*)p;
#pragma unroll
    for (int i = 0; i < 8; i++) r[i] = (float)v[i];
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++) r[i] = i < left ? (float)p[i] : 0.f;
  }
}
template <bool ALIGNED> __device__ __forceinline__ void load8(const float* p, int left, float (&r)[8]) {
  if constexpr (ALIGNED) {
    const float4 u = *(const float4*)p, v = *(const float4*)(p + 4);
    r[0] = u.x; r[1] = u.y; r[2] = u.z; r[3] = u.w; r[4] = v.x; r[5] = v.y; r[6] = v.z; r[7] = v.w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++) r[i] = i < left ? p[i] : 0.f;
  }
}
template <bool ALIGNED> __device__ __forceinline__ void store8(bf16* p, int left, const float (&r)[8]) {
  if constexpr (ALIGNED) {
    bf16x8_v v;
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = (__bf16)r[i];
    *(bf16x8_v*)p = v;
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++) if (i < left) p[i] = (__bf16)r[i];
  }
}
template <bool ALIGNED> __device__ __forceinline__ void store8(float* p, int left, const float (&r)[8]) {
  if constexpr (ALIGNED) {
    *(float4*)p = make_float4(r[0], r[1], r[2], r[3]);
    *(float4*)(p + 4) = make_float4(r[4], r[5], r[6], r[7]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++) if (i < left) p[i] = r[i];
  }
}

// 8 columns as they are in memory: the next row's are on their way while a row is worked on
template <class T, bool ALIGNED> struct Raw8;
template <> struct Raw8<bf16, true> {
  bf16x8_v v;
  __device__ __forceinline__ void load(const bf16* p, int) { v = *(const bf16x8_v*)p; }
  __device__ __forceinline__ void get(float (&r)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; i++) r[i] = (float)v[i];
  }
};
template <> struct Raw8<float, true> {
  float4 u, v;
  __device__ __forceinline__ void load(const float* p, int) { u = *(const float4*)p; v = *(const float4*)(p + 4); }
  __device__ __forceinline__ void get(float (&r)[8]) const { r[0] = u.x; r[1] = u.y; r[2] = u.z; r[3] = u.w; r[4] = v.x; r[5] = v.y; r[6] = v.z; r[7] = v.w; }
};
template <class T> struct Raw8<T, false> {
  T v[8];
  __device__ __forceinline__ void load(const T* p, int left) {
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = i < left ? p[i] : (T)0.f;
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

// Row r of workgroup w: w, w + grid, ..  PARAMS: partial sums of dg and db, [workgroup][2][cols].  CH = 0: rows longer than the registers hold;
// dg and db then come from a kernel of their own.
template <class T, bool ALIGNED, int WAVES, int CH, bool PARAMS>
__global__ void __launch_bounds__(WAVES == 1 ? 256 : WAVES * 64) layernorm_bwd_k(LayerNorm a) {
  constexpr int NT = WAVES * 64, ROWS = WAVES == 1 ? 4 : 1, C = CH > 0 ? CH : 1;
  __shared__ float red[4][WAVES];
  extern __shared__ float sums[];                    // WAVES == 1: [3][2][C * 512]
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
    float* out = a.partial + (i64)blockIdx.x * 2 * cols;
    if constexpr (ROWS == 4) {                       // the four waves' sums, in wave order
      float* mine = sums + (wv - 1) * 2 * C * 512;
      if (wv > 0) {
#pragma unroll
        for (int k = 0; k < C; k++)
#pragma unroll
          for (int i = 0; i < 8; i++) { mine[(k * 8 + i) * 64 + tid] = dg[k][i]; mine[C * 512 + (k * 8 + i) * 64 + tid] = db[k][i]; }
      }
      __syncthreads();
      if (wv > 0) return;
#pragma unroll
      for (int w = 0; w < 3; w++)
#pragma unroll
        for (int k = 0; k < C; k++)
#pragma unroll
          for (int i = 0; i < 8; i++) {
            dg[k][i] += sums[w * 2 * C * 512 + (k * 8 + i) * 64 + tid];
            db[k][i] += sums[w * 2 * C * 512 + C * 512 + (k * 8 + i) * 64 + tid];
          }
    }
#pragma unroll
    for (int k = 0; k < C; k++) {
      const int c = (tid + k * NT) * 8;
#pragma unroll
      for (int i = 0; i < 8; i++) if (c + i < cols) { out[c + i] = dg[k][i]; out[cols + c + i] = db[k][i]; }
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
// 16 columns of one of the two sums per workgroup, 16 threads to a column, each every 16th of the partial sums
template <class T> __global__ void __launch_bounds__(256) layernorm_reduce_k(const float* __restrict__ partial, int n, int cols, T* dgain, T* dbias) {
  __shared__ float part[16][17];
  const int tc = threadIdx.x & 15, w = threadIdx.x >> 4, c = (int)blockIdx.x * 16 + tc;
  T* out = blockIdx.y ? dbias : dgain;
  if (!out) return;
  float s = 0.f;
  if (c < cols) {
    const float* p = partial + (i64)blockIdx.y * cols + c;
#pragma unroll 8
    for (int i = w; i < n; i += 16) s += p[(i64)i * 2 * cols];
  }
  part[w][tc] = s;
  __syncthreads();
  if (w == 0 && c < cols) {
#pragma unroll
    for (int i = 1; i < 16; i++) s += part[i][tc];
    out[c] = from_f<T>(s);
  }
}

// partial sums: one per workgroup of the backward kernel
#define MAX_PARTS 512
size_t layernorm_partial_floats(int rows, int cols) { return (size_t)(rows < 1 ? 1 : rows < MAX_PARTS ? rows : MAX_PARTS) * 2 * cols; }

static bool aligned(const LayerNorm& a, bool back) {
  const uintptr_t p = (uintptr_t)a.x | (uintptr_t)a.gain | (back ? (uintptr_t)a.dy | (uintptr_t)a.dx : (uintptr_t)a.y | (uintptr_t)a.bias);
  const i64 l = a.cols | a.ldx | (back ? a.lddy | a.lddx : a.ldy);
  return (p & 15) == 0 && (l & 7) == 0;
}
// waves per row and 8-column chunks per thread by the row's length
#define BY_COLS(call)                                   \
  do {                                                  \
    if (a.cols <= 512) call(1, 1);                      \
    else if (a.cols <= 1024) call(1, 2);                \
    else if (a.cols <= 2048) call(1, 4);                \
    else if (a.cols <= 4096) call(4, 2);                \
    else if (a.cols <= 8192) call(4, 4);                \
    else if (a.cols <= 32768) call(16, 4);              \
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
      if (grid > MAX_PARTS) grid = MAX_PARTS;
      hipLaunchKernelGGL((layernorm_bwd_k<T, AL, W, CH, true>), dim3(grid), block, W == 1 ? (size_t)3 * 2 * CH * 512 * 4 : 0, s, a);
      return grid;
    }
  }
  hipLaunchKernelGGL((layernorm_bwd_k<T, AL, W, CH, false>), dim3(grid), block, 0, s, a);
  if (!params) return 0;
  grid = a.rows < 4 * 32 ? cdiv(a.rows, 4) : 32;
  hipLaunchKernelGGL(layernorm_params_k<T>, dim3(cdiv(a.cols, 64), grid), dim3(256), 0, s, a);
  return grid;
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
  const dim3 grid(cdiv(a.cols, 16), 2);
  if (a.dt == 0 || a.grads_f32) hipLaunchKernelGGL(layernorm_reduce_k<float>, grid, dim3(256), 0, s, a.partial, n, a.cols, (float*)a.dgain, (float*)a.dbias);
  else hipLaunchKernelGGL(layernorm_reduce_k<bf16>, grid, dim3(256), 0, s, a.partial, n, a.cols, (bf16*)a.dgain, (bf16*)a.dbias);
}
