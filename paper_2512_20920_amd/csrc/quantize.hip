// Rows to 8-bit integers with a scale each: scale = max |x| / 127, code = x / scale rounded to the nearest integer, ties to even.
// One pass over memory: a row's values wait in registers for its maximum.
//
// The quotient is rounded as if it were exact.  k = rint(x (1 / scale)) is right or next to it; x - k scale is a float (a multiple of half a
// step of scale, of at most 25 bits of which the last is zero where the first is not), so one comparison with scale / 2 tells which.
#include "kernels.h"

__device__ __forceinline__ int code_of(float x, float scale, float inv) {
  float k = rintf(x * inv);
  const float r = fmaf(-k, scale, x), half = 0.5f * scale;
  if (fabsf(r) > half || (fabsf(r) == half && ((int)k & 1))) k += r > 0.f ? 1.f : -1.f;
  return (int)k;
}
template <class T, int V> struct Vec { typedef __attribute__((ext_vector_type(V))) T type; };

// V: values per load (8: 16 bytes of bfloat16, 32 of float32; 1: any alignment), N: loads per thread that stay in registers; longer rows are read
// a second time.  W: waves per row (4: a workgroup, 1: four rows per workgroup).
template <class T, int V, int N, int W>
__global__ void __launch_bounds__(256) quantize_rows_k(const T* __restrict__ x, signed char* __restrict__ codes, float* __restrict__ scales, int rows, int cols, i64 ldx, i64 ldc) {
  __shared__ float red[4];
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, row = W == 4 ? (int)blockIdx.x : (int)blockIdx.x * 4 + wv;
  const int t = W == 4 ? (int)threadIdx.x : lane;
  constexpr int STEP = W * 64 * V;
  if (row >= rows) return;                           // (W = 1: no barrier below)
  const T* xr = x + (i64)row * ldx;
  signed char* cr = codes + (i64)row * ldc;
  float v[N][V], top = 0.f;
  bool fine = true;
  auto load = [&](int c, float (&o)[V]) {
    if constexpr (V == 1) o[0] = c < cols ? to_f(xr[c]) : 0.f;
    else {
#pragma unroll
      for (int i = 0; i < V; i++) o[i] = 0.f;
      if (c + V <= cols) {
        const typename Vec<T, V>::type w = *(const typename Vec<T, V>::type*)(xr + c);
#pragma unroll
        for (int i = 0; i < V; i++) o[i] = to_f(w[i]);
      } else {
#pragma unroll
        for (int i = 0; i < V; i++) if (c + i < cols) o[i] = to_f(xr[c + i]);
      }
    }
  };
  auto look = [&](const float (&o)[V]) {
#pragma unroll
    for (int i = 0; i < V; i++) { const float a = fabsf(o[i]); fine = fine && a < INFINITY; top = fmaxf(top, a); }
  };
#pragma unroll
  for (int n = 0; n < N; n++) load(n * STEP + t * V, v[n]);
#pragma unroll
  for (int n = 0; n < N; n++) look(v[n]);
  for (int c = N * STEP + t * V; c < cols; c += STEP) { float o[V]; load(c, o); look(o); }
  if (!fine) top = INFINITY;
  top = wave_max(top);
  if constexpr (W == 4) {
    if (lane == 0) red[wv] = top;
    __syncthreads();
    top = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  }
  float scale = top / 127.f;
  if (scale < 1.17549435e-38f) scale = 0.f;          // (of no normal number: the row counts as zeros)
  const bool live = scale > 0.f && scale < INFINITY;
  const float inv = live ? 1.f / scale : 0.f;
  if (t == 0) scales[row] = scale < INFINITY ? scale : __builtin_nanf("");
  auto put = [&](int c, const float (&o)[V]) {
    if (c >= cols) return;
    signed char k[V];
#pragma unroll
    for (int i = 0; i < V; i++) k[i] = live ? (signed char)code_of(o[i], scale, inv) : 0;
    if constexpr (V == 1) cr[c] = k[0];
    else if (c + V <= cols) {
      typename Vec<signed char, V>::type w;
#pragma unroll
      for (int i = 0; i < V; i++) w[i] = k[i];
      *(typename Vec<signed char, V>::type*)(cr + c) = w;
    } else {
#pragma unroll
      for (int i = 0; i < V; i++) if (c + i < cols) cr[c + i] = k[i];
    }
  };
#pragma unroll
  for (int n = 0; n < N; n++) put(n * STEP + t * V, v[n]);
  for (int c = N * STEP + t * V; c < cols; c += STEP) { float o[V]; load(c, o); put(c, o); }
}

template <class T, int V> static void launch(const void* x, signed char* codes, float* scale, int rows, int cols, i64 ldx, i64 ldc, hipStream_t s) {
  const T* p = (const T*)x;
  if (cols <= 64 * V * 2) hipLaunchKernelGGL((quantize_rows_k<T, V, 2, 1>), dim3(cdiv(rows, 4)), dim3(256), 0, s, p, codes, scale, rows, cols, ldx, ldc);
  else if (cols <= 256 * V * 2) hipLaunchKernelGGL((quantize_rows_k<T, V, 2, 4>), dim3(rows), dim3(256), 0, s, p, codes, scale, rows, cols, ldx, ldc);
  else hipLaunchKernelGGL((quantize_rows_k<T, V, 8, 4>), dim3(rows), dim3(256), 0, s, p, codes, scale, rows, cols, ldx, ldc);
}
void launch_quantize_rows(int dt, const void* x, signed char* codes, float* scale, int rows, int cols, i64 ldx, i64 ldc, hipStream_t s) {
  if (rows < 1) return;
  const bool wide = ldx % 8 == 0 && ldc % 8 == 0 && (uintptr_t)x % 16 == 0 && (uintptr_t)codes % 8 == 0;
  if (dt == 0) { if (wide) launch<float, 8>(x, codes, scale, rows, cols, ldx, ldc, s); else launch<float, 1>(x, codes, scale, rows, cols, ldx, ldc, s); }
  else { if (wide) launch<bf16, 8>(x, codes, scale, rows, cols, ldx, ldc, s); else launch<bf16, 1>(x, codes, scale, rows, cols, ldx, ldc, s); }
}
