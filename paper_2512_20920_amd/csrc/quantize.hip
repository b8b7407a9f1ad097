// Rows to 8-bit integers with a scale each: scale = max |x| / 127, code = x / scale rounded to the nearest integer, ties to even.
// One pass over memory, which bounds it: a row's values wait in registers for its maximum (8192 x 4096 bfloat16: 23 us, 4.4 TB/s; 8 rows: a launch's 3).
//
// The quotient is rounded as if it were exact.  k = rint(x (1 / scale)) is right or next to it; x - k scale is a float (a multiple of half a
// step of scale, of at most 25 bits of which the last is zero where the first is not), so one comparison of twice that with scale tells which
// (scale / 2 itself need be no float: below 2^-125 scale may be an odd number of 2^-149).
#include "kernels.h"

// V codes in the low bytes of k.  x / scale + 1.5 2^23 has the nearest integer in its low bits; where no lane's remainder is half a step or more, as in
// nearly every wavefront, there is nothing to choose.
template <int V> __device__ __forceinline__ void codes_of(const float (&x)[V], float scale, float inv, unsigned (&k)[V]) {
  constexpr float BIG = 12582912.f;
  float worst = 0.f;
#pragma unroll
  for (int i = 0; i < V; i++) {
    const float z = fmaf(x[i], inv, BIG);
    k[i] = __builtin_bit_cast(unsigned, z);
    worst = fmaxf(worst, fabsf(fmaf(BIG - z, scale, x[i])));
  }
  if (__any(2.f * worst >= scale)) {
#pragma unroll
    for (int i = 0; i < V; i++) {
      const float r = 2.f * fmaf(BIG - __builtin_bit_cast(float, k[i]), scale, x[i]);
      if (fabsf(r) > scale || (fabsf(r) == scale && (k[i] & 1))) k[i] += r > 0.f ? 1 : -1;
    }
  }
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
  float v[N][V];
  unsigned most = 0;                                 // the largest |x|, as bits: what is not finite is above all that is
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
    for (int i = 0; i < V; i++) most = max(most, __builtin_bit_cast(unsigned, o[i]) & 0x7fffffffu);
  };
#pragma unroll
  for (int n = 0; n < N; n++) load(n * STEP + t * V, v[n]);
#pragma unroll
  for (int n = 0; n < N; n++) look(v[n]);
  for (int c = N * STEP + t * V; c < cols; c += STEP) { float o[V]; load(c, o); look(o); }
  float top = wave_max(most < 0x7f800000u ? __builtin_bit_cast(float, most) : INFINITY);
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
    unsigned k[V];
    codes_of<V>(o, scale, inv, k);
    if (!live)
#pragma unroll
      for (int i = 0; i < V; i++) k[i] = 0;
    if constexpr (V == 1) cr[c] = (signed char)k[0];
    else if (c + V <= cols) {
      unsigned w[V / 4];
#pragma unroll
      for (int i = 0; i < V / 4; i++)                // the four low bytes
        w[i] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(k[4 * i + 3], k[4 * i + 2], 0x0c0c0400), __builtin_amdgcn_perm(k[4 * i + 1], k[4 * i], 0x0c0c0400), 0x05040100);
      *(uint2*)(cr + c) = make_uint2(w[0], w[1]);
    } else {
#pragma unroll
      for (int i = 0; i < V; i++) if (c + i < cols) cr[c + i] = (signed char)k[i];
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
