// Rotary positions on rows of heads: y = m (u cos - w sin, u sin + w cos) for the pairs of the first `dims` columns of each
// head, the rest copied.  A workgroup takes a few rows: it works out the (cos, sin) of their pairs once, into LDS, and streams all
// heads of the rows past them, so that reading x and writing y is what bounds it and the angle may cost what it needs:
// position * frequency in float64, reduced to a fraction of a turn there, and a full-precision sine and cosine of that.
// bf16, 8192 rows of 40 heads of 128: 37 us (4.5 TB/s); float32, 4096 rows of 32 heads: 29 us (4.6).
#include "kernels.h"

template <class T, int V> struct Vec { typedef __attribute__((ext_vector_type(V))) T type; };
template <class T> struct Vec<T, 1> { typedef T type; };
template <class T, int V> __device__ __forceinline__ void load_vec(const T* p, float (&r)[V]) {
  const typename Vec<T, V>::type v = *(const typename Vec<T, V>::type*)p;
  if constexpr (V == 1) r[0] = to_f(v);
  else {
#pragma unroll
    for (int i = 0; i < V; i++) r[i] = to_f(v[i]);
  }
}
template <class T, int V> __device__ __forceinline__ void store_vec(T* p, const float (&r)[V]) {
  typename Vec<T, V>::type v;
  if constexpr (V == 1) v = from_f<T>(r[0]);
  else {
#pragma unroll
    for (int i = 0; i < V; i++) v[i] = from_f<T>(r[i]);
  }
  *(typename Vec<T, V>::type*)p = v;
}

// A head is cut into units of V columns: half layout: V pairs (two vectors) each, interleaved: V / 2 pairs (V = 1: one pair), then the
// columns that are only copied.  rows_wg rows per workgroup; units = units per head, magic = ceil(2^32 / units): the head of
// unit e < H units is the high half of e magic, exactly so while H units^2 <= 2^32 (a row has 2^22 columns at most, a head 2^10).
template <class T, int V, bool INTER>
__global__ void __launch_bounds__(256) rotary_k(RotaryArgs a, int rows_wg, int units, unsigned magic) {
  extern __shared__ float2 turn[];                   // [rows_wg][dims / 2]
  const T* x = (const T*)a.x;                        // (may be y: each thread reads what it writes before it writes it)
  T* y = (T*)a.y;
  const int half = a.dims / 2, t0 = (int)blockIdx.x * rows_wg, nt = min(rows_wg, a.T - t0);
  for (int e = threadIdx.x; e < nt * half; e += 256) {
    const int t = e / half, c = e - t * half, row = t0 + t;
    const double turns = (double)(a.pos ? a.pos[row] : row % a.S) * a.freq[c];
    float s, co;
    sincospif(2.f * (float)(turns - rint(turns)), &s, &co);
    turn[e] = make_float2(co * a.mag, s * a.mag * a.sign);
  }
  __syncthreads();
  constexpr int P = INTER ? (V == 1 ? 1 : V / 2) : V;                       // pairs per unit
  constexpr int W = INTER && V == 1 ? 2 : V;                                // columns per step of the copied part
  const int turned = half / P, per_row = a.H * units;
  for (int t = 0; t < nt; t++) {
    const T* xr = x + (i64)(t0 + t) * a.ldx;
    T* yr = y + (i64)(t0 + t) * a.ldy;
    const float2* cs = turn + t * half;
#pragma unroll 4
    for (int e = threadIdx.x; e < per_row; e += 256) {
      const int h = units == 1 ? e : (int)__umulhi((unsigned)e, magic), u = e - h * units;
      const T* xh = xr + (i64)h * a.dh;
      T* yh = yr + (i64)h * a.dh;
      if (u < turned) {
        if constexpr (INTER) {
          float v[W];
          if constexpr (V == 1) { v[0] = to_f(xh[2 * u]); v[1] = to_f(xh[2 * u + 1]); }
          else load_vec<T, V>(xh + u * V, v);
#pragma unroll
          for (int i = 0; i < P; i++) {
            const float2 r = cs[u * P + i];
            const float p = v[2 * i], q = v[2 * i + 1];
            v[2 * i] = p * r.x - q * r.y;
            v[2 * i + 1] = p * r.y + q * r.x;
          }
          if constexpr (V == 1) { yh[2 * u] = from_f<T>(v[0]); yh[2 * u + 1] = from_f<T>(v[1]); }
          else store_vec<T, V>(yh + u * V, v);
        } else {
          float p[V], q[V];
          load_vec<T, V>(xh + u * V, p);
          load_vec<T, V>(xh + half + u * V, q);
#pragma unroll
          for (int i = 0; i < V; i++) {
            const float2 r = cs[u * V + i];
            const float w = p[i];
            p[i] = w * r.x - q[i] * r.y;
            q[i] = w * r.y + q[i] * r.x;
          }
          store_vec<T, V>(yh + u * V, p);
          store_vec<T, V>(yh + half + u * V, q);
        }
      } else {
        const int c = a.dims + (u - turned) * W;
        if constexpr (W != V) {
#pragma unroll
          for (int i = 0; i < W; i++) if (c + i < a.dh) yh[c + i] = xh[c + i];
        } else {
          float v[V];
          load_vec<T, V>(xh + c, v);
          store_vec<T, V>(yh + c, v);
        }
      }
    }
  }
}

template <class T, int V, bool INTER> static void launch(const RotaryArgs& a, hipStream_t s) {
  constexpr int P = INTER ? (V == 1 ? 1 : V / 2) : V, W = INTER && V == 1 ? 2 : V;
  const bool in_place = a.x == a.y;
  const int half = a.dims / 2, units = half / P + (in_place ? 0 : cdiv(a.dh - a.dims, W));
  const unsigned magic = (unsigned)(((1ull << 32) + units - 1) / units);
  // enough rows for four units per thread where that leaves enough workgroups, and tables of 32 KiB at most
  int rows = cdiv(1024, (i64)a.H * units);
  if (rows > a.T / 1024) rows = a.T / 1024;
  if (rows > 4096 / half) rows = 4096 / half;
  if (rows < 1) rows = 1;
  hipLaunchKernelGGL((rotary_k<T, V, INTER>), dim3(cdiv(a.T, rows)), dim3(256), (size_t)rows * half * sizeof(float2), s, a, rows, units,
                     magic);
}
template <class T, int V> static void launch(const RotaryArgs& a, hipStream_t s) {
  if (a.interleaved) launch<T, V, true>(a, s); else launch<T, V, false>(a, s);
}
void launch_rotary(const RotaryArgs& a, hipStream_t s) {
  // widest vectors that every row, head and part of a head starts at a multiple of
  const int es = a.dt == 0 ? 4 : 2;
  const i64 all = a.ldx | a.ldy | a.dh | a.dims | (a.interleaved ? 0 : a.dims / 2);
  const uintptr_t at = (uintptr_t)a.x | (uintptr_t)a.y;
  auto fits = [&](int v) { return all % v == 0 && at % (uintptr_t)(v * es) == 0; };
  if (a.dt == 0) {
    if (fits(4)) launch<float, 4>(a, s);
    else if (fits(2)) launch<float, 2>(a, s);
    else launch<float, 1>(a, s);
  } else {
    if (fits(8)) launch<bf16, 8>(a, s);
    else if (fits(4)) launch<bf16, 4>(a, s);
    else if (fits(2)) launch<bf16, 2>(a, s);
    else launch<bf16, 1>(a, s);
  }
}
