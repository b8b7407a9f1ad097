// The turn of a pair of columns at a position, shared by the rotation and by the cache's append: the same bits in both.
#pragma once
#include "kernels.h"

// (cos, sin) of position * frequency (in turns), worked out in float64 and reduced to a fraction of a turn there
__device__ __forceinline__ float2 rotary_turn(double freq, int pos, float mag, float sign) {
  const double turns = (double)pos * freq;
  float s, co;
  sincospif(2.f * (float)(turns - rint(turns)), &s, &co);
  return make_float2(co * mag, s * mag * sign);
}
__device__ __forceinline__ void rotary_pair(float& p, float& q, float2 r) {
  const float w = p;                                 // (which of the products is rounded is said here, not left to the compiler)
  p = fmaf(w, r.x, -(q * r.y));
  q = fmaf(q, r.x, w * r.y);
}
