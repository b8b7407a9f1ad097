// A cache of keys and values in pages of numbers of 8 bits: where a token lies, and which sequence an item of work belongs to.
//
// The numbers are e4m3 (4 bits of exponent, 3 of mantissa, largest 448, one NaN per sign), in units of a power of two per page and key
// head.  e4m3 rather than integers: a key's few large columns do not coarsen the others (half a step is 2^-4 of each value), a larger power of two
// changes only what falls below 2^-6 of the unit, so a page that is filled token by token is, but for that, the page filled at once, and the conversion to
// bfloat16 with its power of two is one instruction for two values, without a rounding.
// Keys lie as rows of a head.  Values lie in groups of 16 tokens, token fastest: the operand of the second product has tokens along its
// contraction, and is then 16 bytes in a row for one column.
#pragma once
#include "attn_range.h"

__device__ __forceinline__ int cache_len(const CacheView& c, int s) { return min(max(c.len[s], 0), 1 << 30); }
// rows of this call that belong to a sequence: the first, and how many
__device__ __forceinline__ int2 cache_rows(const CacheView& c, int s, int T) {
  if (!c.cu) return make_int2(s, s < T ? 1 : 0);
  const int a = min(max(c.cu[s], 0), T), b = min(max(c.cu[s + 1], 0), T);
  return make_int2(a, max(b - a, 0));
}
__device__ __forceinline__ int cache_room(const CacheView& c) { return c.max_pages << c.lg; }
// page of a sequence's token range; -1: there is none
__device__ __forceinline__ int cache_page(const CacheView& c, int s, int p) {
  const int n = c.table[(i64)s * c.max_pages + min(max(p, 0), c.max_pages - 1)];
  return p >= 0 && p < c.max_pages && n >= 0 && n < c.pages ? n : -1;
}
__device__ __forceinline__ i64 cache_block(const CacheView& c, int page, int head) { return (i64)page * c.Hkv + head; }      // of its scales; times page * dh: of its numbers

// inclusive sums over the lanes
__device__ __forceinline__ int wave_running(int v) {
  v += dpp_i<0x111, 0xf>(0, v);
  v += dpp_i<0x112, 0xf>(0, v);
  v += dpp_i<0x114, 0xf>(0, v);
  v += dpp_i<0x118, 0xf>(0, v);
  v += dpp_i<0x142, 0xa>(0, v);
  v += dpp_i<0x143, 0xc>(0, v);
  return v;
}
// Item `id` of a list in which sequence s has count(s) of them: the sequence, and which of its items.  One wave; false: the list is shorter.
template <class F> __device__ __forceinline__ bool find_item(int n_seqs, int id, F count, int* seq, int* at) {
  int before = 0;
  for (int s0 = 0; s0 < n_seqs; s0 += 64) {
    const int s = s0 + (int)(threadIdx.x & 63), mine = s < n_seqs ? count(s) : 0, running = wave_running(mine);
    const int all = __builtin_amdgcn_readlane(running, 63);
    if (id < before + all) {
      const int l = __builtin_ctzll(__ballot(before + running > id));
      *seq = s0 + l;
      *at = id - before - (__builtin_amdgcn_readlane(running, l) - __builtin_amdgcn_readlane(mine, l));
      return true;
    }
    before += all;
  }
  return false;
}
__device__ __forceinline__ float e4m3_value(unsigned byte) { return __builtin_amdgcn_cvt_f32_fp8((int)byte, 0); }
