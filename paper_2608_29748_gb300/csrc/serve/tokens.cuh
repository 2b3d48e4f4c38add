// What the cache operators share on the device: where a sequence's tokens lie in
// a packed batch, and where a position lies in the paged cache.
#pragma once

#include "../../../include/retrace.h"
#include "../common.cuh"

namespace retrace {
namespace {

// x / d for 0 <= x < 2^31 by a multiplication: q = (x + hi(x mul)) >> shift.
struct FastDivide {
  uint32_t mul;
  int shift, by;
  __host__ static FastDivide of(int d) {
    int s = 0;
    while ((1ll << s) < d) ++s;
    return {(uint32_t)(((1ull << 32) * ((1ull << s) - (unsigned long long)d)) / (unsigned long long)d + 1), s, d};
  }
  __device__ __forceinline__ int operator()(int x) const { return (int)((__umulhi((uint32_t)x, mul) + (uint32_t)x) >> shift); }
};

// The tokens of sequence b: rows [first, first + n) of the packed tensors.  The
// list is the caller's device data: whatever it holds, the rows stay in [0, T).
struct SeqTokens {
  int first, n;
};
__device__ __forceinline__ SeqTokens seq_tokens(const int32_t* q_start, int B, int T, int b) {
  if (!q_start) {
    const int n = T / B;
    return {b * n, n};
  }
  const int lo = min(max(q_start[b], 0), T), hi = min(max(q_start[b + 1], 0), T);
  return {lo, max(hi - lo, 0)};
}

// Lengths outside (-2^30, 2^30) are taken as the nearest end, so that positions
// stay in 32 bits (a sequence has at most 2^30 places).
__device__ __forceinline__ int cached_tokens(const int32_t* cache_len, int b) {
  return min(max(cache_len[b], -(1 << 30)), (1 << 30) - 1);
}

// The page of a position, or -1 where it has no place in the cache.
__device__ __forceinline__ int page_of(const retrace_kv_cache& c, int b, int page_index) {
  if (page_index < 0 || page_index >= c.max_pages) return -1;
  const int page = c.page_table[b * c.table_stride + page_index];
  return page >= 0 && page < c.num_pages ? page : -1;
}

}  // namespace
}  // namespace retrace
