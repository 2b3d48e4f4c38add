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

// The sequence of token t and its first token; -1: of none.  Called by a whole warp: without a list
// (`uniform` tokens each) by division, else by a search of 32 starts at a time.
__device__ __forceinline__ int sequence_of(const int32_t* q_start, int B, int uniform, int t, int lane, int* first) {
  if (!q_start) {
    const int b = t / uniform;
    *first = b * uniform;
    return b;
  }
  *first = 0;
  int lo = 0, n = B;  // the last start <= t lies in [lo, lo + n), if any
  while (n > 32) {
    const int step = (n + 31) / 32;
    const int pos = lo + lane * step;
    const bool below = pos < lo + n && q_start[pos] <= t;
    const int c = __popc(__ballot_sync(0xFFFFFFFFu, below));
    if (c == 0) break;
    const int end = lo + n;
    lo += (c - 1) * step;
    n = min(step, end - lo);
  }
  const bool below = lane < n && lane < 32 && q_start[lo + lane] <= t;
  const int c = __popc(__ballot_sync(0xFFFFFFFFu, below));
  if (c == 0) return -1;
  const int b = lo + c - 1;
  *first = q_start[b];
  return t >= q_start[b + 1] || *first < 0 ? -1 : b;  // a token of no sequence
}

// The sequence of token t, before q_start[B], that lies in b or behind it: among the next ones, or by halving
// (a batch may have any number of sequences without tokens).
__device__ __forceinline__ int sequence_from(const int32_t* q_start, int B, int b, int t) {
  for (int i = 0; i < 4; ++i, ++b)
    if (t < q_start[b + 1]) return b;
  for (int hi = B; hi - b > 1;) {  // t is before the start of hi
    const int mid = b + (hi - b) / 2;
    if (t < q_start[mid])
      hi = mid;
    else
      b = mid;
  }
  return b;
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
