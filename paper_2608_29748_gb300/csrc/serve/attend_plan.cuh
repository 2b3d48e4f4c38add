// How the work of an attention call is divided.
//
// A unit is the rows of `unit_tokens` consecutive tokens of a sequence under one
// key/value head (G query heads each), its cost the number of key tiles that any
// of its rows sees, at least one (an empty unit writes zeros).  The units follow
// one another by sequence, head, token; CTA i takes the costs [i share, (i+1) share) of
// that row, so the CTAs have the same number of key tiles whatever the lengths are, and
// a long context is split over as many CTAs as it fills.  The lengths are device data,
// so every CTA finds its own range: one scan over the sequences.  A unit that several
// CTAs share is joined by a second kernel.
#pragma once

#include "tokens.cuh"

namespace retrace {
namespace {

struct AttendShape {
  const int32_t* q_start;
  const int32_t* cache_len;
  int B, T, kv_heads;
  int uniform;  // tokens of every sequence where there is no list
  int causal, window, sinks;
  int places;       // positions a sequence has places for: max_pages * page_size
  int unit_tokens;  // tokens of a unit
};

// The tiles of kKeys keys of a unit: `sink_tiles` from 0, then those from `first` on.
struct UnitKeys {
  int lo, hi;  // any row sees at most [lo, hi] and the sinks
  int sink_tiles, first, count;
  __device__ __forceinline__ int tile(int k) const { return k < sink_tiles ? k : first + (k - sink_tiles); }
};

// Tokens [i0, i1) of a sequence of n tokens after c cached ones.
template <int kKeys>
__device__ __forceinline__ UnitKeys unit_keys(const AttendShape& s, int c, int n, int i0, int i1) {
  UnitKeys u;
  u.hi = min(c + (s.causal ? i1 : n) - 1, s.places - 1);
  u.lo = s.window > 0 ? max(0, c + i0 - s.window + 1) : 0;
  const int sinks = min(s.sinks, u.hi + 1);
  const int end = u.hi < u.lo ? 0 : u.hi / kKeys + 1;
  u.first = u.lo / kKeys;
  if (end == 0) u.first = 0x3FFFFFFF;  // only sinks, if any
  u.sink_tiles = sinks > 0 ? min((sinks + kKeys - 1) / kKeys, u.first) : 0;
  u.count = u.sink_tiles + max(0, end - u.first);
  return u;
}

__device__ __forceinline__ SeqTokens tokens_of(const AttendShape& s, int b) {
  return s.q_start ? seq_tokens(s.q_start, s.B, s.T, b) : SeqTokens{b * s.uniform, s.uniform};
}
__device__ __forceinline__ int units_of(const AttendShape& s, int n) {
  return n <= s.unit_tokens ? n > 0 : (n + s.unit_tokens - 1) / s.unit_tokens;
}
template <int kKeys>
__device__ __forceinline__ int unit_cost(const AttendShape& s, int c, int n, int u) {
  return max(1, unit_keys<kKeys>(s, c, n, u * s.unit_tokens, min(n, (u + 1) * s.unit_tokens)).count);
}

// Cost of one head of sequence b.  Called by whole warps: the sequences with many
// units (prompts) are summed by all lanes, one after another.
template <int kKeys>
__device__ __forceinline__ long long head_cost(const AttendShape& s, int b, bool valid) {
  constexpr int kAlone = 4;
  SeqTokens q{0, 0};
  int c = 0, units = 0;
  long long cost = 0;
  if (valid) {
    q = tokens_of(s, b);
    c = cached_tokens(s.cache_len, b);
    units = units_of(s, q.n);
    if (units <= kAlone)
      for (int u = 0; u < units; ++u) cost += unit_cost<kKeys>(s, c, q.n, u);
  }
  unsigned many = __ballot_sync(0xFFFFFFFFu, units > kAlone);
  while (many) {
    const int l = __ffs(many) - 1;
    many &= many - 1;
    const int cl = __shfl_sync(0xFFFFFFFFu, c, l), nl = __shfl_sync(0xFFFFFFFFu, q.n, l);
    const int ul = __shfl_sync(0xFFFFFFFFu, units, l);
    long long part = 0;
    for (int u = threadIdx.x & 31; u < ul; u += 32) part += unit_cost<kKeys>(s, cl, nl, u);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) part += __shfl_xor_sync(0xFFFFFFFFu, part, o);
    if ((int)(threadIdx.x & 31) == l) cost = part;
  }
  return cost;
}

// A CTA's share, and its first piece.
struct PlanStart {
  long long total;       // cost of the call
  long long begin, end;  // this CTA's range of it
  long long unit_begin;  // where the first unit begins
  long long share;       // cost of a CTA's range (the last may be shorter)
  int b, head, unit;     // the first unit
};

// One piece: key tiles [k0, k1) of a unit.
struct Piece {
  int b, head;
  int row0, n, c;  // first packed row of the sequence, its tokens, its cached tokens
  int i0, i1;      // tokens of the unit
  UnitKeys keys;
  int k0, k1;             // of keys.count (an empty unit: 0, 0)
  int first_cta, pieces;  // the CTAs that share the unit
};

// x / y; a division of 64 bits takes many instructions, and costs rarely need them.
__device__ __forceinline__ long long quotient(long long x, long long y) {
  return ((x | y) >> 32) == 0 ? (long long)((uint32_t)x / (uint32_t)y) : x / y;
}

// Walks a CTA's pieces; every role of the CTA walks them for itself.
struct PieceWalk {
  long long at, unit_begin;
  int b, head, unit;

  __device__ __forceinline__ void start(const PlanStart& p) {
    at = p.begin;
    unit_begin = p.unit_begin;
    b = p.b;
    head = p.head;
    unit = p.unit;
  }
  // The piece at `at`, and on to the next one.  False at the end of the range.  `pieces` is
  // worked out only where it is asked for.
  template <int kKeys, bool kPieces = false>
  __device__ __forceinline__ bool next(const AttendShape& s, const PlanStart& p, Piece* out) {
    if (at >= p.end) return false;
    for (;;) {
      const SeqTokens q = tokens_of(s, b);
      if (unit * (long long)s.unit_tokens < q.n) {
        out->b = b;
        out->head = head;
        out->row0 = q.first;
        out->n = q.n;
        out->c = cached_tokens(s.cache_len, b);
        out->i0 = unit * s.unit_tokens;
        out->i1 = min(q.n, out->i0 + s.unit_tokens);
        out->keys = unit_keys<kKeys>(s, out->c, q.n, out->i0, out->i1);
        break;
      }
      // past the sequence's last unit: the next head, or the next sequence
      unit = 0;
      if (q.n > 0 && head + 1 < s.kv_heads) {
        ++head;
      } else {
        head = 0;
        if (++b >= s.B) return false;
      }
    }
    const int cost = max(1, out->keys.count);
    const long long k0 = at - unit_begin, left = p.end - unit_begin;
    const int k1 = left < cost ? (int)left : cost;
    if (kPieces) {
      const long long first = quotient(unit_begin, p.share);
      out->first_cta = (int)first;
      out->pieces = (int)(quotient(unit_begin + cost - 1, p.share) - first) + 1;
    }
    out->k0 = out->keys.count ? (int)k0 : 0;
    out->k1 = out->keys.count ? k1 : 0;
    at = unit_begin + k1;
    if (k1 == cost) {
      unit_begin += cost;
      ++unit;
    }
    return true;
  }
};

// Finds this CTA's share; all kThreads threads of the CTA call it.  `s_sum` has
// one entry per warp.  At least `least` key tiles to a CTA.
template <int kThreads, int kKeys>
__device__ __forceinline__ void plan_start(const AttendShape& s, int grid, int least, PlanStart* s_plan, long long* s_sum) {
  static_assert(kThreads % 32 == 0, "whole warps");
  const int tid = threadIdx.x;
  // Thread t sums the sequences [t per, (t+1) per).
  const int per = (s.B + kThreads - 1) / kThreads;
  long long mine = 0;
  for (int i = 0; i < per; ++i) {
    const int b = tid * per + i;
    mine += head_cost<kKeys>(s, b, b < s.B) * s.kv_heads;
  }
  // Inclusive scan over the threads: warps, then their sums.
  long long x = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(0xFFFFFFFFu, x, o);
    if ((tid & 31) >= o) x += y;
  }
  if ((tid & 31) == 31) s_sum[tid / 32] = x;
  __syncthreads();
  long long before = 0, total = 0;
  for (int w = 0; w < kThreads / 32; ++w) {
    if (w < tid / 32) before += s_sum[w];
    total += s_sum[w];
  }
  const long long upto = before + x, from = upto - mine;
  if (total == 0) {
    if (tid == 0) *s_plan = PlanStart{0, 0, 0, 0, 0, 0, 0, 0};
    __syncthreads();
    return;
  }
  const long long even = quotient(total + grid - 1, grid), share = even > least ? even : least;
  const long long begin = share * blockIdx.x, end = begin + share < total ? begin + share : total;
  if (begin >= total) {
    if (tid == 0) *s_plan = PlanStart{total, 0, 0, 0, share, 0, 0, 0};
  } else if (from <= begin && begin < upto) {  // one thread: its sequences hold the start
    long long at = from;
    for (int i = 0; i < per; ++i) {
      const int b = tid * per + i;
      if (b >= s.B) break;
      const SeqTokens q = tokens_of(s, b);
      const int c = cached_tokens(s.cache_len, b), units = units_of(s, q.n);
      long long one = 0;
      for (int u = 0; u < units; ++u) one += unit_cost<kKeys>(s, c, q.n, u);
      if (begin < at + one * s.kv_heads) {
        const int head = (int)quotient(begin - at, one);
        at += head * one;
        int u = 0;
        for (;; ++u) {
          const int cost = unit_cost<kKeys>(s, c, q.n, u);
          if (begin < at + cost) break;
          at += cost;
        }
        *s_plan = PlanStart{total, begin, end, at, share, b, head, u};
        break;
      }
      at += one * s.kv_heads;
    }
  }
  __syncthreads();
}

}  // namespace
}  // namespace retrace
