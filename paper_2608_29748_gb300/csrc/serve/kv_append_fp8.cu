// Appending keys and values to a paged cache in 8 bits, rotating keys and queries on the way.
//
// With x' the rotated elements, a page's new tokens and a head: a = max |x'|, e the least
// exponent with a <= 448 2^e, e = max(e, the page's) where the page holds earlier tokens, codes
// round(x' 2^-e).  The maximum comes before the first code, so a team of warps takes a page's new tokens
// of one head (k or v) as a whole and keeps the rotated numbers, 16 to a thread, in between: four warps
// for 16 tokens of 128 in bf16, at most eight; what is beyond that is read twice.  Some CTAs have the
// pages, a share of the heads of 32 tokens each, the others the queries.
// Each element is read once from HBM and written once, 100 MB for 256 blocks of 17 tokens, 32 + 2 x 8 heads of 128
// in bf16: 15 us of HBM.  It takes 35: a CTA is a chain of waits (its tokens' places 2 us, then 2 us for each
// team's next page and head), and the registers allow three CTAs.
#include "fp8.cuh"
#include "tokens.cuh"

namespace retrace {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kCtasPerSm = 3;
constexpr int kMostTokens = 32;  // of a CTA at a time
constexpr int kHeadsEach = 3;    // query heads whose loads a thread has in flight

// Items of a thread that it keeps.
template <int N>
constexpr int kItems = N == 1 ? 1 : 8 / N;
constexpr int kAhead = 2;  // of what is read twice: items (a chunk and its partner, or two chunks of v) whose loads a thread has in flight

// N elements, loaded and stored as one access.  (As words: arrays of elements that are loaded as vectors
// land in local memory.)
template <typename T, int N>
struct Chunk;
template <typename T>
struct Chunk<T, 1> {
  T e;
  __device__ __forceinline__ void load(const T* p) { e = *p; }
  __device__ __forceinline__ void store(T* p) const { *p = e; }
  __device__ __forceinline__ void to(float (&f)[1]) const { f[0] = to_f32(e); }
  __device__ __forceinline__ void from(const float (&f)[1]) { e = from_f32<T>(f[0]); }
};
template <>
struct Chunk<float, 4> {
  float4 v;
  __device__ __forceinline__ void load(const float* p) { v = *reinterpret_cast<const float4*>(p); }
  __device__ __forceinline__ void store(float* p) const { *reinterpret_cast<float4*>(p) = v; }
  __device__ __forceinline__ void to(float (&f)[4]) const {
    f[0] = v.x;
    f[1] = v.y;
    f[2] = v.z;
    f[3] = v.w;
  }
  __device__ __forceinline__ void from(const float (&f)[4]) { v = make_float4(f[0], f[1], f[2], f[3]); }
};
template <>
struct Chunk<__nv_bfloat16, 8> {
  uint4 v;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { v = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void store(__nv_bfloat16* p) const { *reinterpret_cast<uint4*>(p) = v; }
  __device__ __forceinline__ void to(float (&f)[8]) const {
    f[0] = bf16_lo(v.x);
    f[1] = bf16_hi(v.x);
    f[2] = bf16_lo(v.y);
    f[3] = bf16_hi(v.y);
    f[4] = bf16_lo(v.z);
    f[5] = bf16_hi(v.z);
    f[6] = bf16_lo(v.w);
    f[7] = bf16_hi(v.w);
  }
  __device__ __forceinline__ void from(const float (&f)[8]) {
    v = make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
  }
};

// Lanes of a rotated head: first the chunks that rotate with a partner chunk (halves; single
// elements also when interleaved), then those whose pairs lie inside (interleaved), then
// those that are copied.  Without a rotation a head's halves are chunks and their partners, and nothing is
// turned.  Lane i of a head of v has the chunks i and i + lanes.
struct HeadShape {
  int pairs, inside, copies, lanes;  // lanes: their sum
  int step;                          // from a chunk to its partner, elements
  int page_ctas;             // the others have the queries
  int shares, share_tasks;   // of a chunk's heads (k and v apart)
  int tokens, query_tokens;  // of a CTA at a time
  int per_token;  // groups of lanes that share a token's query heads
  int team;       // warps that share a page's tokens of a head
};

// A lane's chunk of a rotated head.
struct Place {
  bool pair, inside;
  int at;
};
template <int N>
__device__ __forceinline__ Place place_of(const HeadShape& s, int rot, int i) {
  Place p;
  p.pair = i < s.pairs;
  p.inside = !p.pair && i < s.pairs + s.inside;
  p.at = p.pair ? (s.step == 1 ? 2 * i : i * N) : p.inside ? (i - s.pairs) * N : rot + (i - s.pairs - s.inside) * N;
  return p;
}

// Cosines and sines of a lane's pairs (of pairs inside a chunk: half as many).
template <int N>
__device__ __forceinline__ void load_angles(float (&cs)[2 * N], const float* rope, int pos, int rot, const Place& p, int i) {
  if (!p.pair && !p.inside) return;
  const float* r = rope + (long long)pos * rot + (p.inside ? p.at : i * 2 * N);
  if constexpr (N == 1) {
    cs[0] = r[0];
    cs[1] = r[1];
  } else {
#pragma unroll
    for (int k = 0; k < 2 * N; k += 4) {
      if (k < N || p.pair) {
        const float4 x = *reinterpret_cast<const float4*>(r + k);
        cs[k] = x.x;
        cs[k + 1] = x.y;
        cs[k + 2] = x.z;
        cs[k + 3] = x.w;
      }
    }
  }
}

// (v, w) turned by (c, s); the products are rounded before they are added.  (As operations on two numbers at once the
// assembler joins a product and a sum into one rounding, although both ask for their own.)
__device__ __forceinline__ void turn(float& v, float& w, float c, float s) {
  const float a = __fsub_rn(__fmul_rn(v, c), __fmul_rn(w, s));
  w = __fadd_rn(__fmul_rn(w, c), __fmul_rn(v, s));
  v = a;
}
template <int N>
__device__ __forceinline__ void turn_chunks(float (&fx)[N], float (&fy)[N], const float (&cs)[2 * N], const Place& p) {
  if (p.pair) {
#pragma unroll
    for (int k = 0; k < N; ++k) turn(fx[k], fy[k], cs[2 * k], cs[2 * k + 1]);
  } else if (N > 1 && p.inside) {
#pragma unroll
    for (int k = 0; k + 1 < N; k += 2) turn(fx[k], fx[k + 1], cs[k], cs[k + 1]);
  }
}
template <typename T, int N>
__device__ __forceinline__ void turned(const Chunk<T, N>& x, const Chunk<T, N>& y, const float (&cs)[2 * N], const Place& p,
                                       float (&fx)[N], float (&fy)[N]) {
  x.to(fx);
  y.to(fy);
  turn_chunks(fx, fy, cs, p);
}

template <int N>
__device__ __forceinline__ void store_codes(uint8_t* to, const float (&f)[N], float unit) {
  if constexpr (N == 1) {
    *to = (uint8_t)to_e4m3x2(f[0] * unit, 0.f);
  } else {
    uint32_t w[N / 4];
#pragma unroll
    for (int k = 0; k < N; k += 4)
      w[k / 4] = to_e4m3x2(f[k] * unit, f[k + 1] * unit) | to_e4m3x2(f[k + 2] * unit, f[k + 3] * unit) << 16;
    if constexpr (N == 8)
      *reinterpret_cast<uint2*>(to) = make_uint2(w[0], w[1]);
    else
      *reinterpret_cast<uint32_t*>(to) = w[0];
  }
}

// The threads of a team of warps.
__device__ __forceinline__ void team_barrier(int team, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "r"(threads) : "memory"); }

// The new tokens of a sequence in one page.
struct PagePiece {
  int t, count;  // first token, and how many
  int pos;       // of the first
  int page, slot;
};

// Where the token of a lane, t0 + lane, lies: its sequence (-1: of none), the sequence's first token and end,
// its position (-1: caches nothing, its query is zero; -2: of no sequence).  The warp finds the first token's
// sequence, the other lanes go on from there: a chain of reads for all tokens and not one for each.
struct TokenPlace {
  int b, first, end, pos;
};
__device__ __forceinline__ TokenPlace place_token(const AppendArgs& a, int uniform, int t0, int lane) {
  TokenPlace x;
  const int t = t0 + lane;
  if (!a.q_start) {
    x.b = t < a.T ? t / uniform : -1;
    x.first = x.b * uniform;
    x.end = x.first + uniform;
  } else {
    x.b = sequence_of(a.q_start, a.B, uniform, t0, lane, &x.first);
    if (x.b < 0) {  // behind the last sequence, or before the first
      const int from = max(min(a.q_start[0], a.T), 0);
      x.b = t0 < from ? 0 : a.B;
      x.first = from;
    }
    const bool inside = x.b < a.B && t >= x.first && t < min(a.q_start[a.B], a.T);
    if (inside && t >= a.q_start[x.b + 1]) {
      x.b = sequence_from(a.q_start, a.B, x.b, t);
      x.first = a.q_start[x.b];
    }
    if (!inside || x.first < 0 || t < x.first) x.b = -1;
    x.end = x.b >= 0 ? min(a.q_start[x.b + 1], a.T) : 0;
  }
  x.pos = x.b < 0 ? -2 : cached_tokens(a.cache_len, x.b) + (t - x.first);
  if (x.b >= 0 && (x.pos < 0 || (a.rope && x.pos >= a.rope_positions))) x.pos = -1;
  return x;
}

struct Shared {
  int pos[kMostTokens];
  PagePiece piece[kMostTokens];
  int pieces;
  uint32_t top[kWarps];
};

// Asks L2 for the rows of the tokens [t0, t0 + tokens) that are on their way into registers soon: a CTA has
// registers for few loads at a time.
template <typename T>
__device__ __forceinline__ void ask_for(const T* base, long long token, long long head, int heads, int D, int t0, int tokens) {
  const int lines = (D * (int)sizeof(T) + 127) / 128, per_token = heads * lines;
  for (int i = threadIdx.x; i < tokens * per_token; i += kThreads) {
    const int k = i / per_token, j = i - k * per_token, h = j / lines;
    const char* at = reinterpret_cast<const char*>(base + (t0 + k) * token + h * head) + (j - h * lines) * 128;
    asm volatile("prefetch.global.L2 [%0];" ::"l"(at));
  }
}

// The queries of the tokens [t0, t0 + tokens).  Lane i of a group owns the same pairs in every head of its token.
template <typename T, int N>
__device__ __forceinline__ void rotate_queries(const AppendArgs& a, const HeadShape& s, Shared& sm, int t0, int tokens) {
  const int tid = threadIdx.x, L = s.lanes, group = tid / L, i = tid % L, each = kThreads / L / s.per_token;
  if (group >= each * s.per_token) return;
  const Place at = place_of<N>(s, a.rot, i), turns{at.pair && a.rot > 0, at.inside, at.at};
  for (int k = group / s.per_token; k < tokens; k += each) {
    const int pos = sm.pos[k], t = t0 + k;
    if (pos == -2) continue;
    float cs[2 * N];
    if (pos >= 0) load_angles<N>(cs, a.rope, pos, a.rot, turns, i);
    for (int h0 = group % s.per_token; h0 < a.q_heads; h0 += kHeadsEach * s.per_token) {
      Chunk<T, N> x[kHeadsEach], y[kHeadsEach];
#pragma unroll
      for (int u = 0; u < kHeadsEach; ++u) {
        const int h = h0 + u * s.per_token;
        if (h >= a.q_heads) break;
        const T* from = static_cast<const T*>(a.q) + (long long)t * a.q_token + h * a.q_head + at.at;
        x[u].load(from);
        if (at.pair) y[u].load(from + s.step);
      }
#pragma unroll
      for (int u = 0; u < kHeadsEach; ++u) {
        const int h = h0 + u * s.per_token;
        if (h >= a.q_heads) break;
        T* to = static_cast<T*>(a.q_out) + (long long)t * a.qo_token + h * a.qo_head + at.at;
        float fx[N], fy[N];
        turned(x[u], y[u], cs, turns, fx, fy);
        if (pos < 0) {
#pragma unroll
          for (int j = 0; j < N; ++j) fx[j] = fy[j] = 0.f;
        }
        if (turns.pair || (N > 1 && at.inside) || pos < 0) {  // else copied as it is
          x[u].from(fx);
          y[u].from(fy);
        }
        x[u].store(to);
        if (at.pair) y[u].store(to + s.step);
      }
    }
  }
}

// The exponent of a page of which a team has new tokens with the maximum `most` (a thread's own) before
// slot `slot`, where `codes` points; what the page holds before that, in units of 2^old, is rounded to the
// new unit.
template <int N>
__device__ __forceinline__ int page_unit(const retrace_kv_cache& c, const HeadShape& s, Shared& sm, float most, int old, uint8_t* codes, int slot) {
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, team = warp / s.team, in_team = warp % s.team;
  // not negative: the order of the bits is that of the numbers
  uint32_t top = __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(most));
  if (s.team > 1) {
    if (lane == 0) sm.top[warp] = top;
    team_barrier(team, s.team * 32);
    for (int w = 0; w < s.team; ++w) top = max(top, sm.top[warp - in_team + w]);
    team_barrier(team, s.team * 32);  // all have read the maxima, and the exponent before
  }
  const int e = max(top > 0u ? exponent_for(__uint_as_float(top)) : -kMostExponent, old);
  if (slot > 0 && e > old) {
    uint8_t* page = codes - (long long)slot * c.slot_stride;
    const float down = power_of_two(old - e);
    const int words = N >= 4 ? c.head_dim / 4 : c.head_dim;
    for (int idx = in_team * 32 + lane; idx < slot * words; idx += s.team * 32) {
      uint8_t* at = page + (long long)(idx / words) * c.slot_stride + idx % words * (N >= 4 ? 4 : 1);
      if constexpr (N >= 4) {
        uint32_t& w = *reinterpret_cast<uint32_t*>(at);
        const float2 lo = e4m3_floats(w & 0xFFFFu), hi = e4m3_floats(w >> 16);
        w = to_e4m3x2(lo.x * down, lo.y * down) | to_e4m3x2(hi.x * down, hi.y * down) << 16;
      } else {
        *at = (uint8_t)to_e4m3x2(e4m3_floats(*at).x * down, 0.f);
      }
    }
  }
  return e;
}

// The pieces among the tokens [t0, t0 + tokens), for one warp.
__device__ __forceinline__ void find_pieces(const AppendArgs& a, Shared& sm, int t0, int tokens, int lane) {
  const retrace_kv_cache& c = a.cache;
  // A token that begins its sequence's part of the call, or a page, begins a piece.
  const TokenPlace x = place_token(a, a.q_start ? 0 : a.T / a.B, t0, lane);
  const int t = t0 + lane, slot = x.pos < 0 ? 0 : x.pos % c.page_size;
  PagePiece piece{t, 0, x.pos, -1, slot};
  if (lane < tokens && x.pos >= 0 && (t == x.first || slot == 0)) {
    piece.count = min(x.end - t, c.page_size - slot);
    if (a.rope) piece.count = min(piece.count, a.rope_positions - x.pos);
    piece.page = page_of(c, x.b, x.pos / c.page_size);
  }
  const unsigned there = __ballot_sync(0xFFFFFFFFu, piece.page >= 0);  // those that have a page, one after another
  if (piece.page >= 0) sm.piece[__popc(there & ((1u << lane) - 1u))] = piece;
  if (lane == 0) sm.pieces = __popc(there);
}

// Keys and values whose rotated numbers a team of warps keeps (N > 1): a lane has the same chunks of tokens
// `apart` from one another.
template <typename T, int N>
__device__ __forceinline__ void fill_pages(const AppendArgs& a, const HeadShape& s, Shared& sm, int first_task, int tasks) {
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const retrace_kv_cache& c = a.cache;
  const int D = c.head_dim, L = s.lanes;
  const int team = warp / s.team, in_team = warp % s.team, teams = kWarps / s.team;
  const int abreast = 32 / L, apart = s.team * abreast, lane_token = in_team * abreast + lane / L, i = lane % L;
  const bool working = lane / L < abreast;
  for (int task = team; task < sm.pieces * tasks; task += teams) {
    const PagePiece p = sm.piece[task / tasks];
    const int head = first_task + task % tasks, h = head >> 1;
    const bool value = head & 1;
    Place at{false, false, i * N < D ? i * N : -1};
    int second = (i + L) * N < D ? (i + L) * N : -1;
    if (!value) {
      at = place_of<N>(s, a.rot, i);
      second = at.pair ? at.at + s.step : -1;
    }
    if (!working) {
      at = Place{false, false, -1};
      second = -1;
    }
    const long long step = value ? a.v_token : a.k_token;
    const T* src = static_cast<const T*>(value ? a.v : a.k) + (p.t + lane_token) * step + h * (value ? a.v_head : a.k_head);
    uint8_t* codes = static_cast<uint8_t*>(value ? c.v : c.k) + p.page * c.page_stride + h * c.head_stride + (long long)p.slot * c.slot_stride;
    int8_t* exp = (value ? a.v_exp : a.k_exp) + p.page * a.exp_page + h * a.exp_head;
    const int old = p.slot > 0 ? *exp : -kMostExponent;
    const int left = p.count - in_team * abreast, mine = p.count - lane_token;  // tokens from the warp's, this lane's first on
    Chunk<T, N> x[kItems<N>], y[kItems<N>];
#pragma unroll
    for (int u = 0; u < kItems<N>; ++u) {
      if (u * apart < mine && at.at >= 0) x[u].load(src + at.at);
      if (u * apart < mine && second >= 0) y[u].load(src + second);
      src += apart * step;
    }
    float fx[kItems<N>][N], fy[kItems<N>][N], most = 0.f;  // fmaxf passes over a NaN
#pragma unroll
    for (int u = 0; u < kItems<N>; ++u) {
      if (u * apart >= left) break;  // of the whole warp
      const bool there = working && u * apart < mine;
      asm volatile("" ::: "memory");  // an item's angles at a time: all at once do not fit the registers
      x[u].to(fx[u]);
      y[u].to(fy[u]);
      if (!value && a.rot > 0) {
        float cs[2 * N];
        if (there) load_angles<N>(cs, a.rope, p.pos + lane_token + u * apart, a.rot, at, i);
        turn_chunks(fx[u], fy[u], cs, at);
      }
      float first = 0.f, other = 0.f;
#pragma unroll
      for (int k = 0; k < N; ++k) {
        first = fmaxf(first, fabsf(fx[u][k]));
        other = fmaxf(other, fabsf(fy[u][k]));
      }
      if (there && at.at >= 0) most = fmaxf(most, first);
      if (there && second >= 0) most = fmaxf(most, other);
    }
    const int e = page_unit<N>(c, s, sm, most, clamp_exponent(old), codes, p.slot);
    const float unit = power_of_two(-e);
    codes += lane_token * c.slot_stride;
#pragma unroll
    for (int u = 0; u < kItems<N>; ++u) {
      if (u * apart >= left) break;
      if (u * apart < mine && at.at >= 0) store_codes(codes + at.at, fx[u], unit);
      if (u * apart < mine && second >= 0) store_codes(codes + second, fy[u], unit);
      codes += apart * c.slot_stride;
    }
    if (in_team == 0 && lane == 0) *exp = (int8_t)e;
  }
}

// The same by reading twice, for pages that hold more, and element by element (N = 1).
template <typename T, int N>
__device__ __forceinline__ void fill_pages_twice(const AppendArgs& a, const HeadShape& s, Shared& sm, int first_task, int tasks) {
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const retrace_kv_cache& c = a.cache;
  const int D = c.head_dim, L = s.lanes;

  // A lane has the same chunks of tokens `apart` from one another (single elements: of 32 of a token's lanes
  // at a time).
  const int team = warp / s.team, in_team = warp % s.team;
  const int steps = N == 1 ? (L + 31) / 32 : 1, abreast = N == 1 && steps > 1 ? 1 : 32 / L;  // tokens of a warp at a time
  const int lane_token = abreast > 1 || steps == 1 ? lane / L : 0, lane_chunk = steps == 1 ? lane % L : lane;
  const int apart = s.team * abreast;
  const bool working = lane_token < abreast;
  for (int task = team; task < sm.pieces * tasks; task += kWarps / s.team) {
    const PagePiece p = sm.piece[task / tasks];
    const int head = first_task + task % tasks, h = head >> 1;
    const bool value = head & 1;
    const long long step = value ? a.v_token : a.k_token;
    const T* src = (value ? static_cast<const T*>(a.v) + h * a.v_head : static_cast<const T*>(a.k) + h * a.k_head) + p.t * step;
    uint8_t* codes = static_cast<uint8_t*>(value ? c.v : c.k) + p.page * c.page_stride + h * c.head_stride + (long long)p.slot * c.slot_stride;
    int8_t* exp = (value ? a.v_exp : a.k_exp) + p.page * a.exp_page + h * a.exp_head;
    const int old = p.slot > 0 ? clamp_exponent(*exp) : -kMostExponent;
    // A lane's chunks: first elements, -1: none.
    struct Chunks {
      Place at;
      int second;
    };
    auto chunks_of = [&](int i) {
      Chunks x{Place{false, false, -1}, -1};
      if (!working || i >= L) return x;
      if (value) {
        if (i * N < D) x.at.at = i * N;
        if ((i + L) * N < D) x.second = (i + L) * N;
      } else {
        x.at = place_of<N>(s, a.rot, i);
        if (x.at.pair) x.second = x.at.at + s.step;
      }
      return x;
    };
    const Chunks mine = chunks_of(lane_chunk);
    // Item q of this lane: a token, and with several steps chunks of its own.
    const int items = (p.count + apart - 1) / apart * steps;
    auto token_of = [&](int q) { return (steps == 1 ? q : q / steps) * apart + in_team * abreast + lane_token; };
    auto item_chunk = [&](int q) { return steps == 1 ? lane_chunk : q % steps * 32 + lane; };
    auto item_chunks = [&](int q) { return N == 1 && steps > 1 ? chunks_of(item_chunk(q)) : mine; };
    // f(token, chunks, rotated first, rotated second) for all of this lane's items.
    auto visit = [&](auto&& f) {
#pragma unroll 1
      for (int q = 0; q < items; q += kAhead) {
        Chunk<T, N> x[kAhead], y[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
          const int t = token_of(q + u);
          const Chunks w = item_chunks(q + u);
          const T* from = src + t * step;
          if (t < p.count && w.at.at >= 0) x[u].load(from + w.at.at);
          if (t < p.count && w.second >= 0) y[u].load(from + w.second);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
          const int t = token_of(q + u);
          const Chunks w = item_chunks(q + u);
          if (t >= p.count) break;
          float cs[2 * N], fx[N], fy[N];
          if (!value && a.rot > 0) load_angles<N>(cs, a.rope, p.pos + t, a.rot, w.at, item_chunk(q + u));
          turned(x[u], y[u], cs, !value && a.rot > 0 ? w.at : Place{false, false, 0}, fx, fy);
          f(t, w, fx, fy);
        }
      }
    };
    float most = 0.f;  // fmaxf passes over a NaN
    visit([&](int, const Chunks& w, const float (&fx)[N], const float (&fy)[N]) {
#pragma unroll
      for (int k = 0; k < N; ++k) {
        if (w.at.at >= 0) most = fmaxf(most, fabsf(fx[k]));
        if (w.second >= 0) most = fmaxf(most, fabsf(fy[k]));
      }
    });
    const int e = page_unit<N>(c, s, sm, most, old, codes, p.slot);
    const float unit = power_of_two(-e);
    visit([&](int t, const Chunks& w, const float (&fx)[N], const float (&fy)[N]) {
      uint8_t* to = codes + t * c.slot_stride;
      if (w.at.at >= 0) store_codes(to + w.at.at, fx, unit);
      if (w.second >= 0) store_codes(to + w.second, fy, unit);
    });
    if (in_team == 0 && lane == 0) *exp = (int8_t)e;
  }
}

// kKeep: what a team has of a page fits its registers.
template <typename T, int N, bool kKeep>
__global__ void __launch_bounds__(kThreads, kCtasPerSm) kv_append_fp8_kernel(const __grid_constant__ AppendArgs a, const __grid_constant__ HeadShape s) {
  __shared__ Shared sm;
  pdl_launch_dependents();
  pdl_wait();
  // Some CTAs have the pages, the others the queries.
  const retrace_kv_cache& c = a.cache;
  if ((int)blockIdx.x < s.page_ctas) {
    // A share of the heads (k and v apart) of a chunk of tokens: pages begin anywhere in a chunk, and small
    // chunks have one or three of them.
    const int share = blockIdx.x % s.shares, first = share * s.share_tasks, tasks = min(s.share_tasks, 2 * c.kv_heads - first);
    for (int t0 = blockIdx.x / s.shares * s.tokens; t0 < a.T; t0 += s.page_ctas / s.shares * s.tokens) {
      const int tokens = min(s.tokens, a.T - t0);
      ask_for(static_cast<const T*>(a.k) + first / 2 * a.k_head, a.k_token, a.k_head, (tasks + 1) / 2, c.head_dim, t0, tokens);
      ask_for(static_cast<const T*>(a.v) + first / 2 * a.v_head, a.v_token, a.v_head, (tasks + 1) / 2, c.head_dim, t0, tokens);
      __syncthreads();  // the tokens before are through
      if (threadIdx.x < 32) find_pieces(a, sm, t0, tokens, threadIdx.x);
      __syncthreads();
      if constexpr (kKeep)
        fill_pages<T, N>(a, s, sm, first, tasks);
      else
        fill_pages_twice<T, N>(a, s, sm, first, tasks);
    }
  } else {
    for (int t0 = (blockIdx.x - s.page_ctas) * s.query_tokens; t0 < a.T; t0 += (gridDim.x - s.page_ctas) * s.query_tokens) {
      const int tokens = min(s.query_tokens, a.T - t0);
      ask_for(static_cast<const T*>(a.q), a.q_token, a.q_head, a.q_heads, c.head_dim, t0, tokens);
      __syncthreads();
      if (threadIdx.x < 32) sm.pos[threadIdx.x] = place_token(a, a.q_start ? 0 : a.T / a.B, t0, threadIdx.x).pos;
      __syncthreads();
      rotate_queries<T, N>(a, s, sm, t0, tokens);
    }
  }
}

// Nothing is turned, and the heads have two halves of whole chunks.
template <int N>
bool halves_of(const AppendArgs& a) {
  return N > 1 && a.rot == 0 && a.cache.head_dim % (2 * N) == 0;
}

template <typename T, int N>
cudaError_t launch(const AppendArgs& a, cudaStream_t stream) {
  HeadShape s{};
  const int D = a.cache.head_dim;
  const bool halves = !a.interleaved || N == 1;
  s.pairs = halves ? a.rot / 2 / N : 0;
  s.inside = halves ? 0 : a.rot / N;
  s.copies = (D - a.rot) / N;
  s.step = a.interleaved ? 1 : a.rot / 2;
  if (halves_of<N>(a)) {
    s.pairs = D / 2 / N;
    s.copies = 0;
    s.step = D / 2;
  }
  s.lanes = s.pairs + s.inside + s.copies;
  const int groups = kThreads / s.lanes, share = (a.q_heads + kHeadsEach - 1) / kHeadsEach;
  s.per_token = share < 1 ? 1 : groups < share ? groups : share;
  // As many warps to a page's tokens as keep them.
  const int each = kItems<N> * std::max(1, 32 / s.lanes);
  for (s.team = 1; s.team < kWarps && s.team * each < std::min(a.cache.page_size, a.T);) s.team *= 2;
  DeviceInfo dev;
  const cudaError_t e = device_info(&dev);
  if (e != cudaSuccess) return e;
  // Chunks of tokens, and of the heads, so that there are about as many CTAs as fit.
  const int resident = dev.sm_count * kCtasPerSm, tasks = 2 * a.cache.kv_heads;
  auto chunks_of = [&](int tokens) { return (a.T + tokens - 1) / tokens; };
  s.tokens = std::min(std::max((a.T + resident - 1) / resident, 1), kMostTokens);
  if (a.T >= resident) s.tokens = kMostTokens;
  s.share_tasks = tasks;
  while (s.share_tasks % 4 == 0 && chunks_of(s.tokens) * (tasks / s.share_tasks) * 2 <= 2 * resident) s.share_tasks /= 2;
  s.shares = (tasks + s.share_tasks - 1) / s.share_tasks;
  s.page_ctas = std::min(chunks_of(s.tokens), 4 * resident) * s.shares;
  int ctas = s.page_ctas;
  if (a.q) {
    s.query_tokens = std::min(std::max((a.T + resident - 1) / resident, 1), kMostTokens);
    ctas += chunks_of(s.query_tokens);
  }
  const dim3 grid(ctas), block(kThreads);
  if constexpr (N > 1)
    if (s.team * each >= std::min(a.cache.page_size, a.T))
      return launch_dependent(kv_append_fp8_kernel<T, N, true>, grid, block, 0, stream, 1u, a, s);
  return launch_dependent(kv_append_fp8_kernel<T, N, false>, grid, block, 0, stream, 1u, a, s);
}

template <typename T>
cudaError_t launch_typed(const AppendArgs& a, cudaStream_t stream) {
  constexpr int N = 16 / sizeof(T);
  auto whole = [](long long x) { return x % N == 0; };
  auto aligned = [](const void* p, int bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; };
  const retrace_kv_cache& c = a.cache;
  bool vec = whole(c.head_dim) && whole(a.interleaved ? a.rot : a.rot / 2) && whole(c.head_stride) &&
             whole(c.slot_stride) && whole(c.page_stride) && whole(a.k_token) && whole(a.k_head) && whole(a.v_token) &&
             whole(a.v_head) && aligned(a.k, 16) && aligned(a.v, 16) && aligned(c.k, N) && aligned(c.v, N) && aligned(a.rope, 16);
  if (a.q)
    vec = vec && whole(a.q_token) && whole(a.q_head) && whole(a.qo_token) && whole(a.qo_head) && aligned(a.q, 16) &&
          aligned(a.q_out, 16);
  // A head's lanes fit a warp (256 numbers in fp32 need 64 where they are copied: element by element).
  const int pairs = a.interleaved ? 0 : a.rot / 2, lanes = halves_of<N>(a) ? c.head_dim / 2 / N : (a.interleaved ? a.rot : pairs) / N + (c.head_dim - a.rot) / N;
  return vec && lanes <= 32 ? launch<T, N>(a, stream) : launch<T, 1>(a, stream);
}

}  // namespace

cudaError_t launch_kv_append_fp8(const AppendArgs& a, cudaStream_t stream) {
  return a.dtype == RETRACE_BF16 ? launch_typed<__nv_bfloat16>(a, stream) : launch_typed<float>(a, stream);
}

}  // namespace retrace
