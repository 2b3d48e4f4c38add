// Appending keys and values to a paged cache in 8 bits, rotating keys and queries on the way.
//
// With x' the rotated elements, a page's new tokens and a head: a = max |x'|, e the least
// exponent with a <= 448 2^e, e = max(e, the page's) where the page holds earlier tokens, codes
// round(x' 2^-e).  The maximum comes before the first code, so a warp takes a page's new
// tokens of one head (k or v) as a whole and keeps what it has loaded (16 tokens of 128 in
// bf16) in registers between the two; the rest of larger pages is read again, from L1.
// Each element is read once from HBM and written once: bound by that.
#include "fp8.cuh"
#include "tokens.cuh"

namespace retrace {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kCtasPerSm = 3;
constexpr int kMostTokens = 32;  // of a CTA at a time
constexpr int kHeadsEach = 3;    // query heads whose loads a thread has in flight
constexpr int kHold = 4;         // chunks of a page's tokens that a lane keeps

template <typename T, int N>
struct Chunk {  // N elements, loaded and stored as one access
  static_assert(N == 1 || N * sizeof(T) == 16, "one element or 16 bytes");
  T e[N];
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (N == 1) e[0] = *p;
    else *reinterpret_cast<uint4*>(e) = *reinterpret_cast<const uint4*>(p);
  }
  __device__ __forceinline__ void store(T* p) const {
    if constexpr (N == 1) *p = e[0];
    else *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(e);
  }
};

// Lanes of a rotated head: first the chunks that rotate with a partner chunk (halves; single
// elements also when interleaved), then those whose pairs lie inside (interleaved), then
// those that are copied.  Lane i of a head of v has the chunks i and i + lanes.
struct HeadShape {
  int pairs, inside, copies, lanes;  // lanes: their sum
  int step;                          // from a chunk to its partner, elements
  FastDivide by_lanes;
  int tokens;     // of a CTA at a time
  int per_token;  // groups of lanes that share a token's query heads
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

// Cosines and sines of a lane's pairs.
template <int N>
__device__ __forceinline__ void load_angles(float (&cs)[2 * N], const float* rope, int pos, int rot, const Place& p, int i) {
  constexpr int kLoad = N > 1 ? 4 : 2;
  if (!p.pair && !p.inside) return;
  const float* r = rope + (long long)pos * rot + (p.inside ? p.at : i * 2 * N);
  const int n = p.inside ? N : 2 * N;
#pragma unroll
  for (int k = 0; k < 2 * N; k += kLoad) {
    if (k >= n) break;
    if constexpr (kLoad == 4) {
      *reinterpret_cast<float4*>(cs + k) = __ldg(reinterpret_cast<const float4*>(r + k));
    } else {
      cs[0] = r[0];
      cs[1] = r[1];
    }
  }
}

// (v, w) turned by (c, s); the products are rounded before they are added.
__device__ __forceinline__ void turn(float& v, float& w, float c, float s) {
  const float a = __fsub_rn(__fmul_rn(v, c), __fmul_rn(w, s));
  w = __fadd_rn(__fmul_rn(w, c), __fmul_rn(v, s));
  v = a;
}
template <typename T, int N>
__device__ __forceinline__ void turned(const Chunk<T, N>& x, const Chunk<T, N>& y, const float (&cs)[2 * N], const Place& p,
                                       float (&fx)[N], float (&fy)[N]) {
#pragma unroll
  for (int k = 0; k < N; ++k) {
    fx[k] = to_f32(x.e[k]);
    fy[k] = to_f32(y.e[k]);
  }
  if (p.pair) {
#pragma unroll
    for (int k = 0; k < N; ++k) turn(fx[k], fy[k], cs[2 * k], cs[2 * k + 1]);
  } else if (N > 1 && p.inside) {
#pragma unroll
    for (int k = 0; k + 1 < N; k += 2) turn(fx[k], fx[k + 1], cs[k], cs[k + 1]);
  }
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

// The new tokens of a sequence in one page.
struct PagePiece {
  int t, count;  // first token, and how many
  int pos;       // of the first
  int page, slot;
};

template <typename T, int N>
__global__ void __launch_bounds__(kThreads, kCtasPerSm) kv_append_fp8_kernel(const __grid_constant__ AppendArgs a, HeadShape s) {
  __shared__ int s_pos[kMostTokens];  // -1: caches nothing, its query is zero; -2: of no sequence
  __shared__ PagePiece s_piece[kMostTokens];
  __shared__ int s_pieces;
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  const retrace_kv_cache& c = a.cache;
  const int uniform = a.q_start ? 0 : a.T / a.B, D = c.head_dim, L = s.lanes;
  pdl_launch_dependents();
  pdl_wait();

  for (int t0 = blockIdx.x * s.tokens; t0 < a.T; t0 += gridDim.x * s.tokens) {
    const int tokens = min(s.tokens, a.T - t0);
    __syncthreads();  // the tokens before are through
    for (int k = warp; k < tokens; k += kWarps) {
      const int t = t0 + k;
      int first;
      const int b = sequence_of(a.q_start, a.B, uniform, t, lane, &first);
      if (lane != 0) continue;
      PagePiece piece{t, 0, 0, -1, 0};
      int pos = -2;
      if (b >= 0) {
        pos = cached_tokens(a.cache_len, b) + (t - first);
        if (pos < 0 || (a.rope && pos >= a.rope_positions)) pos = -1;
        const int slot = pos % c.page_size;
        if (pos >= 0 && (t == first || slot == 0)) {
          const int end = a.q_start ? min(a.q_start[b + 1], a.T) : first + uniform;
          piece.count = min(end - t, c.page_size - slot);
          if (a.rope) piece.count = min(piece.count, a.rope_positions - pos);
          piece.pos = pos;
          piece.page = page_of(c, b, pos / c.page_size);
          piece.slot = slot;
        }
      }
      s_pos[k] = pos;
      s_piece[k] = piece;
    }
    __syncthreads();
    if (warp == 0) {  // pieces that have a page, one after another
      const PagePiece mine = lane < tokens ? s_piece[lane] : PagePiece{0, 0, 0, -1, 0};
      const unsigned there = __ballot_sync(0xFFFFFFFFu, mine.page >= 0);
      __syncwarp();
      if (mine.page >= 0) s_piece[__popc(there & ((1u << lane) - 1u))] = mine;
      if (lane == 0) s_pieces = __popc(there);
    }
    __syncthreads();

    // Keys and values: a warp to a page's tokens of one head.
    const int tasks = s_pieces * 2 * c.kv_heads;
    for (int task = warp; task < tasks; task += kWarps) {
      const PagePiece p = s_piece[task / (2 * c.kv_heads)];
      const int h = task % (2 * c.kv_heads) >> 1;
      const bool value = task & 1;
      const T* src = value ? static_cast<const T*>(a.v) + h * a.v_head : static_cast<const T*>(a.k) + h * a.k_head;
      const long long step = value ? a.v_token : a.k_token;
      uint8_t* codes = static_cast<uint8_t*>(value ? c.v : c.k) + p.page * c.page_stride + h * c.head_stride;
      int8_t* exp = (value ? a.v_exp : a.k_exp) + p.page * a.exp_page + h * a.exp_head;
      const int old = p.slot > 0 ? clamp_exponent(*exp) : -kMostExponent;
      const int total = p.count * L;

      struct Item {
        Place at;
        int token, second;  // second: the other chunk's first element, -1: none
      };
      auto item = [&](int idx) {
        Item it;
        it.token = s.by_lanes(idx);
        const int i = idx - it.token * L;
        if (value) {
          it.at = Place{false, false, i * N < D ? i * N : -1};
          it.second = (i + L) * N < D ? (i + L) * N : -1;
        } else {
          it.at = place_of<N>(s, a.rot, i);
          it.second = it.at.pair ? it.at.at + s.step : -1;
        }
        return it;
      };
      auto load = [&](int idx, Chunk<T, N>& x, Chunk<T, N>& y) {
        const Item it = item(idx);
        const T* from = src + (p.t + it.token) * step;
        if (it.at.at >= 0) x.load(from + it.at.at);
        if (it.second >= 0) y.load(from + it.second);
      };
      auto rotated = [&](int idx, const Item& it, const Chunk<T, N>& x, const Chunk<T, N>& y, float (&fx)[N], float (&fy)[N]) {
        float cs[2 * N];
        if (!value && a.rope) load_angles<N>(cs, a.rope, p.pos + it.token, a.rot, it.at, idx - it.token * L);
        turned(x, y, cs, it.at, fx, fy);
      };
      float most = 0.f;
      auto weigh = [&](int idx, const Chunk<T, N>& x, const Chunk<T, N>& y) {
        const Item it = item(idx);
        float fx[N], fy[N];
        rotated(idx, it, x, y, fx, fy);
        // fmaxf passes over a NaN
#pragma unroll
        for (int k = 0; k < N; ++k) {
          if (it.at.at >= 0) most = fmaxf(most, fabsf(fx[k]));
          if (it.second >= 0) most = fmaxf(most, fabsf(fy[k]));
        }
      };
      Chunk<T, N> x[kHold], y[kHold];
#pragma unroll
      for (int u = 0; u < kHold; ++u)
        if (lane + u * 32 < total) load(lane + u * 32, x[u], y[u]);
#pragma unroll
      for (int u = 0; u < kHold; ++u)
        if (lane + u * 32 < total) weigh(lane + u * 32, x[u], y[u]);
      for (int idx = lane + kHold * 32; idx < total; idx += 32) {
        Chunk<T, N> v, w;
        load(idx, v, w);
        weigh(idx, v, w);
      }
      // not negative: the order of the bits is that of the numbers
      const float top = __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(most)));
      const int e = max(top > 0.f ? exponent_for(top) : -kMostExponent, old);
      if (p.slot > 0 && e > old) {
        // what the page holds already, in the new unit
        const float down = power_of_two(old - e);
        const int words = N >= 4 ? D / 4 : D;
        for (int idx = lane; idx < p.slot * words; idx += 32) {
          uint8_t* at = codes + (long long)(idx / words) * c.slot_stride + idx % words * (N >= 4 ? 4 : 1);
          if constexpr (N >= 4) {
            uint32_t& w = *reinterpret_cast<uint32_t*>(at);
            const float2 lo = e4m3_floats(w & 0xFFFFu), hi = e4m3_floats(w >> 16);
            w = to_e4m3x2(lo.x * down, lo.y * down) | to_e4m3x2(hi.x * down, hi.y * down) << 16;
          } else {
            *at = (uint8_t)to_e4m3x2(e4m3_floats(*at).x * down, 0.f);
          }
        }
      }
      __syncwarp();
      if (lane == 0) *exp = (int8_t)e;
      const float unit = power_of_two(-e);
      auto put = [&](int idx, const Chunk<T, N>& x, const Chunk<T, N>& y) {
        const Item it = item(idx);
        float fx[N], fy[N];
        rotated(idx, it, x, y, fx, fy);
        uint8_t* to = codes + (long long)(p.slot + it.token) * c.slot_stride;
        if (it.at.at >= 0) store_codes(to + it.at.at, fx, unit);
        if (it.second >= 0) store_codes(to + it.second, fy, unit);
      };
#pragma unroll
      for (int u = 0; u < kHold; ++u)
        if (lane + u * 32 < total) put(lane + u * 32, x[u], y[u]);
      for (int idx = lane + kHold * 32; idx < total; idx += 32) {
        Chunk<T, N> v, w;
        load(idx, v, w);
        put(idx, v, w);
      }
    }

    // Queries: lane i of a group owns the same pairs in every head of its token.
    if (!a.q) continue;
    const int group = tid / L, i = tid % L, groups = kThreads / L, each = groups / s.per_token;
    if (group >= each * s.per_token) continue;
    const Place at = place_of<N>(s, a.rot, i);
    for (int k = group / s.per_token; k < tokens; k += each) {
      const int pos = s_pos[k], t = t0 + k;
      if (pos == -2) continue;
      float cs[2 * N];
      if (pos >= 0 && a.rope) load_angles<N>(cs, a.rope, pos, a.rot, at, i);
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
          turned(x[u], y[u], cs, at, fx, fy);
#pragma unroll
          for (int j = 0; j < N; ++j) {
            if (at.pair || (N > 1 && at.inside) || pos < 0) {  // else copied as it is
              x[u].e[j] = from_f32<T>(pos < 0 ? 0.f : fx[j]);
              y[u].e[j] = from_f32<T>(pos < 0 ? 0.f : fy[j]);
            }
          }
          x[u].store(to);
          if (at.pair) y[u].store(to + s.step);
        }
      }
    }
  }
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
  s.lanes = s.pairs + s.inside + s.copies;
  s.by_lanes = FastDivide::of(s.lanes);
  const int groups = kThreads / s.lanes, share = (a.q_heads + kHeadsEach - 1) / kHeadsEach;
  s.per_token = share < 1 ? 1 : groups < share ? groups : share;
  DeviceInfo dev;
  const cudaError_t e = device_info(&dev);
  if (e != cudaSuccess) return e;
  // Few tokens to a CTA where there are few, so that all CTAs have some.
  const int resident = dev.sm_count * kCtasPerSm, even = (a.T + resident - 1) / resident;
  s.tokens = even < 1 ? 1 : even < kMostTokens ? even : kMostTokens;
  const int all = (a.T + s.tokens - 1) / s.tokens;
  return launch_dependent(kv_append_fp8_kernel<T, N>, dim3(all < resident ? all : resident), dim3(kThreads), 0, stream, 1u, a, s);
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
  return vec ? launch<T, N>(a, stream) : launch<T, 1>(a, stream);
}

}  // namespace

cudaError_t launch_kv_append_fp8(const AppendArgs& a, cudaStream_t stream) {
  return a.dtype == RETRACE_BF16 ? launch_typed<__nv_bfloat16>(a, stream) : launch_typed<float>(a, stream);
}

}  // namespace retrace
