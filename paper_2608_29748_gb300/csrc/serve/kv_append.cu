// Appending keys and values to the paged cache, rotating keys and queries on the way.
//
// A pair (x, y) of a rotated head at position p becomes (x c - y s, y c + x s),
// (c, s) = rope[p, pair].  Each element is read once and written once: HBM, at
// 0.75 flop per byte.  A CTA takes one token, or several where a token has few
// heads; within it lane i of a group owns the same pairs in every head, so their
// cosines and sines are loaded once and stay in registers over the heads.
#include "serve.h"
#include "tokens.cuh"

namespace retrace {
namespace {

constexpr int kAppendThreads = 256;

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

// Lanes of a head: first the chunks that rotate with a partner chunk (halves;
// single elements also when interleaved), then those whose pairs lie inside
// (interleaved), then those that are copied.
struct AppendShape {
  int pairs, inside, copies, lanes;  // lanes: their sum
  int step;                          // from a chunk to its partner, elements
  int groups;                        // head groups of a CTA
  int per_token;                     // groups a token takes
};

template <typename T, int N>
__global__ void __launch_bounds__(kAppendThreads) kv_append_kernel(AppendArgs a, AppendShape s) {
  __shared__ int s_seq[kAppendThreads], s_pos[kAppendThreads];
  const int tokens = s.groups / s.per_token;  // tokens of this CTA
  const int t0 = blockIdx.x * tokens;
  // Which sequence a token belongs to: without a list by division, else by one
  // warp's search, 32 starts at a time.
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  for (int i = warp; i < tokens; i += kAppendThreads / 32) {
    const int t = t0 + i;
    if (t >= a.T) break;
    int b = -1, first = 0;
    if (!a.q_start) {
      const int n = a.T / a.B;
      b = t / n;
      first = b * n;
    } else {
      int lo = 0, n = a.B;  // the last start <= t lies in [lo, lo + n), if any
      while (n > 32) {
        const int step = (n + 31) / 32;
        const int at = lo + lane * step;
        const bool below = at < lo + n && a.q_start[at] <= t;
        const int k = __popc(__ballot_sync(0xFFFFFFFFu, below));
        if (k == 0) break;
        const int end = lo + n;
        lo += (k - 1) * step;
        n = min(step, end - lo);
      }
      const bool below = lane < n && lane < 32 && a.q_start[lo + lane] <= t;
      const int k = __popc(__ballot_sync(0xFFFFFFFFu, below));
      if (k > 0) {
        b = lo + k - 1;
        first = a.q_start[b];
        if (t >= a.q_start[b + 1] || first < 0) b = -1;  // a token of no sequence
      }
    }
    if (lane == 0) {
      s_seq[i] = b;
      s_pos[i] = b < 0 ? -1 : cached_tokens(a.cache_len, b) + (t - first);
    }
  }
  __syncthreads();

  const int group = threadIdx.x / s.lanes, i = threadIdx.x % s.lanes;
  if (group >= s.groups) return;
  const int tl = group / s.per_token, t = t0 + tl;
  if (tl >= tokens || t >= a.T) return;
  const int b = s_seq[tl];
  if (b < 0) return;
  const int pos = s_pos[tl];
  const bool placed = pos >= 0 && (!a.rope || pos < a.rope_positions);
  const int D = a.cache.head_dim;
  const int page = placed ? page_of(a.cache, b, pos / a.cache.page_size) : -1;
  const long long slot = page < 0 ? 0 : page * a.cache.page_stride + (pos % a.cache.page_size) * a.cache.slot_stride;

  // This lane's chunk of a rotated head, its partner, and their cosines and sines.
  const bool pair = i < s.pairs, inside = !pair && i < s.pairs + s.inside;
  int at;
  if (pair)
    at = s.step == 1 ? 2 * i : i * N;
  else if (inside)
    at = (i - s.pairs) * N;
  else
    at = a.rot + (i - s.pairs - s.inside) * N;
  constexpr int kLoad = N > 1 ? 4 : 2;
  float cs[2 * N];
  if (placed && (pair || inside)) {
    const float* r = a.rope + (long long)pos * a.rot + (inside ? at : i * 2 * N);
    const int n = inside ? N : 2 * N;
#pragma unroll
    for (int k = 0; k < 2 * N; k += kLoad) {
      if (k >= n) break;
      if constexpr (kLoad == 4) {
        *reinterpret_cast<float4*>(cs + k) = *reinterpret_cast<const float4*>(r + k);
      } else {
        cs[0] = r[0];
        cs[1] = r[1];
      }
    }
  }

  const int rotated = a.q_heads + a.cache.kv_heads, heads = rotated + a.cache.kv_heads;
  for (int h = group % s.per_token; h < heads; h += s.per_token) {
    if (h >= rotated) {  // a value head: every chunk is copied
      if (page < 0) continue;
      const int kh = h - rotated;
      const T* src = static_cast<const T*>(a.v) + (long long)t * a.v_token + kh * a.v_head;
      T* dst = static_cast<T*>(a.cache.v) + slot + kh * a.cache.head_stride;
      Chunk<T, N> x, y;
      const int c0 = i * N, c1 = (i + s.lanes) * N;
      const bool one = c0 < D, two = c1 < D;
      if (one) x.load(src + c0);
      if (two) y.load(src + c1);
      if (one) x.store(dst + c0);
      if (two) y.store(dst + c1);
      continue;
    }
    const bool query = h < a.q_heads;
    const int kh = h - a.q_heads;
    if (!query && page < 0) continue;
    const T* src = query ? static_cast<const T*>(a.q) + (long long)t * a.q_token + h * a.q_head
                         : static_cast<const T*>(a.k) + (long long)t * a.k_token + kh * a.k_head;
    T* dst = query ? static_cast<T*>(a.q_out) + (long long)t * a.qo_token + h * a.qo_head
                   : static_cast<T*>(a.cache.k) + slot + kh * a.cache.head_stride;
    Chunk<T, N> x, y;
    if (!placed) {  // a query without a place among the angles
#pragma unroll
      for (int k = 0; k < N; ++k) x.e[k] = from_f32<T>(0.f);
      x.store(dst + at);
      if (pair) x.store(dst + at + s.step);
      continue;
    }
    x.load(src + at);
    if (pair) {
      y.load(src + at + s.step);
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const float u = to_f32(x.e[k]), w = to_f32(y.e[k]);
        x.e[k] = from_f32<T>(u * cs[2 * k] - w * cs[2 * k + 1]);
        y.e[k] = from_f32<T>(w * cs[2 * k] + u * cs[2 * k + 1]);
      }
      x.store(dst + at);
      y.store(dst + at + s.step);
      continue;
    }
    if constexpr (N > 1) {
      if (inside) {
#pragma unroll
        for (int k = 0; k < N; k += 2) {
          const float u = to_f32(x.e[k]), w = to_f32(x.e[k + 1]);
          x.e[k] = from_f32<T>(u * cs[k] - w * cs[k + 1]);
          x.e[k + 1] = from_f32<T>(w * cs[k] + u * cs[k + 1]);
        }
      }
    }
    x.store(dst + at);
  }
}

template <typename T, int N>
cudaError_t launch(const AppendArgs& a, cudaStream_t stream) {
  AppendShape s{};
  const int D = a.cache.head_dim;
  const bool halves = !a.interleaved || N == 1;
  s.pairs = halves ? a.rot / 2 / N : 0;
  s.inside = halves ? 0 : a.rot / N;
  s.copies = (D - a.rot) / N;
  s.step = a.interleaved ? 1 : a.rot / 2;
  s.lanes = s.pairs + s.inside + s.copies;
  const int heads = a.q_heads + 2 * a.cache.kv_heads;
  s.groups = kAppendThreads / s.lanes;
  s.per_token = s.groups < heads ? s.groups : heads;
  const int tokens = s.groups / s.per_token;
  kv_append_kernel<T, N><<<(a.T + tokens - 1) / tokens, kAppendThreads, 0, stream>>>(a, s);
  return cudaGetLastError();
}

template <typename T>
cudaError_t launch_typed(const AppendArgs& a, cudaStream_t stream) {
  constexpr int N = 16 / sizeof(T);
  auto whole = [](long long x) { return x % N == 0; };
  auto aligned = [](const void* p) { return ((uintptr_t)p & 15u) == 0; };
  const retrace_kv_cache& c = a.cache;
  bool vec = whole(c.head_dim) && whole(a.interleaved ? a.rot : a.rot / 2) && whole(c.head_stride) &&
             whole(c.slot_stride) && whole(c.page_stride) && whole(a.k_token) && whole(a.k_head) && whole(a.v_token) &&
             whole(a.v_head) && aligned(a.k) && aligned(a.v) && aligned(c.k) && aligned(c.v) && aligned(a.rope);
  if (a.q)
    vec = vec && whole(a.q_token) && whole(a.q_head) && whole(a.qo_token) && whole(a.qo_head) && aligned(a.q) &&
          aligned(a.q_out);
  return vec ? launch<T, N>(a, stream) : launch<T, 1>(a, stream);
}

}  // namespace

cudaError_t launch_kv_append(const AppendArgs& a, cudaStream_t stream) {
  return a.cache.dtype == RETRACE_BF16 ? launch_typed<__nv_bfloat16>(a, stream) : launch_typed<float>(a, stream);
}

}  // namespace retrace
