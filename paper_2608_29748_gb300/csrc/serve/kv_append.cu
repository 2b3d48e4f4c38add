// Appending keys and values to the paged cache, rotating keys and queries on the way.
//
// A pair (x, y) of a rotated head at position p becomes (x c - y s, y c + x s),
// (c, s) = rope[p, pair].  Each element is read once and written once: HBM, at
// 0.75 flop per byte.  A CTA takes one token, or several where a token has few
// heads; within it lane i of a group owns the same pairs in every head, so their
// cosines and sines are loaded once and stay in registers over the heads.  256 blocks of 17
// tokens, 32 + 2 x 8 heads of 128, bf16: 23.7 us, 4.6 TB/s of reads and writes; other numbers of
// CTAs and of heads in flight took 27.3 to 30.5.
#include "serve.h"
#include "tokens.cuh"

namespace retrace {
namespace {

constexpr int kAppendThreads = 256;
constexpr int kCtasPerSm = 4;
constexpr int kHeadsEach = 3;  // heads whose loads a thread has in flight

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
__global__ void __launch_bounds__(kAppendThreads, kCtasPerSm) kv_append_kernel(const __grid_constant__ AppendArgs a, AppendShape s) {
  __shared__ int s_seq[kAppendThreads], s_pos[kAppendThreads];
  pdl_wait();
  const int tokens = s.groups / s.per_token;  // tokens of this CTA
  const int group = threadIdx.x / s.lanes, i = threadIdx.x % s.lanes;
  const int tl = group / s.per_token, first_head = group % s.per_token;
  const int uniform = a.q_start ? 0 : a.T / a.B;  // tokens of a sequence
  const int D = a.cache.head_dim;

  // This lane's chunk of a rotated head, and whether it has a partner or pairs inside.
  const bool pair = i < s.pairs, inside = !pair && i < s.pairs + s.inside;
  int at;
  if (pair)
    at = s.step == 1 ? 2 * i : i * N;
  else if (inside)
    at = (i - s.pairs) * N;
  else
    at = a.rot + (i - s.pairs - s.inside) * N;

  // The heads of this group, kHeadsEach at a time; what is read does not depend on where the token
  // goes, so the first ones are on their way while that is found out.
  const int rotated = a.q_heads + a.cache.kv_heads, heads = rotated + a.cache.kv_heads;
  Chunk<T, N> x[kHeadsEach], y[kHeadsEach];
  auto load = [&](int t, int h0) {
#pragma unroll
    for (int u = 0; u < kHeadsEach; ++u) {
      const int h = h0 + u * s.per_token;
      if (h >= heads) break;
      if (h >= rotated) {  // a value head: chunks i and i + lanes
        const T* src = static_cast<const T*>(a.v) + (long long)t * a.v_token + (h - rotated) * a.v_head;
        if (i * N < D) x[u].load(src + i * N);
        if ((i + s.lanes) * N < D) y[u].load(src + (i + s.lanes) * N);
      } else {
        const T* src = h < a.q_heads ? static_cast<const T*>(a.q) + (long long)t * a.q_token + h * a.q_head
                                     : static_cast<const T*>(a.k) + (long long)t * a.k_token + (h - a.q_heads) * a.k_head;
        x[u].load(src + at);
        if (pair) y[u].load(src + at + s.step);
      }
    }
  };
  for (int t0 = blockIdx.x * tokens; t0 < a.T; t0 += gridDim.x * tokens) {
    const int t = t0 + tl;
    const bool working = group < s.groups && tl < tokens && t < a.T;
    if (working) load(t, first_head);

    // Which sequence a token belongs to: without a list by division, else by one
    // warp's search, 32 starts at a time.
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    for (int k = warp; k < tokens; k += kAppendThreads / 32) {
      const int tk = t0 + k;
      if (tk >= a.T) break;
      int first;
      const int b = sequence_of(a.q_start, a.B, uniform, tk, lane, &first);
      if (lane == 0) {
        s_seq[k] = b;
        s_pos[k] = b < 0 ? -1 : cached_tokens(a.cache_len, b) + (tk - first);
      }
    }
    __syncthreads();
    const int b = working ? s_seq[tl] : -1;
    const int pos = working ? s_pos[tl] : -1;
    __syncthreads();  // both are read before the next tokens' are written
    if (b < 0) continue;
    const bool placed = pos >= 0 && (!a.rope || pos < a.rope_positions);
    const int page = placed ? page_of(a.cache, b, pos / a.cache.page_size) : -1;
    const long long slot = page < 0 ? 0 : page * a.cache.page_stride + (pos % a.cache.page_size) * a.cache.slot_stride;
    constexpr int kLoad = N > 1 ? 4 : 2;
    float cs[2 * N];  // cosines and sines of this lane's pairs
    if (placed && (pair || inside)) {
      const float* r = a.rope + (long long)pos * a.rot + (inside ? at : i * 2 * N);
      const int n = inside ? N : 2 * N;
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

    for (int h0 = first_head; h0 < heads; h0 += kHeadsEach * s.per_token) {
      if (h0 != first_head) load(t, h0);
#pragma unroll
      for (int u = 0; u < kHeadsEach; ++u) {
        const int h = h0 + u * s.per_token;
        if (h >= heads) break;
        if (h >= rotated) {
          if (page < 0) continue;
          T* dst = static_cast<T*>(a.cache.v) + slot + (h - rotated) * a.cache.head_stride;
          if (i * N < D) x[u].store(dst + i * N);
          if ((i + s.lanes) * N < D) y[u].store(dst + (i + s.lanes) * N);
          continue;
        }
        const bool query = h < a.q_heads;
        if (!query && page < 0) continue;
        T* dst = query ? static_cast<T*>(a.q_out) + (long long)t * a.qo_token + h * a.qo_head
                       : static_cast<T*>(a.cache.k) + slot + (h - a.q_heads) * a.cache.head_stride;
        if (!placed) {  // a query without a place among the angles
#pragma unroll
          for (int k = 0; k < N; ++k) x[u].e[k] = y[u].e[k] = from_f32<T>(0.f);
        } else if (pair) {
#pragma unroll
          for (int k = 0; k < N; ++k) {
            const float v = to_f32(x[u].e[k]), w = to_f32(y[u].e[k]);
            x[u].e[k] = from_f32<T>(v * cs[2 * k] - w * cs[2 * k + 1]);
            y[u].e[k] = from_f32<T>(w * cs[2 * k] + v * cs[2 * k + 1]);
          }
        } else if (N > 1 && inside) {
#pragma unroll
          for (int k = 0; k + 1 < N; k += 2) {
            const float v = to_f32(x[u].e[k]), w = to_f32(x[u].e[k + 1]);
            x[u].e[k] = from_f32<T>(v * cs[k] - w * cs[k + 1]);
            x[u].e[k + 1] = from_f32<T>(w * cs[k] + v * cs[k + 1]);
          }
        }
        x[u].store(dst + at);
        if (pair) y[u].store(dst + at + s.step);
      }
    }
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
  const int groups = (heads + kHeadsEach - 1) / kHeadsEach;
  s.per_token = s.groups < groups ? s.groups : groups;
  const int tokens = s.groups / s.per_token;
  DeviceInfo dev;
  const cudaError_t e = device_info(&dev);
  if (e != cudaSuccess) return e;
  const int all = (a.T + tokens - 1) / tokens, resident = dev.sm_count * kCtasPerSm;
  return launch_dependent(kv_append_kernel<T, N>, dim3(all < resident ? all : resident), dim3(kAppendThreads), 0, stream, 1u, a, s);
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
