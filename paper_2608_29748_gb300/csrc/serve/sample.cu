// Sampling a token from each logits row with temperature, top-k, top-p and min-p.
//
// With x the row's logits, m their maximum and T the temperature, token v weighs
// w_v = round(2^31 exp((x_v - m) / T)), a whole number, so that sums of weights do not
// depend on their order.  In the order of descending logits (the lower index first
// among equal ones) each filter keeps a prefix, and a prefix is a threshold: the
// key t of a logit, and how many of the tokens equal to it are kept.  top-k is the
// threshold at which the count reaches k, top-p the one at which the mass reaches
// ceil(p W_k), both found by radix selection over the 32-bit order-preserving keys.
// The token is then the first one in index order at which the running sum of the
// kept weights exceeds floor(u W).
#include <math.h>

#include "serve.h"
#include "../common.cuh"

namespace retrace {
namespace {

constexpr int kThreads = 1024;
constexpr int kWarps = kThreads / 32;
constexpr float kUnit = 2147483648.f;  // 2^31: the weight of the maximum

typedef unsigned long long u64;

// The settings of a row.
struct Filter {
  float inv_t, min_p, top_p;
  int top_k;
};
__device__ __forceinline__ Filter row_filter(const SampleArgs& a, int b) {
  Filter f;
  const float T = a.temperature ? a.temperature[b] : 1.f;
  f.top_k = a.top_k ? a.top_k[b] : 0;
  f.top_p = a.top_p ? a.top_p[b] : 1.f;
  f.min_p = a.min_p ? a.min_p[b] : 0.f;
  if (!(T > 0.f)) {  // greedy
    f.inv_t = 1.f;
    f.top_k = 1;
  } else {
    f.inv_t = __fdiv_rn(1.f, T);
  }
  if (f.top_k <= 0 || f.top_k > a.V) f.top_k = a.V;
  return f;
}

// exp((x - top) / T), at most 1; the maximum itself gives 1, also where it is infinite.
__device__ __forceinline__ float weight(float x, float top, float inv_t) {
  return x == top ? 1.f : expf(__fmul_rn(x - top, inv_t));
}
__device__ __forceinline__ uint32_t whole_weight(float e) { return __float2uint_rn(e * kUnit); }

template <typename T>
__device__ __forceinline__ float logit(const T* row, int v) {
  const float x = to_f32(row[v]);
  return x == x ? x : -INFINITY;
}

__device__ __forceinline__ u64 warp_sum(u64 x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
  return x;
}
// Sum over the block, to every thread.
__device__ __forceinline__ u64 block_sum(u64 x, u64* s) {
  x = warp_sum(x);
  __syncthreads();
  if (threadIdx.x % 32 == 0) s[threadIdx.x / 32] = x;
  __syncthreads();
  return warp_sum(s[threadIdx.x % 32]);
}

struct Shared {
  u64 hist[256];
  u64 part[kWarps];
  float top[kWarps];
  uint32_t digit;
  u64 above;
  int token;
  int cut;
};

// The key t with M(> t) < target <= M(>= t), where M sums `metric` over the row's
// tokens; *above = M(> t).  1 <= target <= the whole sum.
template <typename T, typename Metric>
__device__ uint32_t select_key(const T* row, int V, u64 target, Metric metric, Shared& sm, u64* above) {
  uint32_t prefix = 0;
  u64 over = 0;
  for (int shift = 24; shift >= 0; shift -= 8) {
    __syncthreads();
    for (int i = threadIdx.x; i < 256; i += kThreads) sm.hist[i] = 0;
    __syncthreads();
    const uint32_t mask = shift == 24 ? 0u : 0xFFFFFFFFu << (shift + 8);
    for (int v = threadIdx.x; v < V; v += kThreads) {
      const float x = logit(row, v);
      const uint32_t key = ordered_bits(x);
      if ((key & mask) == prefix) {
        const u64 w = metric(x);
        if (w) atomicAdd(&sm.hist[key >> shift & 255u], w);
      }
    }
    __syncthreads();
    if (threadIdx.x == 0) {
      int d = 255;
      for (; d > 0 && over + sm.hist[d] < target; --d) over += sm.hist[d];
      sm.digit = d;
      sm.above = over;
    }
    __syncthreads();
    over = sm.above;
    prefix |= sm.digit << shift;
  }
  *above = over;
  return prefix;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) sample_kernel(SampleArgs a) {
  __shared__ Shared sm;
  const int r = blockIdx.x, b = r / a.R, tid = threadIdx.x, lane = tid % 32, warp = tid / 32, V = a.V;
  const T* row = static_cast<const T*>(a.logits) + b * a.batch_stride + (r % a.R) * a.row_stride;
  const Filter f = row_filter(a, b);

  float top = -INFINITY;
  for (int v = tid; v < V; v += kThreads) top = fmaxf(top, logit(row, v));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
  if (lane == 0) sm.top[warp] = top;
  __syncthreads();
  top = sm.top[lane];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
  if (top == -INFINITY) {
    if (tid == 0) {
      a.tokens[r] = -1;
      if (a.probs) a.probs[r] = 0.f;
    }
    return;
  }
  auto mass = [&](float x) { return (u64)whole_weight(weight(x, top, f.inv_t)); };

  // The threshold: keys above t, and `ties` of those equal to it (all of them where
  // ties is V).
  uint32_t t = 0;
  u64 ties = V;
  u64 total;  // mass of what top-k keeps
  if (f.top_k < V) {
    u64 above;
    t = select_key(row, V, (u64)f.top_k, [](float) { return (u64)1; }, sm, &above);
    ties = f.top_k - above;
    u64 sum = 0;
    for (int v = tid; v < V; v += kThreads) {
      const float x = logit(row, v);
      if (ordered_bits(x) > t) sum += mass(x);
    }
    total = block_sum(sum, sm.part) + ties * mass(key_value((u64)t << 32));
  } else {
    u64 sum = 0;
    for (int v = tid; v < V; v += kThreads) sum += mass(logit(row, v));
    total = block_sum(sum, sm.part);
  }
  if (f.top_p < 1.f) {
    const double want = ceil((double)f.top_p * (double)total);
    const u64 target = want < 1.0 ? 1ull : (u64)want;
    u64 above;
    t = select_key(row, V, target, mass, sm, &above);
    const u64 one = mass(key_value((u64)t << 32));
    ties = (target - above + one - 1) / one;
  }

  // The index of the last kept token among those equal to t.
  int cut = V;
  const int seg = (V + kWarps - 1) / kWarps, v0 = warp * seg, v1 = min(V, v0 + seg);  // a warp's tokens
  {
    u64 mine = 0;
    for (int v = v0 + lane; v < v1; v += 32) mine += ordered_bits(logit(row, v)) == t;
    mine = warp_sum(mine);
    __syncthreads();
    if (lane == 0) sm.part[warp] = mine;
    if (tid == 0) sm.cut = V;
    __syncthreads();
    u64 before = 0;
    for (int w = 0; w < warp; ++w) before += sm.part[w];
    if (before < ties && ties <= before + mine) {
      u64 left = ties - before;
      for (int v = v0; v < v1; v += 32) {
        const bool is = v + lane < v1 && ordered_bits(logit(row, v + lane)) == t;
        const unsigned m = __ballot_sync(0xFFFFFFFFu, is);
        if ((u64)__popc(m) >= left) {
          if (is && (u64)__popc(m & ((2u << lane) - 1u)) == left) sm.cut = v + lane;
          break;
        }
        left -= __popc(m);
      }
    }
    __syncthreads();
    cut = sm.cut;
  }
  auto kept = [&](int v, float x) -> u64 {
    const uint32_t key = ordered_bits(x);
    if (key < t || (key == t && v > cut)) return 0;
    const float e = weight(x, top, f.inv_t);
    return x == top || !(e < f.min_p) ? whole_weight(e) : 0;
  };
  u64 mine = 0;
  for (int v = v0 + lane; v < v1; v += 32) mine += kept(v, logit(row, v));
  mine = warp_sum(mine);
  __syncthreads();
  if (lane == 0) sm.part[warp] = mine;
  __syncthreads();
  u64 before = 0, sum = 0;
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) before += sm.part[w];
    sum += sm.part[w];
  }
  const float u0 = a.uniforms[r], u = u0 > 0.f ? u0 : 0.f;
  u64 at = (u64)floor((double)u * (double)sum);
  if (u >= 1.f || at >= sum) at = sum - 1;
  if (before <= at && at < before + mine) {
    u64 run = before;
    for (int v = v0; v < v1; v += 32) {
      const float x = v + lane < v1 ? logit(row, v + lane) : -INFINITY;
      const u64 w = v + lane < v1 ? kept(v + lane, x) : 0;
      u64 upto = w;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const u64 y = __shfl_up_sync(0xFFFFFFFFu, upto, o);
        if (lane >= o) upto += y;
      }
      const unsigned m = __ballot_sync(0xFFFFFFFFu, run + upto > at);
      if (m) {
        if (lane == __ffs(m) - 1) {
          a.tokens[r] = v + lane;
          if (a.probs) a.probs[r] = (float)((double)weight(x, top, f.inv_t) * (double)kUnit / (double)sum);
        }
        break;
      }
      run += __shfl_sync(0xFFFFFFFFu, upto, 31);
    }
  }
}

}  // namespace

cudaError_t launch_sample(const SampleArgs& a, retrace_dtype dtype, cudaStream_t stream) {
  const int rows = a.B * a.R;
  if (dtype == RETRACE_BF16)
    sample_kernel<__nv_bfloat16><<<rows, kThreads, 0, stream>>>(a);
  else
    sample_kernel<float><<<rows, kThreads, 0, stream>>>(a);
  return cudaGetLastError();
}

}  // namespace retrace
