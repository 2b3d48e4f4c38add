// Sampling a token from each logits row with temperature, top-k, top-p and min-p.
//
// With x the row's logits, m their maximum and T the temperature, token v weighs
// w_v = round(2^31 exp((x_v - m) / T)), a whole number, so that sums of weights do not
// depend on their order.  In the order of descending logits (the lower index first
// among equal ones) each filter keeps a prefix: top-k the first k tokens, top-p those
// before which the mass is below p times the mass that top-k keeps, min-p those of
// weight at least min_p times the first one's.  The token is then the first one in
// index order at which the running sum of the kept weights exceeds floor(u W).
//
// sample_cluster_kernel: a row lies in the registers of a cluster of CTAs (read once,
// in 16-byte vectors), so that every pass over it is arithmetic.  Sorting it would
// cost far more than reading it, and so would a histogram of every token in shared
// memory (its atomics).  Instead a sample of the row gives a logit that about enough
// tokens reach; these few are collected and sorted, and where they hold all that the
// filters keep, which is the rule with top-k, or with top-p over a peaked
// distribution, the rest is done among them.  Otherwise the place where a count or a
// mass is reached is found by two histograms, the second within a bin of the first,
// and an exact sum.  Whatever does not fit (thousands of tokens with one logit) goes to
// sample_row, which needs no memory for the row: radix selection over the 32-bit keys
// of the logits, also for rows that no cluster holds.
#include <math.h>

#include "../tc_pair.cuh"
#include "serve.h"

namespace retrace {
namespace {

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
template <int kThreads>
__device__ __forceinline__ u64 block_sum(u64 x, u64* s) {
  constexpr int kWarps = kThreads / 32;
  x = warp_sum(x);
  __syncthreads();
  if (threadIdx.x % 32 == 0) s[threadIdx.x / 32] = x;
  __syncthreads();
  return warp_sum(threadIdx.x % 32 < kWarps ? s[threadIdx.x % 32] : 0);
}

struct RowShared {  // of sample_row
  u64 hist[256];
  u64 part[32];
  float top[32];
  uint32_t digit;
  u64 above;
  int cut;
};

// The key t with M(> t) < target <= M(>= t), where M sums `metric` over the row's
// tokens; *above = M(> t).  1 <= target <= the whole sum.
template <typename T, int kThreads, typename Metric>
__device__ uint32_t select_key(const T* row, int V, u64 target, Metric metric, RowShared& sm, u64* above) {
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

// Row r by one CTA, from global memory.
template <typename T, int kThreads>
__device__ void sample_row(const SampleArgs& a, int r, RowShared& sm) {
  constexpr int kWarps = kThreads / 32;
  const int b = r / a.R, tid = threadIdx.x, lane = tid % 32, warp = tid / 32, V = a.V;
  const T* row = static_cast<const T*>(a.logits) + b * a.batch_stride + (r % a.R) * a.row_stride;
  const Filter f = row_filter(a, b);

  float top = -INFINITY;
  for (int v = tid; v < V; v += kThreads) top = fmaxf(top, logit(row, v));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
  if (lane == 0) sm.top[warp] = top;
  __syncthreads();
  top = lane < kWarps ? sm.top[lane] : -INFINITY;
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
    t = select_key<T, kThreads>(row, V, (u64)f.top_k, [](float) { return (u64)1; }, sm, &above);
    ties = f.top_k - above;
    u64 sum = 0;
    for (int v = tid; v < V; v += kThreads) {
      const float x = logit(row, v);
      if (ordered_bits(x) > t) sum += mass(x);
    }
    total = block_sum<kThreads>(sum, sm.part) + ties * mass(key_value((u64)t << 32));
  } else {
    u64 sum = 0;
    for (int v = tid; v < V; v += kThreads) sum += mass(logit(row, v));
    total = block_sum<kThreads>(sum, sm.part);
  }
  if (f.top_p < 1.f) {
    const double want = ceil((double)f.top_p * (double)total);
    const u64 target = want < 1.0 ? 1ull : (u64)want;
    u64 above;
    t = select_key<T, kThreads>(row, V, target, mass, sm, &above);
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


constexpr int kRowThreads = 1024;
template <typename T>
__global__ void __launch_bounds__(kRowThreads) sample_row_kernel(SampleArgs a) {
  __shared__ RowShared sm;
  sample_row<T, kRowThreads>(a, blockIdx.x, sm);
}

// ---- a row in the registers of a cluster ---------------------------------------
constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kList = 4096;       // collected tokens
constexpr int kBins = 256;        // of the first histogram, and of the sample's
constexpr int kFineBins = 1024;   // of the second
constexpr float kBinsPerNat = 11.5f;  // so that a token past the last bin (22.26 nats) weighs 0
constexpr int kListTopK = 1024;   // largest top_k for which the list is tried
constexpr int kListTopP = 400;    // tokens that the list aims at without top_k
constexpr int kMaxCluster = 8;

struct ClusterShared {
  union {
    struct {
      u64 list[kList];
      union {
        float mass[kFineBins];
        uint32_t count[kFineBins];
      };
    };
    RowShared row;
  };
  u64 seg[16 * kWarps + 2];  // kept mass by vector number and warp, before and after them
  u64 part[kWarps];
  float wtop[kWarps];
  // written by this CTA, read by the others of the cluster
  float top;
  int first;       // index of its first maximum
  int listed;      // tokens in its list
  u64 sum;         // exact sums of a pass
  // results that a CTA works out for itself
  int bin[2];
  u64 before;
  // written by CTA 0, read by all
  u64 key;         // the last kept token, as an argmax key
  int state;
  int pick;
};

// States of a row after its list: done, or the general way.
enum : int { kDone = 0, kGeneral = 1, kSlow = 2 };

template <typename T, int NV>
struct Row {
  static constexpr int E = 16 / sizeof(T);
  uint4 x[NV];  // this thread's vectors, rank * NV * kThreads + i * kThreads + tid
  float edge;   // and an element before or after the row's vectors
  int edge_at;  // its index, past the row where there is none
  int head;     // elements before the vectors
  int v0;       // index of the first element of vector 0 of this thread
  int V;
  float top, inv_t, ys;

  __device__ __forceinline__ float value(const uint4& q, int e) const {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
    if constexpr (E == 8) return e & 1 ? bf16_hi(w[e >> 1]) : bf16_lo(w[e >> 1]);
    return __uint_as_float(w[e & 3]);
  }
  // f(logit, index) for every element of this thread; past the row: -inf, an index >= V.
  template <typename F>
  __device__ __forceinline__ void each(F f) const {
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < E; ++e) f(value(x[i], e), v0 + i * kThreads * E + e);
    f(edge, edge_at);
  }
  // How far below the maximum, in bins; 256 or more: of no weight.
  __device__ __forceinline__ float depth(float v) const { return v == top ? 0.f : (top - v) * ys; }
  __device__ __forceinline__ uint32_t mass(float v) const { return whole_weight(weight(v, top, inv_t)); }
};

__device__ __forceinline__ float4 no_nan(float4 v) {
  v.x = v.x == v.x ? v.x : -INFINITY;
  v.y = v.y == v.y ? v.y : -INFINITY;
  v.z = v.z == v.z ? v.z : -INFINITY;
  v.w = v.w == v.w ? v.w : -INFINITY;
  return v;
}
// Two bf16 values with NaN replaced by -inf.
__device__ __forceinline__ uint32_t no_nan2(uint32_t w) {
  const uint32_t lo = (w & 0x7FFFu) > 0x7F80u ? 0xFF80u : w & 0xFFFFu;
  const uint32_t hi = (w & 0x7FFF0000u) > 0x7F800000u ? 0xFF800000u : w & 0xFFFF0000u;
  return lo | hi;
}

// Sorts the first `n` of the list (n at most kList) in descending order.
__device__ void sort_list(u64* list, int n) {
  int size = 1;
  while (size < n) size <<= 1;
  for (int i = n + threadIdx.x; i < size; i += kThreads) list[i] = 0;
  __syncthreads();
  for (int k = 2; k <= size; k <<= 1)
    for (int j = k >> 1; j > 0; j >>= 1) {
      for (int t = threadIdx.x; t < size / 2; t += kThreads) {
        const int i = 2 * t - (t & (j - 1)), o = i + j;
        const u64 a = list[i], b = list[o];
        if ((a < b) == ((i & k) == 0)) {
          list[i] = b;
          list[o] = a;
        }
      }
      __syncthreads();
    }
}

// Exclusive prefix of x over the block; *total the whole sum.
__device__ u64 block_scan(u64 x, u64* part, u64* total) {
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  u64 upto = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const u64 y = __shfl_up_sync(0xFFFFFFFFu, upto, o);
    if (lane >= o) upto += y;
  }
  __syncthreads();
  if (lane == 31) part[warp] = upto;
  __syncthreads();
  u64 before = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) before += part[w];
    sum += part[w];
  }
  *total = sum;
  return before + upto - x;
}

// The random number's place among `sum`.
__device__ __forceinline__ u64 place_of(float u0, u64 sum) {
  const float u = u0 > 0.f ? u0 : 0.f;
  const u64 at = (u64)floor((double)u * (double)sum);
  return u >= 1.f || at >= sum ? sum - 1 : at;
}
__device__ __forceinline__ u64 top_p_target(float p, u64 total) {
  const double want = ceil((double)p * (double)total);
  return want < 1.0 ? 1ull : (u64)want;
}

// CTA 0, with the sorted list of the row's first n tokens: what the filters keep, and the
// token.  `total` is the row's mass (top_k off); `all`: every token of any weight is in
// the list.  False where the list does not hold all that is kept.
__device__ __noinline__ bool finish_list(const SampleArgs& a, int r, const Filter& f, ClusterShared& sm, float top, int n,
                                         u64 total, bool all) {
  const int tid = threadIdx.x;
  constexpr int kEach = kList / kThreads;
  if (f.top_k < a.V && f.top_k > n && !all) return false;
  const int k = min(f.top_k, n);
  // thread t: entries [t per, (t + 1) per)
  const int per = (n + kThreads - 1) / kThreads;
  uint32_t w[kEach];
  u64 mine = 0;
  int heavy = 0;  // entries that min-p keeps
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int at = tid * per + i;
    w[i] = 0;
    if (i < per && at < k) {
      const float x = key_value(sm.list[at]), e = weight(x, top, f.inv_t);
      w[i] = whole_weight(e);
      heavy += x == top || !(e < f.min_p);
      mine += w[i];
    }
  }
  u64 listed;
  const u64 before = block_scan(mine, sm.part, &listed);
  if (f.top_k < a.V || all) total = listed;
  u64 target = ~0ull;
  if (f.top_p < 1.f) {
    target = top_p_target(f.top_p, total);
    if (target > listed) return false;
  }
  // kept: the first ones, as many as top-p and min-p both keep
  int kept = 0;
  u64 upto = before;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    if (i < per && tid * per + i < k) kept += upto < target;
    upto += w[i];
  }
  u64 all_kept, all_heavy;
  block_scan((u64)kept, sm.part, &all_kept);
  block_scan((u64)heavy, sm.part, &all_heavy);
  const int K = (int)(all_kept < all_heavy ? all_kept : all_heavy);
  __syncthreads();
  // in index order: (index, entry) ascending is ~(...) descending
  u64 sum = 0;
#pragma unroll
  for (int i = 0; i < kEach; ++i)
    if (i < per && tid * per + i < K) sum += w[i];
  block_scan(sum, sm.part, &sum);
  const u64 at = place_of(a.uniforms[r], sum);
  if (K == 1) {
    if (tid == 0) {
      a.tokens[r] = (int)key_index(sm.list[0]);
      if (a.probs) a.probs[r] = 1.f;
    }
    return true;
  }
  // weights with their order: the low half of a key is ~index, so that is sorted on
  u64 key[kEach];
#pragma unroll
  for (int i = 0; i < kEach; ++i)
    if (i < per && tid * per + i < K) key[i] = sm.list[tid * per + i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kEach; ++i)
    if (i < per && tid * per + i < K) sm.list[tid * per + i] = key[i] << 32 | key[i] >> 32;
  __syncthreads();
  sort_list(sm.list, K);
  const int each = (K + kThreads - 1) / kThreads;
  mine = 0;
  for (int i = 0; i < each; ++i) {
    const int e = tid * each + i;
    if (e < K) mine += whole_weight(weight(key_value(sm.list[e] << 32), top, f.inv_t));
  }
  u64 unused, run = block_scan(mine, sm.part, &unused);
  if (run <= at && at < run + mine) {
    for (int i = 0; i < each; ++i) {
      const u64 q = sm.list[tid * each + i];
      const float e = weight(key_value(q << 32), top, f.inv_t);
      run += whole_weight(e);
      if (run > at) {
        a.tokens[r] = (int)(0xFFFFFFFFu - (uint32_t)(q >> 32));
        if (a.probs) a.probs[r] = (float)((double)e * (double)kUnit / (double)sum);
        break;
      }
    }
  }
  return true;
}

template <typename T, int NV>
__global__ void __launch_bounds__(kThreads, 2) sample_cluster_kernel(SampleArgs a, int C) {
  extern __shared__ __align__(16) unsigned char raw[];
  ClusterShared& sm = *reinterpret_cast<ClusterShared*>(raw);
  constexpr int E = Row<T, NV>::E;
  const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32, V = a.V;
  const int rank = C > 1 ? (int)cluster_rank() : 0, r = blockIdx.x / C, b = r / a.R;
  auto sync = [&]() {
    if (C > 1)
      cluster_sync_all();
    else
      __syncthreads();
  };
  auto remote = [&](const void* p, int cta) { return map_rank(smem_u32(p), (uint32_t)cta); };

  pdl_wait();
  // ---- the row ----
  Row<T, NV> row;
  row.V = V;
  {
    const T* p = static_cast<const T*>(a.logits) + b * a.batch_stride + (r % a.R) * a.row_stride;
    const int head = min(V, (int)((16u - ((uintptr_t)p & 15u)) % 16u / sizeof(T)));
    const int vecs = (V - head) / E, tail = V - head - vecs * E;
    const uint4* q = reinterpret_cast<const uint4*>(p + head);
    const int first = rank * NV * kThreads + tid;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const uint32_t none = E == 8 ? 0xFF80FF80u : 0xFF800000u;  // -inf
      row.x[i] = first + i * kThreads < vecs ? __ldcs(q + first + i * kThreads) : make_uint4(none, none, none, none);
    }
    row.head = head;
    row.v0 = head + first * E;
    row.edge = -INFINITY;
    row.edge_at = 0x7FFFFFFF;
    if (rank == 0 && tid < head + tail) {
      row.edge_at = tid < head ? tid : head + vecs * E + tid - head;
      row.edge = logit(p, row.edge_at);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if constexpr (E == 8)
        row.x[i] = make_uint4(no_nan2(row.x[i].x), no_nan2(row.x[i].y), no_nan2(row.x[i].z), no_nan2(row.x[i].w));
      else
        *reinterpret_cast<float4*>(&row.x[i]) = no_nan(*reinterpret_cast<const float4*>(&row.x[i]));
    }
  }
  const Filter f = row_filter(a, b);

  // ---- the maximum ----
  {
    float top = -INFINITY;
    row.each([&](float v, int) { top = fmaxf(top, v); });
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
    if (lane == 0) sm.wtop[warp] = top;
    for (int i = tid; i < kFineBins; i += kThreads) sm.mass[i] = 0.f;
    if (tid == 0) sm.listed = 0;
    __syncthreads();
    if (warp == 0) {
      top = lane < kWarps ? sm.wtop[lane] : -INFINITY;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
      if (lane == 0) sm.top = top;
    }
    sync();
    top = -INFINITY;
    for (int c = 0; c < C; ++c) top = fmaxf(top, C > 1 ? ld_cluster_f1(remote(&sm.top, c)) : sm.top);
    row.top = top;
  }
  row.inv_t = f.inv_t;
  row.ys = f.inv_t * kBinsPerNat;
  if (row.top == -INFINITY || f.top_k == 1) {
    // no token, or the first maximum
    int at = 0x7FFFFFFF;
    if (row.top != -INFINITY) row.each([&](float v, int i) { at = v == row.top ? min(at, i) : at; });
    at = __reduce_min_sync(0xFFFFFFFFu, at);
    if (lane == 0) sm.part[warp] = (u64)at;
    __syncthreads();
    if (tid == 0) {
      for (int w = 0; w < kWarps; ++w) at = min(at, (int)sm.part[w]);
      sm.first = at;
    }
    sync();
    if (rank == 0 && tid == 0) {
      for (int c = 0; c < C; ++c) at = min(at, C > 1 ? ld_cluster_s32(remote(&sm.first, c)) : sm.first);
      a.tokens[r] = row.top == -INFINITY ? -1 : at;
      if (a.probs) a.probs[r] = row.top == -INFINITY ? 0.f : 1.f;
    }
    sync();  // CTA 0 has read the others
    return;
  }

  // Sum over the cluster of a value per thread, to every thread.
  auto cluster_sum = [&](u64 x) {
    const u64 mine = block_sum<kThreads>(x, sm.part);
    if (C == 1) return mine;
    if (tid == 0) sm.sum = mine;
    sync();
    u64 all = 0;
    for (int c = 0; c < C; ++c) all += ld_cluster_u64(remote(&sm.sum, c));
    sync();  // `sum` is read before it is written again
    return all;
  };
  // Two bins of a histogram over the cluster (in sm.mass, or sm.count): the first at
  // which the running sum reaches `lo`, and the first at which it reaches `hi` (the last bin
  // where none does); the histogram is cleared.
  auto find_bins = [&](int bins, bool counts, double lo, double hi) {
    sync();
    // thread t sums bins 2t and 2t + 1 over the CTAs
    double x[2] = {0.0, 0.0};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int at = 2 * tid + i;
      if (at < bins)
        for (int c = 0; c < C; ++c) {
          if (counts)
            x[i] += (double)(C > 1 ? (uint32_t)ld_cluster_s32(remote(&sm.count[at], c)) : sm.count[at]);
          else
            x[i] += (double)(C > 1 ? ld_cluster_f1(remote(&sm.mass[at], c)) : sm.mass[at]);
        }
    }
    double upto = x[0] + x[1];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const double y = __shfl_up_sync(0xFFFFFFFFu, upto, o);
      if (lane >= o) upto += y;
    }
    __syncthreads();
    if (lane == 31) sm.part[warp] = (u64)__double_as_longlong(upto);
    if (tid < 2) sm.bin[tid] = bins - 1;
    __syncthreads();
    double before = upto - x[0] - x[1];
    for (int w = 0; w < warp; ++w) before += __longlong_as_double((long long)sm.part[w]);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int at = 2 * tid + i;
      if (at < bins) {
        if (before < lo && before + x[i] >= lo) atomicMin(&sm.bin[0], at);  // lo > 0
        if (before < hi && before + x[i] >= hi) atomicMin(&sm.bin[1], at);
      }
      before += x[i];
    }
    sync();  // every CTA has read the histograms
    for (int i = tid; i < kFineBins; i += kThreads) sm.mass[i] = 0.f;
    const int2 found = make_int2(sm.bin[0], sm.bin[1]);
    __syncthreads();
    return found;
  };
  // Collects the tokens for which take(logit, index) holds.
  auto collect = [&](auto take) {
    row.each([&](float v, int i) {
      if (take(v, i)) {
        const int at = atomicAdd(&sm.listed, 1);
        if (at < kList) sm.list[at] = make_key(v, (uint32_t)i);
      }
    });
  };
  // CTA 0: the others' lists after its own; -1 where they are too long.  All CTAs call it.
  auto gather_lists = [&]() {
    sync();
    int n = sm.listed;
    if (rank == 0 && C > 1) {
      int all = 0;
      for (int c = 0; c < C; ++c) all += ld_cluster_s32(remote(&sm.listed, c));
      if (all <= kList) {
        for (int c = 1; c < C; ++c) {
          const int m = ld_cluster_s32(remote(&sm.listed, c));
          for (int i = tid; i < m; i += kThreads) sm.list[n + i] = ld_cluster_u64(remote(&sm.list[i], c));
          n += m;
        }
      } else {
        n = kList + 1;
      }
    }
    __syncthreads();
    return n <= kList ? n : -1;
  };
  // The last token of the prefix in which `metric` reaches `target`, as a key (0 where it was
  // not found this way).
  auto find_key = [&](u64 target, bool counts) -> u64 {
    auto metric = [&](float v) -> u64 { return counts ? 1u : row.mass(v); };
    const double slack = counts ? 0.0 : 1e-3 * (double)target;  // the masses in a histogram are fp32
    row.each([&](float v, int i) {
      const float y = row.depth(v);
      if (i < V && y < (float)kBins) {
        if (counts)
          atomicAdd(&sm.count[(int)y], 1u);
        else
          atomicAdd(&sm.mass[(int)y], (float)row.mass(v));
      }
    });
    const int2 coarse = find_bins(kBins, counts, (double)target - slack, (double)target + slack);
    // a fine bin is 2^-shift of a coarse one, whole coarse bins together at most kFineBins
    int shift = 10;
    while (((coarse.y - coarse.x + 1) << shift) > kFineBins && shift > 0) --shift;
    const float lo = (float)coarse.x, hi = (float)(coarse.y + 1), per = (float)(1 << shift);
    u64 above = 0;
    row.each([&](float v, int i) {
      const float y = row.depth(v);
      if (i < V && y < hi) {
        if (y < lo) {
          above += metric(v);
        } else if (counts) {
          atomicAdd(&sm.count[min(kFineBins - 1, (int)((y - lo) * per))], 1u);
        } else {
          atomicAdd(&sm.mass[min(kFineBins - 1, (int)((y - lo) * per))], (float)row.mass(v));
        }
      }
    });
    above = cluster_sum(above);
    if (above >= target) return 0;
    const double left = (double)(target - above);
    const int2 fine = find_bins(kFineBins, counts, fmax(left - slack, 0.5), left + slack);
    auto fine_bin = [&](float v) {
      const float y = row.depth(v);
      return y < lo ? -1 : y < hi ? min(kFineBins - 1, (int)((y - lo) * per)) : kFineBins;
    };
    if (tid == 0) sm.listed = 0;
    __syncthreads();
    above = 0;
    row.each([&](float v, int i) {
      const int bin = i < V ? fine_bin(v) : kFineBins;
      if (bin < fine.x) above += metric(v);
    });
    collect([&](float v, int i) {
      const int bin = i < V ? fine_bin(v) : kFineBins;
      return bin >= fine.x && bin <= fine.y;
    });
    above = cluster_sum(above);
    const int n = gather_lists();
    if (rank == 0) {
      if (tid == 0) sm.key = 0;
      if (n > 0 && above < target) {
        sort_list(sm.list, n);
        const int per_thread = (n + kThreads - 1) / kThreads;
        u64 mine = 0;
        for (int i = 0; i < per_thread; ++i) {
          const int e = tid * per_thread + i;
          if (e < n) mine += metric(key_value(sm.list[e]));
        }
        u64 all, run = above + block_scan(mine, sm.part, &all);
        if (run < target && run + mine >= target)
          for (int i = 0; i < per_thread; ++i) {
            run += metric(key_value(sm.list[tid * per_thread + i]));
            if (run >= target) {
              sm.key = sm.list[tid * per_thread + i];
              break;
            }
          }
      }
    }
    sync();
    const u64 key = C > 1 ? ld_cluster_u64(remote(&sm.key, 0)) : sm.key;
    sync();
    return key;
  };

  const bool by_k = f.top_k < V;
  u64 total = 0;  // the row's mass
  int state = kGeneral;
  if (!by_k && f.top_p < 1.f) {
    u64 mine = 0;
    row.each([&](float v, int) { mine += row.mass(v); });
    total = cluster_sum(mine);
  }
  if ((by_k && f.top_k <= kListTopK) || (!by_k && f.top_p < 1.f)) {
    // ---- the list ----
    // A quarter of the vectors, half their elements, are the sample.
    constexpr int kStep = NV >= 4 ? 4 : 1;
#pragma unroll
    for (int i = 0; i < NV; i += kStep)
#pragma unroll
      for (int e = 0; e < E; e += 2) {
        const float y = row.depth(row.value(row.x[i], e));
        if (y < (float)kBins) atomicAdd(&sm.count[(int)y], 1u);
      }
    const float share = (float)((NV + kStep - 1) / kStep) / (float)(2 * NV);
    const float want = (float)(by_k ? f.top_k : kListTopP) * share;
    const double reach = (double)(want + 4.f * sqrtf(want) + 4.f);
    const int bin = find_bins(kBins, true, reach, reach).x;
    collect([&](float v, int) { return row.depth(v) < (float)(bin + 1); });
    const int n = gather_lists();
    if (rank == 0) {
      int st = kGeneral;
      if (n > 0) {
        sort_list(sm.list, n);
        if (finish_list(a, r, f, sm, row.top, n, total, bin == kBins - 1)) st = kDone;
      }
      __syncthreads();
      if (tid == 0) sm.state = st;
    }
    sync();
    state = C > 1 ? ld_cluster_s32(remote(&sm.state, 0)) : sm.state;
    sync();
    if (state == kDone) return;
  }

  // ---- the general way: the last kept token, then the draw over the row ----
  u64 last = 0;  // keys from this one on are kept
  if (by_k) {
    u64 heavy = 0;  // tokens of any weight; no other one is drawn
    row.each([&](float v, int) { heavy += row.depth(v) < (float)kBins; });
    if (cluster_sum(heavy) > (u64)f.top_k) {
      last = find_key((u64)f.top_k, true);
      if (last == 0) state = kSlow;
    }
    if (state != kSlow && f.top_p < 1.f) {
      u64 mine = 0;
      row.each([&](float v, int i) {
        if (make_key(v, (uint32_t)i) >= last) mine += row.mass(v);
      });
      total = cluster_sum(mine);
    }
  }
  if (state != kSlow && f.top_p < 1.f) {
    const u64 key = find_key(top_p_target(f.top_p, total), false);
    if (key == 0)
      state = kSlow;
    else
      last = key;
  }
  if (state == kSlow) {
    sync();  // nobody reads CTA 0's lists any more
    if (rank == 0) sample_row<T, kThreads>(a, r, sm.row);
    return;
  }
  auto kept = [&](float v, int i) -> u64 {
    if (i >= V || make_key(v, (uint32_t)i) < last) return 0;
    const float e = weight(v, row.top, f.inv_t);
    return v == row.top || !(e < f.min_p) ? whole_weight(e) : 0;
  };
  // In index order: the elements before the vectors, vectors i = 0, 1, ... of warps 0, 1,
  // ... of the CTAs in turn, the elements after them.
  u64 mine = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    u64 x = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) x += kept(row.value(row.x[i], e), row.v0 + i * kThreads * E + e);
    x = warp_sum(x);
    if (lane == 0) sm.seg[1 + i * kWarps + warp] = x;
    mine += x;
  }
  if (warp == 0) {
    const u64 x = kept(row.edge, row.edge_at);
    const bool early = row.edge_at < row.head;
    const u64 head = warp_sum(early ? x : 0), tail = warp_sum(early ? 0 : x);
    if (lane == 0) {
      sm.seg[0] = head;
      sm.seg[1 + NV * kWarps] = tail;
    }
    mine += head;  // the tail follows the last CTA
  }
  const u64 whole = block_sum<kThreads>(lane == 0 ? mine : 0, sm.part);
  if (tid == 0) sm.sum = whole;
  sync();
  u64 before = 0, sum = 0;
  for (int c = 0; c < C; ++c) {
    if (c == rank) before = sum;
    sum += C > 1 ? ld_cluster_u64(remote(&sm.sum, c)) : sm.sum;
  }
  const u64 body = sum, tail = C > 1 ? ld_cluster_u64(remote(&sm.seg[1 + NV * kWarps], 0)) : sm.seg[1 + NV * kWarps];
  sum += tail;
  const u64 at = place_of(a.uniforms[r], sum);
  auto take = [&](float v, int i) {
    a.tokens[r] = i;
    if (a.probs) a.probs[r] = (float)((double)weight(v, row.top, f.inv_t) * (double)kUnit / (double)sum);
  };
  // A warp whose segment holds the place looks through its lanes.
  auto look = [&](u64 x, u64 run, auto each_of_lane) {
    u64 upto = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const u64 y = __shfl_up_sync(0xFFFFFFFFu, upto, o);
      if (lane >= o) upto += y;
    }
    if (run + upto > at && run + upto - x <= at) each_of_lane(run + upto - x);
  };
  if (rank == 0 && warp == 0) {
    const u64 x = kept(row.edge, row.edge_at);
    const bool early = row.edge_at < row.head;
    if (at < sm.seg[0]) look(early ? x : 0, 0, [&](u64) { take(row.edge, row.edge_at); });
    if (at >= body) look(early ? 0 : x, body, [&](u64) { take(row.edge, row.edge_at); });
  }
  // this CTA's segments
  u64 run = before + sm.seg[0];
  if (rank != 0) run = before;
  if (run <= at && at < before + whole) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      u64 start = run;
      for (int w = 0; w < warp; ++w) start += sm.seg[1 + i * kWarps + w];
      if (start <= at && at < start + sm.seg[1 + i * kWarps + warp]) {
        u64 x = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) x += kept(row.value(row.x[i], e), row.v0 + i * kThreads * E + e);
        look(x, start, [&](u64 s) {
          bool found = false;
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const float v = row.value(row.x[i], e);
            const int index = row.v0 + i * kThreads * E + e;
            s += kept(v, index);
            if (!found && s > at) {
              found = true;
              take(v, index);
            }
          }
        });
      }
      for (int w = 0; w < kWarps; ++w) run += sm.seg[1 + i * kWarps + w];
    }
  }
  sync();  // the others have read this CTA's sums
}

template <typename T, int NV>
cudaError_t launch_cluster_rows(const SampleArgs& a, int C, cudaStream_t stream) {
  auto kernel = sample_cluster_kernel<T, NV>;
  constexpr size_t smem = sizeof(ClusterShared);
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  return launch_dependent(kernel, dim3((unsigned)(a.B * a.R) * C), dim3(kThreads), smem, stream, (unsigned)C, a, C);
}

template <typename T>
cudaError_t launch_typed(const SampleArgs& a, cudaStream_t stream) {
  constexpr int E = 16 / sizeof(T);
  const int rows = a.B * a.R;
  DeviceInfo dev;
  cudaError_t e = device_info(&dev);
  if (e != cudaSuccess) return e;
  const long long vecs = (a.V + E - 1) / E;
  auto need = [&](int C) { return (int)((vecs + (long long)C * kThreads - 1) / ((long long)C * kThreads)); };
  // The fewest CTAs that hold a row; more of them while they are idle otherwise.
  int C = 1;
  while (C < kMaxCluster && need(C) > 10) C *= 2;
  if (need(C) > 10 || (long long)rows * kMaxCluster > (1ll << 31) - 1) {
    sample_row_kernel<T><<<rows, kRowThreads, 0, stream>>>(a);
    return cudaGetLastError();
  }
  while (C < kMaxCluster && need(C) > 1 && (long long)rows * C * 2 <= dev.sm_count) C *= 2;
  const int n = need(C);
  if (n <= 1) return launch_cluster_rows<T, 1>(a, C, stream);
  if (n <= 2) return launch_cluster_rows<T, 2>(a, C, stream);
  if (n <= 5) return launch_cluster_rows<T, 5>(a, C, stream);
  return launch_cluster_rows<T, 10>(a, C, stream);
}

}  // namespace

cudaError_t launch_sample(const SampleArgs& a, retrace_dtype dtype, cudaStream_t stream) {
  return dtype == RETRACE_BF16 ? launch_typed<__nv_bfloat16>(a, stream) : launch_typed<float>(a, stream);
}

}  // namespace retrace
