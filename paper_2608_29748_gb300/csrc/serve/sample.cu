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
// Sorting a row would cost far more than reading it, and so would a histogram of all of
// its tokens in shared memory (its atomics).  Instead a sample of the row gives a logit
// that about enough tokens reach; these few are collected and sorted, and where they
// hold all that the filters keep, which is the rule with top-k, or with top-p over a
// peaked distribution, the rest is done among them.  Otherwise the place where a count
// or a mass is reached is found by two histograms, the second within a bin of the first,
// and an exact sum.  Whatever does not fit (thousands of tokens with one logit) goes to
// sample_row: radix selection over the 32-bit keys of the logits.
//
// With many rows a CTA takes one and streams it (Stream), four of them to an SM.  Where a
// list suffices the row is read once.  Later passes read it again: 608 rows of 151936 in bf16 are
// 185 MB at a time, more than L2 holds, and 1024 of them under top-p 0.9 read 1.40 GB for 311 MB
// of rows, at a sixth of the memory's rate.  With few rows a cluster of up to eight CTAs holds
// one in registers (Held), so that later passes are arithmetic; of ten bf16 vectors to a thread, as
// 16 rows of 151936 have, some spill.
// 4096 rows of 151936 in bf16 with filters of their own: 288 us, 4.3 TB/s; 16 of them, top-k 20 and
// top-p: 14 us, all latency.  528 flat rows of 32003 in fp32, top-p 0.98: 136 us, seven
// passes of about 25 instructions and an exponential a logit.
// More than 4096 tokens with the deciding logit (sample_row): an atomic a token and digit, nearly all on
// one address; 151936 equal logits take 25 ms for top-k or top-p and 50 for both, a thousand such
// rows 53 and 103.
#include <math.h>

#include <type_traits>

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

// x n for a float x in [0, 1] and n <= 2^55 (2^24 weights of 2^31), rounded to 53 bits as their product in fp64
// is, in whole numbers (fp64 arithmetic is slow here): its floor, or its ceiling.
__device__ __forceinline__ u64 scaled(float x, u64 n, bool up) {
  const uint32_t bits = __float_as_uint(x);
  if (n == 0 || bits == 0) return 0;
  const int exponent = (int)(bits >> 23);
  const u64 m = (bits & 0x7FFFFFu) | (exponent ? 0x800000u : 0u);
  int drop = 150 - (exponent ? exponent : 1);  // x = m 2^-drop
  u64 hi = __umul64hi(m, n), lo = m * n;
  // to 53 bits, nearest, ties to even
  const int length = hi ? 128 - __clzll((long long)hi) : 64 - __clzll((long long)lo);
  if (length > 53) {
    const int cut = length - 53;  // at most 27
    const u64 rest = lo & ((1ull << cut) - 1), half = 1ull << (cut - 1);
    lo = lo >> cut | hi << (64 - cut);
    lo += rest > half || (rest == half && (lo & 1));
    drop -= cut;
  }
  if (drop <= 0) return lo << -drop;
  if (drop > 63) return up ? 1 : 0;
  return (lo >> drop) + (up && (lo & ((1ull << drop) - 1)) ? 1 : 0);
}
// The random number's place among `sum`.
__device__ __forceinline__ u64 place_of(float u, u64 sum) {
  if (!(u > 0.f)) return 0;
  const u64 at = u < 1.f ? scaled(u, sum, false) : sum;
  return at >= sum ? sum - 1 : at;
}
// The mass that top-p wants of `total`, p < 1.
__device__ __forceinline__ u64 top_p_target(float p, u64 total) {
  const u64 want = p > 0.f ? scaled(p, total, true) : 0;
  return want < 1 ? 1 : want;
}
// e of a weight among the sum of whole weights; the sum rounded to fp32, which moves the result by
// no more than its own rounding.
__device__ __forceinline__ float probability(float e, u64 sum) { return __fdiv_rn(e * kUnit, (float)sum); }

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
    const u64 target = top_p_target(f.top_p, total);
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
  const u64 at = place_of(a.uniforms[r], sum);
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
          if (a.probs) a.probs[r] = probability(weight(x, top, f.inv_t), sum);
        }
        break;
      }
      run += __shfl_sync(0xFFFFFFFFu, upto, 31);
    }
  }
}


// ---- rows as the kernel below reads them ----------------------------------------
constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kList = 4096;           // collected tokens
constexpr int kBins = 256;            // of the first histogram, and of the sample's
constexpr int kFineBins = 1024;       // of the second
constexpr float kBinsPerNat = 11.5f;  // so that a token past the last bin (22.26 nats) weighs 0
constexpr int kListTopK = 1024;       // largest top_k for which the list is tried
constexpr int kListTopP = 400;        // tokens that the list aims at without top_k
constexpr int kMaxCluster = 8;

template <typename T>
struct Vec {  // 16 bytes of a row
  static constexpr int E = 16 / sizeof(T);
  __device__ __forceinline__ static float value(const uint4& q, int e) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
    if constexpr (E == 8) return e & 1 ? bf16_hi(w[e >> 1]) : bf16_lo(w[e >> 1]);
    return __uint_as_float(w[e & 3]);
  }
  __device__ __forceinline__ static uint4 none() {
    const uint32_t w = E == 8 ? 0xFF80FF80u : 0xFF800000u;  // -inf
    return make_uint4(w, w, w, w);
  }
  // The largest of the 16 bytes' values; NaN where all of them are.
  __device__ __forceinline__ static float top(const uint4& q) {
    if constexpr (E == 8) {
      const __nv_bfloat162* v = reinterpret_cast<const __nv_bfloat162*>(&q);
      const __nv_bfloat162 m = __hmax2(__hmax2(v[0], v[1]), __hmax2(v[2], v[3]));
      return fmaxf(__low2float(m), __high2float(m));
    }
    return fmaxf(fmaxf(value(q, 0), value(q, 1)), fmaxf(value(q, 2), value(q, 3)));
  }
};

// What both forms of a row share: its vectors, and the elements before and after them.
template <typename T>
struct RowParts {
  static constexpr int E = Vec<T>::E;
  const T* p;
  const uint4* q;
  int V, head, vecs;
  float edge;   // this thread's element before or after the vectors
  int edge_at;  // its index; past the row where there is none
  float top, inv_t, ys;

  __device__ __forceinline__ void find(const SampleArgs& a, int r, bool edges) {
    p = static_cast<const T*>(a.logits) + (r / a.R) * a.batch_stride + (r % a.R) * a.row_stride;
    V = a.V;
    head = min(V, (int)((16u - ((uintptr_t)p & 15u)) % 16u / sizeof(T)));
    vecs = (V - head) / E;
    q = reinterpret_cast<const uint4*>(p + head);
    edge = -INFINITY;
    edge_at = 0x7FFFFFFF;
    const int t = threadIdx.x, tail = V - head - vecs * E;
    if (edges && t < head + tail) {
      edge_at = t < head ? t : head + vecs * E + t - head;
      edge = logit(p, edge_at);
    }
  }
  __device__ __forceinline__ int index(int vec) const { return head + vec * E; }
  // How far below the maximum, in bins; 256 or more, or NaN: of no weight.
  __device__ __forceinline__ float depth(float v) const { return v == top ? 0.f : (top - v) * ys; }
  __device__ __forceinline__ uint32_t mass(float v) const { return whole_weight(weight(v, top, inv_t)); }
};

// A row in the registers of a cluster: vector `(rank NV + i) kThreads + tid` is x[i].
template <typename T, int NV>
struct Held : RowParts<T> {
  static constexpr int kSegments = NV * kWarps;
  uint4 x[NV];
  int first;  // vector of x[0]

  __device__ __forceinline__ void load(const SampleArgs& a, int r, int rank) {
    this->find(a, r, rank == 0);
    first = rank * NV * kThreads + threadIdx.x;
#pragma unroll
    for (int i = 0; i < NV; ++i)
      x[i] = first + i * kThreads < this->vecs ? __ldcs(this->q + first + i * kThreads) : Vec<T>::none();
  }
  // f(vector, index of its first element); past the row: -inf.
  template <typename F>
  __device__ __forceinline__ void vectors(F f) const {
#pragma unroll
    for (int i = 0; i < NV; ++i) f(x[i], this->index(first + i * kThreads));
  }
  // Some vectors; the share of the row that they are.
  template <typename F>
  __device__ __forceinline__ float sample(F f) const {
#pragma unroll
    for (int i = 0; i < NV; i += kStep) f(x[i]);
    return (float)((NV + kStep - 1) / kStep) / (float)NV;
  }
  static constexpr int kStep = NV >= 5 ? 5 : 1;
  // The row in index order: segment s of warp w.  f(vector, index) of this thread's part.
  __device__ __forceinline__ int segments() const { return NV; }
  template <typename F>
  __device__ __forceinline__ void segment(int s, F f) const {
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (i == s) f(x[i], this->index(first + i * kThreads));
  }
};

// A row that a CTA streams.
template <typename T>
struct Stream : RowParts<T> {
  static constexpr int kSegments = kWarps;
  static constexpr int kRuns = 64;
  static constexpr int kAhead = 8;  // loads in flight per thread
  __device__ __forceinline__ void load(const SampleArgs& a, int r, int) { this->find(a, r, true); }
  template <typename F>
  __device__ __forceinline__ void vectors(F f) const {
    int v = threadIdx.x;
    for (; v + (kAhead - 1) * kThreads < this->vecs; v += kAhead * kThreads) {
      uint4 x[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) x[i] = __ldg(this->q + v + i * kThreads);
#pragma unroll
      for (int i = 0; i < kAhead; ++i) f(x[i], this->index(v + i * kThreads));
    }
    for (; v < this->vecs; v += kThreads) f(__ldg(this->q + v), this->index(v));
  }
  // 64 runs of 32 vectors, spread over the row.
  template <typename F>
  __device__ __forceinline__ float sample(F f) const {
    const int runs = this->vecs / 32, taken = runs < kRuns ? runs : kRuns;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
#pragma unroll 4
    for (int j = warp; j < taken; j += kWarps) f(__ldg(this->q + (j * runs / taken) * 32 + lane));
    return (float)taken * 32.f / (float)(this->vecs > 0 ? this->vecs : 1);
  }
  // Warp w has the vectors [w per, (w + 1) per), 32 at a time.
  __device__ __forceinline__ int per() const { return ((this->vecs + kWarps - 1) / kWarps + 31) / 32 * 32; }
  __device__ __forceinline__ int segments() const { return 1; }
  template <typename F>
  __device__ __forceinline__ void run(F f) const {  // f(vector or none, index), whole warps
    const int w = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int end = min(this->vecs, (w + 1) * per());
    for (int v = w * per() + lane; v - lane < end; v += 4 * 32) {
      uint4 x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = v + i * 32 < end ? __ldg(this->q + v + i * 32) : Vec<T>::none();
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (!f(x[i], this->index(v + i * 32))) return;
    }
  }
};

struct ClusterShared {
  union {
    struct {
      u64 list[kList];
      u64 spare[kList / 4];  // of sort_list
      uint32_t count[kFineBins];
    };
    RowShared row;
  };
  u64 seg[10 * kWarps + 2];  // kept mass of the segments, of what is before and after the vectors
  u64 part[kWarps];
  float wtop[kWarps];
  int bin[2];
  u64 before, upto;
  int entries;  // of the list that are kept
  // written by this CTA, read by the others of the cluster
  float top;
  int listed;  // tokens in its list
  u64 sum[2];  // exact sums of a pass, in turn
  // written by CTA 0, read by all
  u64 key;     // the last kept token
  int state;
};
enum : int { kDone = 0, kGeneral = 1, kSlow = 2 };  // what is left to do for a row after its list

// Exclusive prefix of x over the block; *total the whole sum.
__device__ __forceinline__ u64 block_scan(u64 x, u64* part, u64* total) {
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
    const u64 y = part[w];
    if (w < warp) before += y;
    sum += y;
  }
  *total = sum;
  return before + upto - x;
}

// Sorts the first n (at most kList) of the list in descending order, in place.  Up to a
// quarter of the list: into bins by the depth of a logit below the maximum, then by counting
// the larger ones within a bin, few where the logits differ.  More: bitonic.
__device__ __noinline__ void sort_list(ClusterShared& sm, int n, float top, float scale) {
  const int tid = threadIdx.x;
  u64* list = sm.list;
  if (n <= kList / 4) {
    constexpr int kEach = kList / 4 / kThreads;
    auto bin_of = [&](u64 key) {
      const float v = key_value(key), y = v == top ? 0.f : (top - v) * scale;
      return y < (float)kFineBins ? max(0, (int)y) : kFineBins - 1;
    };
    // sm.count is zero here
    u64 key[kEach];
    int place[kEach], bin[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int e = tid + i * kThreads;
      if (e < n) {
        key[i] = list[e];
        bin[i] = bin_of(key[i]);
        place[i] = (int)atomicAdd(&sm.count[bin[i]], 1u);
      }
    }
    __syncthreads();
    constexpr int kBinsEach = kFineBins / kThreads;
    uint32_t size[kBinsEach], sum = 0;
#pragma unroll
    for (int i = 0; i < kBinsEach; ++i) sum += size[i] = sm.count[kBinsEach * tid + i];
    u64 all;
    uint32_t start = (uint32_t)block_scan(sum, sm.part, &all);
    // start of a bin in the low half, its size in the high half
#pragma unroll
    for (int i = 0; i < kBinsEach; ++i) {
      sm.count[kBinsEach * tid + i] = start | size[i] << 16;
      start += size[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      if (tid + i * kThreads < n) sm.spare[(sm.count[bin[i]] & 0xFFFFu) + place[i]] = key[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      if (tid + i * kThreads < n) {
        const int from = (int)(sm.count[bin[i]] & 0xFFFFu), size = (int)(sm.count[bin[i]] >> 16);
        int larger = 0;
        for (int e = from; e < from + size; ++e) larger += sm.spare[e] > key[i];
        list[from + larger] = key[i];
      }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kBinsEach; ++i) sm.count[kBinsEach * tid + i] = 0;
    __syncthreads();
    return;
  }
  int size = 1;
  while (size < n) size <<= 1;
  for (int i = n + tid; i < size; i += kThreads) list[i] = 0;
  __syncthreads();
  for (int k = 2; k <= size; k <<= 1)
    for (int j = k >> 1; j > 0; j >>= 1) {
      for (int t = tid; t < size / 2; t += kThreads) {
        const int i = 2 * t - (t & (j - 1)), o = i + j;
        const u64 x = list[i], y = list[o];
        if ((x < y) == ((i & k) == 0)) {
          list[i] = y;
          list[o] = x;
        }
      }
      __syncthreads();
    }
}

__device__ __forceinline__ void write_token(const SampleArgs& a, int r, int token, float e, u64 sum) {
  a.tokens[r] = token;
  if (a.probs) a.probs[r] = probability(e, sum);
}

// One CTA, with the sorted list of the row's first n tokens: what the filters keep, and the
// token.  `total` is the row's mass (read with top-p and without top-k); `all`: every token
// of any weight is in the list.  False where the list does not hold all that is kept.
__device__ __noinline__ bool finish_list(const SampleArgs& a, int r, const Filter& f, ClusterShared& sm, float top, int n,
                                         u64 total, bool all) {
  const int tid = threadIdx.x;
  if (f.top_k < a.V && f.top_k > n && !all) return false;
  if (f.top_k >= a.V && f.top_p >= 1.f && !all) return false;
  const int k = min(f.top_k, n), per = (k + kThreads - 1) / kThreads;  // thread t: entries [t per, (t + 1) per)
  if (tid == 0) sm.entries = k;
  u64 mine = 0;
  for (int i = 0; i < per; ++i)
    if (tid * per + i < k) mine += whole_weight(weight(key_value(sm.list[tid * per + i]), top, f.inv_t));
  u64 listed;
  const u64 before = block_scan(mine, sm.part, &listed);
  if (f.top_k < a.V || all) total = listed;
  u64 target = ~0ull;
  if (f.top_p < 1.f) target = top_p_target(f.top_p, total);
  if (f.top_p < 1.f && target > listed) return false;
  // the first entry that a filter does not keep ends the list
  u64 run = before;
  for (int i = 0; i < per; ++i) {
    const int e = tid * per + i;
    if (e >= k) break;
    const float x = key_value(sm.list[e]), w = weight(x, top, f.inv_t);
    if (run >= target || (x != top && w < f.min_p)) {
      atomicMin(&sm.entries, e);
      break;
    }
    run += whole_weight(w);
  }
  __syncthreads();
  const int K = sm.entries;
  // the kept mass: what is before entry K
  run = before;
  for (int i = 0; i < per; ++i) {
    const int e = tid * per + i;
    if (e >= k) break;
    run += whole_weight(weight(key_value(sm.list[e]), top, f.inv_t));
    if (e == K - 1) sm.key = run;
  }
  __syncthreads();
  const u64 sum = sm.key, at = place_of(a.uniforms[r], sum);
  if (K <= kThreads) {
    // an entry's place in index order: the mass of the entries of lower indices
    if (tid < K) sm.spare[tid] = (u64)whole_weight(weight(key_value(sm.list[tid]), top, f.inv_t));
    __syncthreads();
    if (tid < K) {
      const uint32_t index = key_index(sm.list[tid]);
      u64 below = 0;
      for (int e = 0; e < K; ++e)
        if (key_index(sm.list[e]) < index) below += sm.spare[e];
      if (below <= at && at < below + sm.spare[tid])
        write_token(a, r, (int)index, weight(key_value(sm.list[tid]), top, f.inv_t), sum);
    }
    return true;
  }
  // many: sorted by ~index, the low half of a key, its halves exchanged
  for (int e = tid; e < K; e += kThreads) sm.list[e] = sm.list[e] << 32 | sm.list[e] >> 32;
  __syncthreads();
  int size = 1;
  while (size < K) size <<= 1;
  for (int e = K + tid; e < size; e += kThreads) sm.list[e] = 0;
  __syncthreads();
  for (int kk = 2; kk <= size; kk <<= 1)
    for (int j = kk >> 1; j > 0; j >>= 1) {
      for (int t = tid; t < size / 2; t += kThreads) {
        const int i = 2 * t - (t & (j - 1)), o = i + j;
        const u64 x = sm.list[i], y = sm.list[o];
        if ((x < y) == ((i & kk) == 0)) {
          sm.list[i] = y;
          sm.list[o] = x;
        }
      }
      __syncthreads();
    }
  const int each = (K + kThreads - 1) / kThreads;
  mine = 0;
  for (int i = 0; i < each; ++i)
    if (tid * each + i < K) mine += whole_weight(weight(key_value(sm.list[tid * each + i] << 32), top, f.inv_t));
  u64 unused;
  run = block_scan(mine, sm.part, &unused);
  if (run <= at && at < run + mine)
    for (int i = 0; i < each; ++i) {
      const u64 x = sm.list[tid * each + i];
      const float w = weight(key_value(x << 32), top, f.inv_t);
      run += whole_weight(w);
      if (run > at) {
        write_token(a, r, (int)(0xFFFFFFFFu - (uint32_t)(x >> 32)), w, sum);
        break;
      }
    }
  return true;
}

// One row by one CTA (Stream, C = 1) or a cluster of C (Held).
template <typename T, typename Src>
__device__ __forceinline__ void sample_by(const SampleArgs& a, int C, ClusterShared& sm) {
  constexpr int E = Vec<T>::E;
  constexpr bool kHeld = !std::is_same<Src, Stream<T>>::value;
  const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32, V = a.V;
  const int rank = kHeld && C > 1 ? (int)cluster_rank() : 0, r = kHeld ? blockIdx.x / C : blockIdx.x;
  const bool many = kHeld && C > 1;
  auto sync = [&]() {
    if (many)
      cluster_sync_all();
    else
      __syncthreads();
  };
  auto remote = [&](const void* p, int cta) { return map_rank(smem_u32(p), (uint32_t)cta); };

  Src row;
  row.load(a, r, rank);
  const Filter f = row_filter(a, r / a.R);
  row.inv_t = f.inv_t;
  row.ys = f.inv_t * kBinsPerNat;
  const bool by_k = f.top_k < V;
  const bool listing = (by_k && f.top_k <= kListTopK) || (!by_k && f.top_p < 1.f);

  // Sum over the cluster of a value per thread, to every thread.
  int turn = 0;
  auto cluster_sum = [&](u64 x) {
    const u64 mine = block_sum<kThreads>(x, sm.part);
    if (!many) return mine;
    turn ^= 1;  // the sum before this one may still be read
    if (tid == 0) sm.sum[turn] = mine;
    sync();
    u64 all = 0;
#pragma unroll
    for (int c = 0; c < kMaxCluster; ++c)
      if (c < C) all += ld_cluster_u64(remote(&sm.sum[turn], c));
    return all;
  };
  // Maximum over the block.
  auto block_top = [&](float top) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
    if (lane == 0) sm.wtop[warp] = top;
    __syncthreads();
    top = sm.wtop[lane % kWarps];
#pragma unroll
    for (int o = kWarps / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
    return top;
  };
  // Of a histogram over the cluster (sm.count): the first bin at which the running sum
  // reaches `lo` (positive), the first at which it reaches `hi` (the last bin where none
  // does), and what is before the former; the histogram is cleared.  In whole numbers: a bin
  // has one thread that finds it, and every CTA of a cluster finds the same, as its barriers
  // further on need.
  struct Bins {
    int x, y;
    u64 before, inside;  // of bin x; of bins x to y, also where y is the last one
  };
  auto find_bins = [&](int bins, u64 lo, u64 hi) {
    if (tid < 2) sm.bin[tid] = bins - 1;
    if (tid == 0) sm.before = sm.upto = 0;
    sync();
    // thread t sums bins 4t to 4t + 3 over the CTAs
    u64 x[4] = {0, 0, 0, 0};
    if (4 * tid < bins) {
#pragma unroll
      for (int c = 0; c < kMaxCluster; ++c) {
        if (c >= C) break;
        const float4 y = many ? ld_cluster_f4(remote(&sm.count[4 * tid], c)) : *reinterpret_cast<const float4*>(&sm.count[4 * tid]);
        x[0] += __float_as_uint(y.x);
        x[1] += __float_as_uint(y.y);
        x[2] += __float_as_uint(y.z);
        x[3] += __float_as_uint(y.w);
      }
    }
    u64 all;
    u64 before = block_scan((x[0] + x[1]) + (x[2] + x[3]), sm.part, &all);
    if (4 * tid < bins) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (before < lo && before + x[i] >= lo) {
          sm.bin[0] = 4 * tid + i;
          sm.before = before;
        }
        if (before < hi && before + x[i] >= hi) {
          sm.bin[1] = 4 * tid + i;
          sm.upto = before + x[i];
        }
        before += x[i];
      }
    }
    sync();  // every CTA has read the histograms
    if (4 * tid < kFineBins) *reinterpret_cast<uint4*>(&sm.count[4 * tid]) = make_uint4(0u, 0u, 0u, 0u);
    const Bins found{sm.bin[0], sm.bin[1], sm.before, (sm.bin[1] == bins - 1 ? all : sm.upto) - sm.before};
    __syncthreads();
    return found;
  };
  auto each = [&](auto take) {  // take(logit, index)
    row.vectors([&](const uint4& q, int index) {
#pragma unroll
      for (int e = 0; e < E; ++e) take(Vec<T>::value(q, e), index + e);
    });
    take(row.edge, row.edge_at);
  };
  auto append = [&](float v, int i) {
    const int at = atomicAdd(&sm.listed, 1);
    if (at < kList) sm.list[at] = make_key(v, (uint32_t)i);
  };
  // The tokens that reach `floor` into the list.
  auto collect = [&](const uint4& q, int index, float floor, float top) {
    if (top >= floor) {
      uint32_t hits = 0;
#pragma unroll
      for (int e = 0; e < E; ++e) hits |= (uint32_t)(Vec<T>::value(q, e) >= floor) << e;
      const int n = __popc(hits);
      int at = atomicAdd(&sm.listed, n);
      if (at + n > kList) hits = 0;
      for (; hits; hits &= hits - 1) {
        const int e = __ffs(hits) - 1;
        float v = Vec<T>::value(q, 0);
#pragma unroll
        for (int i = 1; i < E; ++i) v = e == i ? Vec<T>::value(q, i) : v;
        sm.list[at++] = make_key(v, (uint32_t)(index + e));
      }
    }
  };
  // CTA 0: the others' lists after its own; -1 where they are too long.  All CTAs call it.
  auto gather_lists = [&]() {
    sync();
    int n = sm.listed;
    if (rank == 0 && many) {
      int m[kMaxCluster], all = 0;
#pragma unroll
      for (int c = 0; c < kMaxCluster; ++c) {
        m[c] = c < C ? ld_cluster_s32(remote(&sm.listed, c)) : 0;
        all += m[c];
      }
      if (all <= kList) {
#pragma unroll
        for (int c = 1; c < kMaxCluster; ++c) {
          for (int i = tid; i < m[c]; i += kThreads) sm.list[n + i] = ld_cluster_u64(remote(&sm.list[i], c));
          n += m[c];
        }
      } else {
        n = kList + 1;
      }
      __syncthreads();
    }
    return n <= kList ? n : -1;
  };

  // ---- the maximum, and the sample ----
  if (tid == 0) sm.listed = 0;
  if (4 * tid < kFineBins) *reinterpret_cast<uint4*>(&sm.count[4 * tid]) = make_uint4(0u, 0u, 0u, 0u);
  float top = -INFINITY;
  float share = 1.f;
  if constexpr (kHeld) {
    row.vectors([&](const uint4& q, int) { top = fmaxf(top, Vec<T>::top(q)); });
    top = block_top(fmaxf(top, row.edge));
    if (many) {
      if (tid == 0) sm.top = top;
      sync();
#pragma unroll
      for (int c = 0; c < kMaxCluster; ++c)
        if (c < C) top = fmaxf(top, ld_cluster_f1(remote(&sm.top, c)));
    }
  } else {
    share = row.sample([&](const uint4& q) { top = fmaxf(top, Vec<T>::top(q)); });
    top = block_top(top);  // of the sample
  }
  row.top = top;
  // A logit that about enough tokens reach; where there are fewer of any weight, one that
  // all of these reach, at least the lowest finite one.
  constexpr float kLowest = -3.402823466e38f;
  float floor = kLowest;
  if (listing && top != -INFINITY) {
    share = row.sample([&](const uint4& q) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float y = row.depth(Vec<T>::value(q, e));
        if (y < (float)kBins) atomicAdd(&sm.count[(int)y], 1u);
      }
    });
    const float want = (float)(by_k ? f.top_k : kListTopP) * share;
    const u64 reach = f.top_k == 1 ? 1 : (u64)ceilf(want + 4.f * sqrtf(want) + 4.f);
    const int bin = find_bins(kBins, reach, reach).x;
    floor = fmaxf(kLowest, top - (bin < kBins - 1 ? (float)(bin + 1) : kBins + 1.f) / row.ys);
  } else {
    __syncthreads();
  }
  // ---- the list ----
  int state = kGeneral;
  if constexpr (!kHeld) {
    // the row's first reading: its maximum, and the list
    const float least = listing ? floor : INFINITY;
    row.vectors([&](const uint4& q, int index) {
      const float t = Vec<T>::top(q);
      top = fmaxf(top, t);
      collect(q, index, least, t);
    });
    top = fmaxf(top, row.edge);
    if (row.edge >= least && row.edge_at < V) append(row.edge, row.edge_at);
    top = block_top(top);
    row.top = top;
  } else if (listing) {
    row.vectors([&](const uint4& q, int index) { collect(q, index, floor, Vec<T>::top(q)); });
    if (row.edge >= floor && row.edge_at < V) append(row.edge, row.edge_at);
  }
  if (row.top == -INFINITY) {
    if (rank == 0 && tid == 0) {
      a.tokens[r] = -1;
      if (a.probs) a.probs[r] = 0.f;
    }
    sync();  // nobody reads this CTA's shared memory any more
    return;
  }
  u64 total = 0;  // the row's mass
  if (!by_k && f.top_p < 1.f) {
    u64 mine = 0;
    each([&](float v, int) { mine += row.mass(v); });
    total = cluster_sum(mine);
  }
  if (listing) {
    // whether what does not reach the floor has no weight
    const bool all = floor == kLowest || row.depth(floor) >= (float)kBins;
    const int n = gather_lists();
    if (rank == 0) {
      int st = kGeneral;
      if (n > 0) {
        if (f.top_k == 1) {
          u64 best = 0;
          for (int e = tid; e < n; e += kThreads) best = umax64(best, sm.list[e]);
          best = warp_max_key(best);
          if (lane == 0) sm.part[warp] = best;
          __syncthreads();
          if (tid == 0) {
            for (int w = 0; w < kWarps; ++w) best = umax64(best, sm.part[w]);
            a.tokens[r] = (int)key_index(best);
            if (a.probs) a.probs[r] = 1.f;
          }
          st = kDone;
        } else {
          // without top-k: whether the list holds the mass that top-p wants, before it is sorted
          bool holds = by_k || all;
          if (!holds) {
            u64 mine = 0;
            for (int e = tid; e < n; e += kThreads) mine += row.mass(key_value(sm.list[e]));
            holds = block_sum<kThreads>(mine, sm.part) >= top_p_target(f.top_p, total);
          }
          if (holds) {
            const float deep = fminf(fmaxf(row.depth(floor), 1.f), (float)kBins);
            sort_list(sm, n, row.top, row.ys * ((float)kFineBins / deep));
            if (finish_list(a, r, f, sm, row.top, n, total, all)) st = kDone;
          }
        }
      }
      state = st;
      if (many) {
        __syncthreads();
        if (tid == 0) sm.state = st;
      }
    }
    if (many) {
      sync();
      state = ld_cluster_s32(remote(&sm.state, 0));
    }
    if (state == kDone) {
      if (many) sync();  // CTA 0's state has been read
      return;
    }
    __syncthreads();
  }

  // ---- the general way: the last kept token, then the draw over the row ----
  // The last token of the prefix of the row in which a count or the mass reaches `target`,
  // as a key (0: not found this way).  `whole`: the count or mass of all of it; only keys
  // from `from` on are looked at.
  auto find_key = [&](u64 target, u64 whole, bool counts, u64 from) -> u64 {
    const float from_v = from ? key_value(from) : -INFINITY;
    const int from_i = (int)key_index(from);
    auto in = [&](float v, int i) { return v > from_v || (v == from_v && (uint32_t)i <= (uint32_t)from_i); };
    auto metric = [&](float v) -> u64 { return counts ? 1u : row.mass(v); };
    // The histograms hold counts, or masses without their low bits, so that they fit 32: a running
    // sum lacks less than a unit per token.
    const int bits = 64 - __clzll((long long)whole), low = !counts && bits > 32 ? bits - 32 : 0;
    auto place = [&](u64 goal, int low) {
      const u64 lack = low ? V : 0;
      goal = (goal + (1ull << low) - 1) >> low;
      return find_bins(kFineBins, goal > lack ? goal - lack : 1, goal);
    };
    constexpr float kSplit = (float)(kFineBins / kBins);
    each([&](float v, int i) {
      const float y = row.depth(v) * kSplit;
      const uint32_t w = counts ? 1u : row.mass(v) >> low;
      if (y < (float)kFineBins && in(v, i)) atomicAdd(&sm.count[(int)y], w);
    });
    const Bins coarse = place(target, low);
    float lo = (float)coarse.x / kSplit, hi = (float)(coarse.y + 1) / kSplit;
    // About how many tokens these bins hold, from their mass and the weight there: where that
    // is more than the list takes, a second histogram within them, in the units that their mass
    // allows, and the exact sum of what is before them.
    u64 above = 0;
    float from_y = 0.f;  // `above` has what is before it
    const float each_w = counts ? 1.f : fmaxf(1.f, kUnit / (float)(1ull << low) * expf(-hi / kBinsPerNat));
    if ((float)coarse.inside > each_w * (float)(kList / 2)) {
      const u64 most = coarse.inside + (low ? V : 0);
      const int less = max(0, 64 - __clzll((long long)most) + low - 32);
      const float per = (float)kFineBins / (hi - lo) * 0.999f;
      from_y = lo;
      each([&](float v, int i) {
        const float y = row.depth(v);
        const uint32_t w = counts ? 1u : row.mass(v);
        above += y < from_y ? w : 0u;
        if (y >= from_y && y < hi && in(v, i)) atomicAdd(&sm.count[(int)((y - from_y) * per)], w >> less);
      });
      above = cluster_sum(above);
      const Bins fine = place(target - min(target, above), less);
      // the bins' limits, moved apart by more than their rounding
      lo = from_y + ((float)fine.x / per) * 0.9999f - 1e-5f * from_y;
      hi = from_y + ((float)(fine.y + 1) / per) * 1.0001f + 1e-5f * from_y;
    }
    u64 between = 0;
    if (tid == 0) sm.listed = 0;
    __syncthreads();
    each([&](float v, int i) {
      const float y = row.depth(v);
      if (y >= from_y && y < hi) {
        if (y < lo)
          between += metric(v);
        else if (i < V && in(v, i))
          append(v, i);
      }
    });
    above += cluster_sum(between);
    const int n = gather_lists();
    if (rank == 0) {
      if (tid == 0) sm.key = 0;
      __syncthreads();
      if (n > 0 && above < target) {
        sort_list(sm, n, row.top - lo / row.ys, row.ys * ((float)kFineBins / (hi - lo)));
        const int per_thread = (n + kThreads - 1) / kThreads;
        u64 mine = 0;
        for (int i = 0; i < per_thread; ++i)
          if (tid * per_thread + i < n) mine += metric(key_value(sm.list[tid * per_thread + i]));
        u64 unused, run = above + block_scan(mine, sm.part, &unused);
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
    const u64 key = many ? ld_cluster_u64(remote(&sm.key, 0)) : sm.key;
    sync();
    return key;
  };

  u64 last = 0;  // keys from this one on are kept
  if (by_k) {
    u64 heavy = 0;  // tokens of any weight; no other one is drawn
    each([&](float v, int) { heavy += row.depth(v) < (float)kBins; });
    heavy = cluster_sum(heavy);
    if (heavy > (u64)f.top_k) {
      last = find_key((u64)f.top_k, heavy, true, 0);
      if (last == 0) state = kSlow;
    }
    if (state != kSlow && f.top_p < 1.f) {
      u64 mine = 0;
      each([&](float v, int i) {
        if (make_key(v, (uint32_t)i) >= last) mine += row.mass(v);
      });
      total = cluster_sum(mine);
    }
  }
  if (state != kSlow && f.top_p < 1.f) {
    const u64 target = top_p_target(f.top_p, total);
    const u64 key = find_key(target, total, false, last);
    if (key == 0)
      state = kSlow;
    else
      last = key;
  }
  if (state == kSlow) {
    sync();  // nobody reads the others' shared memory any more
    if (rank == 0) sample_row<T, kThreads>(a, r, sm.row);
    return;
  }
  const float last_v = last ? key_value(last) : -INFINITY;
  const int last_i = last ? (int)key_index(last) : V - 1;
  auto kept = [&](float v, int i) -> u64 {
    const float e = weight(v, row.top, f.inv_t);
    const uint32_t w = whole_weight(e);
    return (v > last_v || (v == last_v && i <= last_i)) && (v == row.top || !(e < f.min_p)) ? w : 0u;
  };
  auto kept_of = [&](const uint4& q, int index) {
    u64 x = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) x += kept(Vec<T>::value(q, e), index + e);
    return x;
  };
  // In index order: the elements before the vectors, the segments (of warps 0, 1, ..., then
  // those of the next number), CTA by CTA, the elements after the vectors.
  u64 mine = 0;
  if constexpr (kHeld) {
#pragma unroll
    for (int i = 0; i < Src::kSegments / kWarps; ++i) {
      u64 x = 0;
      row.segment(i, [&](const uint4& q, int index) { x = kept_of(q, index); });
      x = warp_sum(x);
      if (lane == 0) sm.seg[1 + i * kWarps + warp] = x;
      mine += x;
    }
  } else {
    row.run([&](const uint4& q, int index) {
      mine += kept_of(q, index);
      return true;
    });
    mine = warp_sum(mine);
    if (lane == 0) sm.seg[1 + warp] = mine;
  }
  const bool early = row.edge_at < row.head;
  if (warp == 0) {
    const u64 x = kept(row.edge, row.edge_at);
    const u64 head = warp_sum(early ? x : 0), tail = warp_sum(early ? 0 : x);
    if (lane == 0) {
      sm.seg[0] = head;
      sm.seg[1 + Src::kSegments] = tail;
    }
    mine += head;  // the tail follows the last CTA
  }
  const u64 whole = block_sum<kThreads>(lane == 0 ? mine : 0, sm.part);
  u64 before = 0, sum = whole, tail = sm.seg[1 + Src::kSegments];
  if (many) {
    turn ^= 1;
    if (tid == 0) sm.sum[turn] = whole;
    sync();
    sum = 0;
    for (int c = 0; c < C; ++c) {
      if (c == rank) before = sum;
      sum += ld_cluster_u64(remote(&sm.sum[turn], c));
    }
    tail = ld_cluster_u64(remote(&sm.seg[1 + Src::kSegments], 0));
  }
  const u64 body = sum;
  sum += tail;
  const u64 at = place_of(a.uniforms[r], sum);
  // A warp's elements with `run` before them: the one that holds the place, if any.
  auto look = [&](u64 x, u64 run, auto found) {
    u64 upto = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const u64 y = __shfl_up_sync(0xFFFFFFFFu, upto, o);
      if (lane >= o) upto += y;
    }
    if (run + upto > at && run + upto - x <= at) found(run + upto - x);
    return run + __shfl_sync(0xFFFFFFFFu, upto, 31);
  };
  auto look_vector = [&](const uint4& q, int index, u64 run) {
    return look(kept_of(q, index), run, [&](u64 s) {
      bool done = false;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float v = Vec<T>::value(q, e);
        s += kept(v, index + e);
        if (!done && s > at) {
          done = true;
          write_token(a, r, index + e, weight(v, row.top, f.inv_t), sum);
        }
      }
    });
  };
  if (rank == 0 && warp == 0) {
    const u64 x = kept(row.edge, row.edge_at);
    auto take = [&](u64) { write_token(a, r, row.edge_at, weight(row.edge, row.top, f.inv_t), sum); };
    if (at < sm.seg[0]) look(early ? x : 0, 0, take);
    if (at >= body) look(early ? 0 : x, body, take);
  }
  u64 run = before + (rank == 0 ? sm.seg[0] : 0);
  if (run <= at && at < before + whole) {
#pragma unroll
    for (int i = 0; i < Src::kSegments / kWarps; ++i) {
      u64 start = run;
      for (int w = 0; w < warp; ++w) start += sm.seg[1 + i * kWarps + w];
      if (start <= at && at < start + sm.seg[1 + i * kWarps + warp]) {
        if constexpr (kHeld) {
          row.segment(i, [&](const uint4& q, int index) { look_vector(q, index, start); });
        } else {
          row.run([&](const uint4& q, int index) {
            start = look_vector(q, index, start);
            return start <= at;
          });
        }
      }
      for (int w = 0; w < kWarps; ++w) run += sm.seg[1 + i * kWarps + w];
    }
  }
  if (many) sync();  // the others have read this CTA's sums
}

template <typename T, int NV>
__global__ void __launch_bounds__(kThreads, 2) sample_cluster_kernel(SampleArgs a, int C) {
  extern __shared__ __align__(16) unsigned char raw[];
  pdl_wait();
  sample_by<T, Held<T, NV>>(a, C, *reinterpret_cast<ClusterShared*>(raw));
}
template <typename T>
__global__ void __launch_bounds__(kThreads, 4) sample_stream_kernel(SampleArgs a) {
  extern __shared__ __align__(16) unsigned char raw[];
  pdl_wait();
  sample_by<T, Stream<T>>(a, 1, *reinterpret_cast<ClusterShared*>(raw));
}

template <auto kernel, typename... Args>
cudaError_t launch_rows(const SampleArgs& a, const DeviceInfo& dev, int C, cudaStream_t stream, Args... args) {
  constexpr size_t smem = sizeof(ClusterShared);
  static std::atomic<uint64_t> allowed{0};
  const cudaError_t e = allow_shared(kernel, smem, dev, allowed);
  if (e != cudaSuccess) return e;
  return launch_dependent(kernel, dim3((unsigned)(a.B * a.R) * C), dim3(kThreads), smem, stream, (unsigned)C, a, args...);
}

template <typename T>
cudaError_t launch_typed(const SampleArgs& a, cudaStream_t stream) {
  constexpr int E = Vec<T>::E;
  const long long rows = (long long)a.B * a.R, vecs = (a.V + E - 1) / E;
  DeviceInfo dev;
  const cudaError_t e = device_info(&dev);
  if (e != cudaSuccess) return e;
  auto need = [&](int C) { return (int)((vecs + (long long)C * kThreads - 1) / ((long long)C * kThreads)); };
  // A cluster for a row while the device has CTAs enough for all rows at once, as large as
  // that allows and the row fills.
  // Two of its CTAs fit an SM: with one, 15 clusters of eight find room, and 16 rows of
  // 151936 took 24.0 us, as two rounds of 12.9, where they take 14.1; streamed 18.7.
  // One row: 12.9, streamed 18.2; 64 rows of 20000: 10.9 in clusters of two, streamed 12.2;
  // 144: 9.5 and 12.5.  From 20 rows of 151936 on, clusters of four would need more than ten vectors to a
  // thread, and rows are streamed: 19 rows 15.2, 20 19.1, 64 19.3, 128 24.6, 256 30.6.
  int C = 1;
  while (C < kMaxCluster && need(C) > 1 && rows * C * 2 <= dev.sm_count) C *= 2;
  const int n = need(C);
  if (rows * C > dev.sm_count || n > 10) return launch_rows<sample_stream_kernel<T>>(a, dev, 1, stream);
  if (n <= 1) return launch_rows<sample_cluster_kernel<T, 1>>(a, dev, C, stream, C);
  if (n <= 2) return launch_rows<sample_cluster_kernel<T, 2>>(a, dev, C, stream, C);
  if (n <= 5) return launch_rows<sample_cluster_kernel<T, 5>>(a, dev, C, stream, C);
  return launch_rows<sample_cluster_kernel<T, 10>>(a, dev, C, stream, C);
}

}  // namespace

cudaError_t launch_sample(const SampleArgs& a, retrace_dtype dtype, cudaStream_t stream) {
  return dtype == RETRACE_BF16 ? launch_typed<__nv_bfloat16>(a, stream) : launch_typed<float>(a, stream);
}

}  // namespace retrace
