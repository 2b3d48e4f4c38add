// Pages for a batch's next tokens, from a stack of free ones, and where the tokens go.
//
// need = ceil((cached + new) / page size) pages a sequence; running sums over the sequences of
// what each takes, gives back and appends say which entry of the stack, and of the
// token list, is whose.  One cluster of CTAs does a call: each works the sums out for itself
// (they are a few words a sequence); then a thread takes a page, or a token, and finds its sequence among
// the sums, so the lengths may be as they like.  What is read in place is written after a barrier of the
// cluster: the places on the stack that are given back to are in part those that were taken from.
// Long lists of tokens are written by a second kernel on the whole device.  Latency: a few reads, three barriers.  In a
// graph a call takes 3 us for 8 sequences of a token, 5 for 256 of 17, 11 for 2048 prompts of 1000 tokens (and 7 to list
// those, 16 MB).
#include "serve.h"
#include "tokens.cuh"

namespace retrace {
namespace {

constexpr int kMostThreads = 1024;
constexpr int kEach = 2;  // sequences of a thread
constexpr int kMostCtas = 8;
constexpr int kListThreads = 256;
constexpr int kListTokens = 16384;  // from here on a kernel of its own lists the tokens
constexpr int kListEach = 8;        // tokens of a lane of that

struct Sums {
  long long take, give, tokens;
  __device__ __forceinline__ Sums operator+(const Sums& o) const { return {take + o.take, give + o.give, tokens + o.tokens}; }
};

struct Sequence {
  int cached, tokens;  // in the cache, new
  int held, need;      // pages
  __device__ __forceinline__ int take() const { return max(need - held, 0); }
  __device__ __forceinline__ int give() const { return max(held - need, 0); }
  __device__ __forceinline__ Sums sums() const { return {take(), give(), tokens}; }
};

__device__ __forceinline__ Sequence load_sequence(const ReserveArgs& a, int b) {
  Sequence q{};
  if (b >= a.B) return q;
  q.cached = cached_tokens(a.cache_len, b);
  q.tokens = min(max(a.new_len[b], 0), 1 << 30);
  const int end = min(max(q.cached + q.tokens, 0), a.max_pages * a.page_size);
  q.need = end / a.page_size + (end % a.page_size > 0);
  q.held = min(max(a.held[b], 0), a.max_pages);
  return q;
}

__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

struct Shared {
  Sums warp[kMostThreads / 32];
  __device__ __forceinline__ Sums* upto() { return reinterpret_cast<Sums*>(this + 1); }  // of the sequences up to each one of the chunk
  __device__ __forceinline__ Sequence* seq() { return reinterpret_cast<Sequence*>(upto() + blockDim.x * kEach); }
};
constexpr int kSharedEach = kEach * (sizeof(Sums) + sizeof(Sequence));  // bytes to a thread

// The chunk's n sequences from b0 and the sums up to each, into shared memory; returns the sums up to the last.
__device__ __forceinline__ Sums scan_chunk(const ReserveArgs& a, Shared& sm, int b0, int n, const Sums& before) {
  const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32, warps = (n + 32 * kEach - 1) / (32 * kEach);
  Sequence q[kEach];
  Sums mine{0, 0, 0}, x = mine;
  if (warp < warps) {
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      q[i] = load_sequence(a, b0 + tid * kEach + i);
      mine = mine + q[i].sums();
    }
    x = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const Sums y{__shfl_up_sync(0xFFFFFFFFu, x.take, o), __shfl_up_sync(0xFFFFFFFFu, x.give, o), __shfl_up_sync(0xFFFFFFFFu, x.tokens, o)};
      if (lane >= o) x = x + y;
    }
  }
  __syncthreads();  // the chunk before has been read
  if (warp < warps && lane == 31) sm.warp[warp] = x;
  __syncthreads();
  Sums at = before, all = before;
  for (int w = 0; w < warps; ++w) {
    if (w < warp) at = at + sm.warp[w];
    all = all + sm.warp[w];
  }
  if (warp < warps) {
    at = Sums{at.take + x.take - mine.take, at.give + x.give - mine.give, at.tokens + x.tokens - mine.tokens};
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      at = at + q[i].sums();
      sm.seq()[tid * kEach + i] = q[i];
      sm.upto()[tid * kEach + i] = at;
    }
  }
  __syncthreads();
  return all;
}

// The first of the chunk's n sequences whose sum passes `at`.
template <typename Sum>
__device__ __forceinline__ int find(Shared& sm, int n, long long at, Sum&& sum) {
  int lo = 0;
  while (n > 0) {
    const int half = n / 2;
    const bool below = sum(sm.upto()[lo + half]) <= at;
    lo = below ? lo + half + 1 : lo;
    n = below ? n - half - 1 : half;
  }
  return lo;
}

__global__ void __launch_bounds__(kMostThreads) kv_reserve_kernel(const __grid_constant__ ReserveArgs a, int list_tokens) {
  extern __shared__ __align__(16) unsigned char raw[];
  Shared& sm = *reinterpret_cast<Shared*>(raw);
  const int thread = blockIdx.x * blockDim.x + threadIdx.x, threads = gridDim.x * blockDim.x, chunk = blockDim.x * kEach;
  pdl_launch_dependents();
  pdl_wait();
  const int count = min(max(a.counts[0], 0), a.num_pages);
  const bool one = a.B <= chunk;  // one chunk, scanned once
  Sums all{0, 0, 0};
  for (int b0 = 0; b0 < a.B; b0 += chunk) all = scan_chunk(a, sm, b0, min(chunk, a.B - b0), all);
  const long long got = min(all.take, (long long)count), left = count - got;

  // work(first sequence, sequences of the chunk, sums before it, up to its end) for all chunks; `apart`: what
  // work writes is what the scan reads.
  auto chunks = [&](bool apart, auto&& work) {
    Sums before{0, 0, 0};
    for (int b0 = 0; b0 < a.B; b0 += chunk) {
      const int n = min(chunk, a.B - b0);
      const Sums upto = one ? all : scan_chunk(a, sm, b0, n, before);
      if (!one && apart) cluster_barrier();
      work(b0, n, before, upto);
      before = upto;
    }
  };
  // The page of the stack for the k-th page that is taken.
  auto taken = [&](long long k) { return k < count ? a.free_pages[count - 1 - k] : -1; };
  chunks(false, [&](int b0, int n, const Sums& before, const Sums& upto) {
    for (long long k = before.take + thread; k < upto.take; k += threads) {
      const int i = find(sm, n, k, [](const Sums& x) { return x.take; });
      a.page_table[(b0 + i) * a.table_stride + sm.seq()[i].need - (sm.upto()[i].take - k)] = taken(k);
    }
    if (a.q_start)
      for (int i = thread; i < n; i += threads) a.q_start[b0 + i] = (int)min(sm.upto()[i].tokens - sm.seq()[i].tokens, (long long)a.T);
    if (!list_tokens) return;
    const long long end = min(upto.tokens, (long long)a.T);
    for (long long t = before.tokens + thread; t < end; t += threads) {
      const int i = find(sm, n, t, [](const Sums& x) { return x.tokens; });
      const Sequence q = sm.seq()[i];
      const int p = q.cached + q.tokens - (int)(sm.upto()[i].tokens - t);
      long long slot = -1;
      if (p >= 0 && p < a.max_pages * a.page_size) {
        // a page that this call takes may not be in the table yet
        const int index = p / a.page_size;
        const int page = index < q.held ? a.page_table[(b0 + i) * a.table_stride + index] : taken(sm.upto()[i].take - (q.need - index));
        if (page >= 0) slot = (long long)page * a.page_size + (p - index * a.page_size);
      }
      a.slots[t] = slot;
    }
  });
  if (a.q_start && thread == 0) a.q_start[a.B] = (int)min(all.tokens, (long long)a.T);
  if (list_tokens)
    for (long long t = all.tokens + thread; t < a.T; t += threads) a.slots[t] = -1;

  cluster_barrier();  // the stack and the lengths have been read
  if (all.give > 0)
    chunks(false, [&](int b0, int n, const Sums& before, const Sums& upto) {
      for (long long k = before.give + thread; k < upto.give; k += threads) {
        const int i = find(sm, n, k, [](const Sums& x) { return x.give; });
        int32_t* at = a.page_table + (b0 + i) * a.table_stride + sm.seq()[i].held - (sm.upto()[i].give - k);
        const long long to = left + all.give - 1 - k;
        if (to < a.num_pages) a.free_pages[to] = *at;
        *at = -1;
      }
    });
  chunks(true, [&](int b0, int n, const Sums&, const Sums&) {
    for (int i = thread; i < n; i += threads) {
      const Sequence q = sm.seq()[i];
      const long long mine = min(max(count - (sm.upto()[i].take - q.take()), 0ll), (long long)q.take());
      a.held[b0 + i] = q.give() > 0 ? q.need : q.held + (int)mine;
    }
  });
  if (thread == 0) {
    a.counts[0] = (int)min(left + all.give, (long long)a.num_pages);
    a.counts[1] = (int)min(all.take - got, (long long)0x7FFFFFFF);
  }
}

// The token list from the table and the starts: a warp finds the sequence of the first of its tokens, the
// lanes go on from there.
__global__ void __launch_bounds__(kListThreads) kv_slots_kernel(const __grid_constant__ ReserveArgs a, FastDivide page_size) {
  pdl_launch_dependents();
  pdl_wait();
  constexpr int kSpan = 32 * kListEach;
  const int lane = threadIdx.x % 32, total = a.q_start[a.B], places = a.max_pages * a.page_size;
  const int warps = gridDim.x * (kListThreads / 32);
  for (int t0 = (blockIdx.x * (kListThreads / 32) + threadIdx.x / 32) * kSpan; t0 < a.T; t0 += warps * kSpan) {
    int first, b = sequence_of(a.q_start, a.B, 0, t0, lane, &first);
    int next = b >= 0 ? a.q_start[b + 1] : 0, cached = b >= 0 ? cached_tokens(a.cache_len, b) : 0;
#pragma unroll
    for (int u = 0; u < kListEach; ++u) {
      const int t = t0 + u * 32 + lane;
      long long slot = -1;
      if (b >= 0 && t < total) {
        if (t >= next) {
          b = sequence_from(a.q_start, a.B, b, t);
          first = a.q_start[b];
          next = a.q_start[b + 1];
          cached = cached_tokens(a.cache_len, b);
        }
        const int p = cached + (t - first);
        if (p >= 0 && p < places) {
          const int index = page_size(p), page = a.page_table[b * a.table_stride + index];
          if (page >= 0) slot = (long long)page * a.page_size + (p - index * a.page_size);
        }
      }
      if (t < a.T) a.slots[t] = slot;
    }
  }
}

}  // namespace

cudaError_t launch_kv_reserve(const ReserveArgs& a, cudaStream_t stream) {
  // One small CTA where its threads have a few tokens and pages each.  In one graph, a call that takes and a call
  // that gives back: 8 sequences of a token 6.5 us on one CTA of 512 (8.0 on eight of 1024), 256 sequences of 17 tokens
  // 15.1 (9.8), 2048 prompts of 1000 tokens 148 (30.6).  It does not look at pages: 128 prompts of 4096 tokens in pages of
  // 16 take 81 us without a list of their tokens, and 53, with more threads, where they are listed too.
  const bool few = a.B <= 128 && (!a.slots || a.T <= 4096);
  const bool listed = a.slots && a.T > kListTokens;
  const int ctas = few ? 1 : kMostCtas, threads = few ? 512 : kMostThreads;
  const int shared = sizeof(Shared) + threads * kSharedEach;
  DeviceInfo dev;
  cudaError_t e = device_info(&dev);
  if (e != cudaSuccess) return e;
  static std::atomic<uint64_t> allowed{0};
  if ((e = allow_shared(kv_reserve_kernel, sizeof(Shared) + kMostThreads * kSharedEach, dev, allowed)) != cudaSuccess) return e;
  e = launch_dependent(kv_reserve_kernel, dim3(ctas), dim3(threads), shared, stream, (unsigned)ctas, a, (int)(a.slots && !listed));
  if (e != cudaSuccess || !listed) return e;
  const int span = kListThreads * kListEach, all = (a.T + span - 1) / span, resident = dev.sm_count * 8;
  return launch_dependent(kv_slots_kernel, dim3(all < resident ? all : resident), dim3(kListThreads), 0, stream, 1u, a,
                          FastDivide::of(a.page_size));
}

}  // namespace retrace
