// Pages for a batch's next tokens, from a stack of free ones, and where the tokens go.
//
// need = ceil((cached + new) / page size) pages a sequence; running sums over the sequences of
// what each takes, gives back and appends say which entry of the stack, and of the
// token list, is whose.  One cluster of CTAs does a call: each works the sums out for itself
// (they are a few words a sequence) and moves the pages of its share of the sequences.  What is read in
// place is written after a barrier of the cluster: the places on the stack that are
// given back to are in part those that were taken from.  Long lists of tokens are written by
// a second kernel on the whole device.  Latency: a few reads, three barriers.
#include "serve.h"
#include "tokens.cuh"

namespace retrace {
namespace {

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kMostCtas = 8;
constexpr int kListThreads = 256;
constexpr int kListTokens = 16384;  // from here on a kernel of its own lists the tokens

struct Sums {
  long long take, give, tokens;
  __device__ __forceinline__ Sums operator+(const Sums& o) const { return {take + o.take, give + o.give, tokens + o.tokens}; }
};

struct Sequence {
  int cached, tokens;  // in the cache, new
  int held, need;      // pages
  __device__ __forceinline__ int take() const { return max(need - held, 0); }
  __device__ __forceinline__ int give() const { return max(held - need, 0); }
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
  Sums warp[kWarps];
  Sequence seq[kThreads];
  Sums before[kThreads];  // of the sequences before each one of the chunk
};

// The sequences [b0, b0 + kThreads) and the sums before them, into shared memory; returns
// `before` plus the chunk's own sums.
__device__ __forceinline__ Sums scan_chunk(const ReserveArgs& a, Shared& sm, int b0, const Sums& before) {
  const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
  const Sequence q = load_sequence(a, b0 + tid);
  const Sums mine{q.take(), q.give(), q.tokens};
  Sums x = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const Sums y{__shfl_up_sync(0xFFFFFFFFu, x.take, o), __shfl_up_sync(0xFFFFFFFFu, x.give, o), __shfl_up_sync(0xFFFFFFFFu, x.tokens, o)};
    if (lane >= o) x = x + y;
  }
  __syncthreads();  // the chunk before has been read
  if (lane == 31) sm.warp[warp] = x;
  __syncthreads();
  Sums from = before, all = before;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) from = from + sm.warp[w];
    all = all + sm.warp[w];
  }
  sm.seq[tid] = q;
  sm.before[tid] = Sums{from.take + x.take - mine.take, from.give + x.give - mine.give, from.tokens + x.tokens - mine.tokens};
  __syncthreads();
  return all;
}

__device__ __forceinline__ long long slot_of(const ReserveArgs& a, int b, int p) {
  if (p < 0 || p >= a.max_pages * a.page_size) return -1;
  const int page = a.page_table[b * a.table_stride + p / a.page_size];
  return page < 0 ? -1 : (long long)page * a.page_size + p % a.page_size;
}

__global__ void __launch_bounds__(kThreads) kv_reserve_kernel(const __grid_constant__ ReserveArgs a, int list_tokens) {
  __shared__ Shared sm;
  const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
  pdl_launch_dependents();
  pdl_wait();
  const int count = min(max(a.counts[0], 0), a.num_pages);
  const bool one = a.B <= kThreads;  // one chunk, scanned once
  Sums all{0, 0, 0};
  for (int b0 = 0; b0 < a.B; b0 += kThreads) all = scan_chunk(a, sm, b0, all);
  const long long got = min(all.take, (long long)count), left = count - got;

  // This warp's sequences of each chunk; `apart`: what work writes is what the scan reads.
  const int first = blockIdx.x * kWarps + warp, stride = gridDim.x * kWarps;
  auto each = [&](bool apart, auto&& work) {
    Sums before{0, 0, 0};
    for (int b0 = 0; b0 < a.B; b0 += kThreads) {
      if (!one) before = scan_chunk(a, sm, b0, before);
      if (!one && apart) cluster_barrier();
      for (int i = first; i < min(kThreads, a.B - b0); i += stride) work(b0 + i, sm.seq[i], sm.before[i]);
    }
  };
  // Pages taken; then the sequence's tokens, whose pages this warp has just written.
  each(false, [&](int b, const Sequence& q, const Sums& before) {
    int32_t* row = a.page_table + b * a.table_stride;
    for (int k = lane; k < q.take(); k += 32) {
      const long long at = count - 1 - (before.take + k);
      row[q.held + k] = at >= 0 ? a.free_pages[at] : -1;
    }
    if (a.q_start && lane == 0) a.q_start[b] = (int)min(before.tokens, (long long)a.T);
    if (!list_tokens) return;
    __syncwarp();
    for (int k = lane; k < q.tokens; k += 32) {
      if (before.tokens + k >= a.T) break;
      a.slots[before.tokens + k] = slot_of(a, b, q.cached + k);
    }
  });
  const int thread = blockIdx.x * kThreads + tid, threads = gridDim.x * kThreads;
  if (a.q_start && thread == 0) a.q_start[a.B] = (int)min(all.tokens, (long long)a.T);
  if (list_tokens)
    for (long long t = all.tokens + thread; t < a.T; t += threads) a.slots[t] = -1;

  cluster_barrier();  // the stack and the lengths have been read
  if (all.give > 0)
    each(false, [&](int b, const Sequence& q, const Sums& before) {
      int32_t* row = a.page_table + b * a.table_stride;
      for (int k = lane; k < q.give(); k += 32) {
        const long long at = left + all.give - 1 - (before.give + k);
        if (at < a.num_pages) a.free_pages[at] = row[q.need + k];
        row[q.need + k] = -1;
      }
    });
  each(true, [&](int b, const Sequence& q, const Sums& before) {
    if (lane != 0) return;
    const long long mine = min(max(count - before.take, 0ll), (long long)q.take());
    a.held[b] = q.give() > 0 ? q.need : q.held + (int)mine;
  });
  if (thread == 0) {
    a.counts[0] = (int)min(left + all.give, (long long)a.num_pages);
    a.counts[1] = (int)min(all.take - got, (long long)0x7FFFFFFF);
  }
}

// The token list from the table and the starts: a warp finds the sequence of the first of
// its 32 tokens, the others go on from there.
__global__ void __launch_bounds__(kListThreads) kv_slots_kernel(const __grid_constant__ ReserveArgs a) {
  pdl_launch_dependents();
  pdl_wait();
  const int lane = threadIdx.x % 32, total = a.q_start[a.B];
  const int warps = gridDim.x * (kListThreads / 32);
  for (int t0 = (blockIdx.x * (kListThreads / 32) + threadIdx.x / 32) * 32; t0 < a.T; t0 += warps * 32) {
    const int t = t0 + lane;
    int first, b = sequence_of(a.q_start, a.B, 0, t0, lane, &first);
    long long slot = -1;
    if (b >= 0 && t < total) {
      int next = a.q_start[b + 1];
      while (t >= next) {  // t < total: it ends
        first = next;
        next = a.q_start[++b + 1];
      }
      slot = slot_of(a, b, cached_tokens(a.cache_len, b) + (t - first));
    }
    if (t < a.T) a.slots[t] = slot;
  }
}

}  // namespace

cudaError_t launch_kv_reserve(const ReserveArgs& a, cudaStream_t stream) {
  // One CTA where it has a sequence or two to a warp.
  const bool few = a.B <= 2 * kWarps && (!a.slots || a.T <= 4096);
  const bool listed = a.slots && a.T > kListTokens;
  const int ctas = few ? 1 : kMostCtas;
  cudaError_t e = launch_dependent(kv_reserve_kernel, dim3(ctas), dim3(kThreads), 0, stream, (unsigned)ctas, a, (int)(a.slots && !listed));
  if (e != cudaSuccess || !listed) return e;
  DeviceInfo dev;
  if ((e = device_info(&dev)) != cudaSuccess) return e;
  const int all = (a.T + kListThreads - 1) / kListThreads, resident = dev.sm_count * 8;
  return launch_dependent(kv_slots_kernel, dim3(all < resident ? all : resident), dim3(kListThreads), 0, stream, 1u, a);
}

}  // namespace retrace
