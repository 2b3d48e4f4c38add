// Attention over the paged cache on the CUDA cores: fp32, and the bf16 shapes that
// the tensor-core kernel does not take.
//
// Online softmax over tiles of 64 keys: with the running maximum m and sum l of a
// row, a tile's scores x give m' = max(m, x), p = exp(x - m'), l = l exp(m - m') + sum p,
// o = o exp(m - m') + p v.  A CTA of four warps holds R rows (tokens times query
// heads of one key/value head): scores as 4 rows x 4 keys (R = 8: x 1) per thread
// from K and Q in shared memory, the weights through shared memory, o in registers
// as 4 rows x D/16 (R = 8: D/64) columns.  The next tile's K loads while the softmax and
// the product with V run, the next V during the next scores.
#include <math.h>

#include "attend_plan.cuh"
#include "serve.h"

namespace retrace {
namespace {

constexpr int kThreads = 128;
constexpr int kKeys = 64;

__device__ __forceinline__ void cp_async16_zfill(uint32_t dst, const void* src, bool take) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(take ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

struct SimtParams {
  AttendArgs a;
  AttendShape shape;   // kv_heads: key/value heads times `splits`
  int splits, group;   // a key/value head's query heads in `splits` parts of `group`
  int vec;             // 16-byte accesses
};

template <int DP, int R>
struct SimtShared {
  float k[kKeys][DP + 4];  // + 4: 16-byte reads of consecutive rows fall into different banks
  float v[kKeys][DP];
  float q[R][DP + 4];
  float p[R][kKeys + 4];
  float m[R], l[R], alpha[R];
  long long off[2][kKeys];  // a key's place in the cache, -1: none, or seen by no row
  long long sum[kThreads / 32];
  PlanStart plan;
};

// Rows of D elements as fp32, zero beyond D, into rows of shared memory.
template <typename T, int DP, int kStride>
__device__ __forceinline__ void load_rows(float* dst, const T* base, const long long* off, int rows, int D, bool vec) {
  if (vec) {
    constexpr int N = 16 / sizeof(T), kChunks = DP / N;
    for (int i = threadIdx.x; i < rows * kChunks; i += kThreads) {
      const int r = i / kChunks, c = i % kChunks * N;
      const bool take = off[r] >= 0 && c < D;
      float* to = dst + r * kStride + c;
      const T* from = base + (take ? off[r] + c : 0);
      if constexpr (sizeof(T) == 4) {
        cp_async16_zfill(smem_u32(to), from, take);
      } else {
        const uint4 x = take ? __ldg(reinterpret_cast<const uint4*>(from)) : make_uint4(0u, 0u, 0u, 0u);
        *reinterpret_cast<float4*>(to) = make_float4(bf16_lo(x.x), bf16_hi(x.x), bf16_lo(x.y), bf16_hi(x.y));
        *reinterpret_cast<float4*>(to + 4) = make_float4(bf16_lo(x.z), bf16_hi(x.z), bf16_lo(x.w), bf16_hi(x.w));
      }
    }
    return;
  }
  for (int i = threadIdx.x; i < rows * DP; i += kThreads) {
    const int r = i / DP, c = i % DP;
    dst[r * kStride + c] = off[r] >= 0 && c < D ? to_f32(base[off[r] + c]) : 0.f;
  }
}

template <typename T, int DP, int R>
__global__ void __launch_bounds__(kThreads) attend_simt_kernel(const __grid_constant__ SimtParams P) {
  extern __shared__ __align__(16) unsigned char raw[];
  SimtShared<DP, R>& sm = *reinterpret_cast<SimtShared<DP, R>*>(raw);
  const AttendArgs& a = P.a;
  const retrace_kv_cache& cache = a.cache;
  const int tid = threadIdx.x, D = cache.head_dim;
  plan_start<kThreads, kKeys>(P.shape, gridDim.x, 1, &sm.plan, sm.sum);
  const PlanStart plan = sm.plan;
  PieceWalk walk;
  walk.start(plan);

  // A thread's part of the scores and of o: 4 rows each.
  constexpr int kRowGroups = R / 4, kLanes = kThreads / kRowGroups;  // threads of a row group
  constexpr int kKeysEach = kKeys / kLanes;                          // 4 or 1
  constexpr int kCols = DP / kLanes;                                 // columns of o per thread
  constexpr int kColVec = kCols >= 4 ? 4 : 1, kColSteps = kCols / kColVec;
  const int rg = tid / kLanes, lane = tid % kLanes;

  JoinUnit unit{};
  Piece pc;
  while (walk.next<kKeys, true>(P.shape, plan, &pc)) {
    const int kv_head = pc.head / P.splits, part = pc.head % P.splits;
    const int G_all = a.q_heads / cache.kv_heads;
    const int G = min(P.group, G_all - part * P.group), h0 = kv_head * G_all + part * P.group;
    const int rows = (pc.i1 - pc.i0) * G;
    const UnitKeys& keys = pc.keys;
    const T* kbase = static_cast<const T*>(cache.k) + kv_head * cache.head_stride;
    const T* vbase = static_cast<const T*>(cache.v) + kv_head * cache.head_stride;

    auto offsets = [&](int k) {  // of tile k of the piece
      if (tid < kKeys && k < pc.k1) {
        const int j = keys.tile(k) * kKeys + tid;
        long long off = -1;
        if (j <= keys.hi && (j >= keys.lo || j < a.sinks)) {
          const int page = page_of(cache, pc.b, j / cache.page_size);
          if (page >= 0) off = page * cache.page_stride + (j % cache.page_size) * cache.slot_stride;
        }
        sm.off[k & 1][tid] = off;
      }
    };

    __syncthreads();  // the previous piece's shared memory is free
    offsets(pc.k0);
    if (tid < R) {
      sm.m[tid] = -INFINITY;
      sm.l[tid] = 0.f;
    }
    for (int i = tid; i < R * DP; i += kThreads) {
      const int r = i / DP, c = i % DP;
      float x = 0.f;
      if (r < rows && c < D)
        x = to_f32(static_cast<const T*>(a.q)[(long long)(pc.row0 + pc.i0 + r / G) * a.q_token + (h0 + r % G) * a.q_head + c]);
      sm.q[r][c] = x;
    }
    float acc[4][kCols];
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int c = 0; c < kCols; ++c) acc[r][c] = 0.f;
    __syncthreads();
    if (pc.k0 < pc.k1) {
      load_rows<T, DP, DP + 4>(&sm.k[0][0], kbase, sm.off[pc.k0 & 1], kKeys, D, P.vec);
      cp_async_commit();
      load_rows<T, DP, DP>(&sm.v[0][0], vbase, sm.off[pc.k0 & 1], kKeys, D, P.vec);
      cp_async_commit();
    }

    for (int k = pc.k0; k < pc.k1; ++k) {
      offsets(k + 1);
      cp_async_wait<1>();  // this tile's K
      __syncthreads();
      {
        float s[4][kKeysEach];
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int j = 0; j < kKeysEach; ++j) s[r][j] = 0.f;
#pragma unroll 4
        for (int c = 0; c < DP; c += 4) {
          float4 q[4], x[kKeysEach];
#pragma unroll
          for (int r = 0; r < 4; ++r) q[r] = *reinterpret_cast<const float4*>(&sm.q[rg * 4 + r][c]);
#pragma unroll
          for (int j = 0; j < kKeysEach; ++j) x[j] = *reinterpret_cast<const float4*>(&sm.k[lane + j * kLanes][c]);
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < kKeysEach; ++j) {
              s[r][j] = fmaf(q[r].x, x[j].x, s[r][j]);
              s[r][j] = fmaf(q[r].y, x[j].y, s[r][j]);
              s[r][j] = fmaf(q[r].z, x[j].z, s[r][j]);
              s[r][j] = fmaf(q[r].w, x[j].w, s[r][j]);
            }
        }
        // What a row does not see is replaced, not added to: its bits may be anything.
        const int j0 = keys.tile(k) * kKeys;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int row = rg * 4 + r, p = pc.c + pc.i0 + row / G;
          const int hi = a.causal ? p : pc.c + pc.n - 1, lo = a.window > 0 ? p - a.window + 1 : 0;
#pragma unroll
          for (int j = 0; j < kKeysEach; ++j) {
            const int at = j0 + lane + j * kLanes;
            const bool seen = at <= hi && (at >= lo || at < a.sinks) && sm.off[k & 1][lane + j * kLanes] >= 0;
            sm.p[row][lane + j * kLanes] = seen ? s[r][j] * a.scale : -INFINITY;
          }
        }
      }
      __syncthreads();
      if (k + 1 < pc.k1) load_rows<T, DP, DP + 4>(&sm.k[0][0], kbase, sm.off[(k + 1) & 1], kKeys, D, P.vec);
      cp_async_commit();
      {
        constexpr int kEach = kThreads / R;  // threads of a row
        const int row = tid / kEach, i0 = tid % kEach;
        float top = -INFINITY;
#pragma unroll
        for (int i = i0; i < kKeys; i += kEach) top = fmaxf(top, sm.p[row][i]);
#pragma unroll
        for (int o = kEach / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
        const float old = sm.m[row], m = fmaxf(old, top), ref = m == -INFINITY ? 0.f : m;
        float sum = 0.f;
#pragma unroll
        for (int i = i0; i < kKeys; i += kEach) {
          const float w = expf(sm.p[row][i] - ref);
          sm.p[row][i] = w;
          sum += w;
        }
#pragma unroll
        for (int o = kEach / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
        if (i0 == 0) {
          const float al = expf(old - ref);
          sm.m[row] = m;
          sm.alpha[row] = al;
          sm.l[row] = sm.l[row] * al + sum;
        }
      }
      cp_async_wait<1>();  // this tile's V
      __syncthreads();
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float al = sm.alpha[rg * 4 + r];
#pragma unroll
        for (int c = 0; c < kCols; ++c) acc[r][c] *= al;
      }
#pragma unroll 2
      for (int j = 0; j < kKeys; j += 4) {
        float4 w[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) w[r] = *reinterpret_cast<const float4*>(&sm.p[rg * 4 + r][j]);
#pragma unroll
        for (int jj = 0; jj < 4; ++jj) {
          float x[kCols];
#pragma unroll
          for (int c = 0; c < kColSteps; ++c) {
            const float* from = &sm.v[j + jj][(lane + c * kLanes) * kColVec];
            if constexpr (kColVec == 4)
              *reinterpret_cast<float4*>(&x[c * 4]) = *reinterpret_cast<const float4*>(from);
            else
              x[c] = *from;
          }
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float ww = jj == 0 ? w[r].x : jj == 1 ? w[r].y : jj == 2 ? w[r].z : w[r].w;
#pragma unroll
            for (int c = 0; c < kCols; ++c) acc[r][c] = fmaf(ww, x[c], acc[r][c]);
          }
        }
      }
      __syncthreads();
      if (k + 1 < pc.k1) load_rows<T, DP, DP>(&sm.v[0][0], vbase, sm.off[(k + 1) & 1], kKeys, D, P.vec);
      cp_async_commit();
    }
    cp_async_wait<0>();
    __syncthreads();

    auto column = [&](int c) { return (lane + c / kColVec * kLanes) * kColVec + c % kColVec; };
    auto put = [&](int row, int col, float x) {
      static_cast<T*>(a.out)[(long long)(pc.row0 + pc.i0 + row / G) * a.out_token + (h0 + row % G) * a.out_head + col] =
          from_f32<T>(x);
    };
    if (pc.pieces == 1) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = rg * 4 + r;
        if (row >= rows) continue;
        const float l = sm.l[row], inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
        for (int c = 0; c < kCols; ++c)
          if (column(c) < D) put(row, column(c), acc[r][c] * inv);
      }
      continue;
    }
    // A part of a unit: rows, maxima and sums to the workspace.
    constexpr int kPart = R * (DP + 2);
    float* to = a.partials + ((long long)blockIdx.x * 2 + (pc.k0 == 0 ? 1 : 0)) * kPart;
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int c = 0; c < kCols; ++c) to[(rg * 4 + r) * DP + column(c)] = acc[r][c];
    if (tid < R) *reinterpret_cast<float2*>(to + R * DP + tid * 2) = make_float2(sm.m[tid], sm.l[tid]);
    if (pc.k0 == 0) unit = JoinUnit{pc.pieces, rows, rows, pc.row0 + pc.i0, h0, G, {0, 0}};
  }
  if (tid == 0) a.units[blockIdx.x] = unit;
}

template <typename T, int DP, int R>
cudaError_t launch(SimtParams& p, cudaStream_t stream) {
  constexpr size_t smem = sizeof(SimtShared<DP, R>);
  auto kernel = attend_simt_kernel<T, DP, R>;
  DeviceInfo dev;
  cudaError_t e = device_info(&dev);
  if (e != cudaSuccess) return e;
  static std::atomic<uint64_t> allowed{0};
  if ((e = allow_shared(kernel, smem, dev, allowed)) != cudaSuccess) return e;
  constexpr int kPerSm = smem <= 75 * 1024 ? 3 : smem <= 113 * 1024 ? 2 : 1;
  int grid = dev.sm_count * kPerSm;
  if (grid > kAttendMaxCtas) grid = kAttendMaxCtas;
  p.splits = (p.a.q_heads / p.a.cache.kv_heads + R - 1) / R;
  p.group = (p.a.q_heads / p.a.cache.kv_heads + p.splits - 1) / p.splits;
  p.shape.kv_heads = p.a.cache.kv_heads * p.splits;
  p.shape.unit_tokens = R / p.group;
  kernel<<<grid, kThreads, smem, stream>>>(p);
  if ((e = cudaGetLastError()) != cudaSuccess) return e;
  return launch_attend_join(p.a, PartShape{R, DP, 0}, grid, stream);
}

template <typename T, int DP>
cudaError_t launch_rows(SimtParams& p, cudaStream_t stream) {
  // Eight rows where a sequence has no more on average, 32 otherwise.
  const long long G = p.a.q_heads / p.a.cache.kv_heads;
  return (long long)p.a.T * G <= 8ll * p.a.B ? launch<T, DP, 8>(p, stream) : launch<T, DP, 32>(p, stream);
}

template <typename T>
cudaError_t launch_typed(SimtParams& p, cudaStream_t stream) {
  const int D = p.a.cache.head_dim;
  return D <= 64 ? launch_rows<T, 64>(p, stream) : D <= 128 ? launch_rows<T, 128>(p, stream) : launch_rows<T, 256>(p, stream);
}

}  // namespace

size_t attend_simt_partial_bytes(int head_dim) {
  const size_t DP = head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : 256;
  return (size_t)kAttendMaxCtas * 2 * 32 * (DP + 2) * 4;
}

cudaError_t launch_attend_simt(const AttendArgs& a, cudaStream_t stream) {
  SimtParams p{};
  p.a = a;
  const retrace_kv_cache& c = a.cache;
  p.shape.q_start = a.q_start;
  p.shape.cache_len = a.cache_len;
  p.shape.B = a.B;
  p.shape.T = a.T;
  p.shape.uniform = a.q_start ? 0 : a.T / a.B;
  p.shape.causal = a.causal;
  p.shape.window = a.window;
  p.shape.sinks = a.sinks;
  p.shape.places = c.max_pages * c.page_size;
  const int n = c.dtype == RETRACE_BF16 ? 8 : 4;
  auto whole = [n](long long x) { return x % n == 0; };
  p.vec = whole(c.head_dim) && whole(c.head_stride) && whole(c.slot_stride) && whole(c.page_stride) &&
          (((uintptr_t)c.k | (uintptr_t)c.v) & 15u) == 0;
  return c.dtype == RETRACE_BF16 ? launch_typed<__nv_bfloat16>(p, stream) : launch_typed<float>(p, stream);
}

}  // namespace retrace
