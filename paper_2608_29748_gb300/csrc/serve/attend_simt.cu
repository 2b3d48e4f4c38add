// Attention over the paged cache on the CUDA cores: fp32, and the bf16 shapes that
// the tensor-core kernel does not take.
//
// Online softmax over tiles of 64 keys: with the running maximum m and sum l of a
// row, a tile's scores x give m' = max(m, x), p = exp(x - m'), l = l exp(m - m') + sum p,
// o = o exp(m - m') + p v.  Rows are the query heads of one key/value head times tokens.
//
// Many rows (32 or 128 to a CTA): bound by the fp32 pipes.  16 lanes share a group of 4 or
// 8 rows; a lane has 4 keys' scores of each, in pairs of partial sums so that one
// instruction does two products, and the maximum is taken over the 16 lanes in
// registers.  Only a warp's own rows of weights go through shared memory, so the CTA
// meets twice a tile, when K and when V have landed; the next K loads during the softmax
// and the product with V, the next V during the next scores.
// Prompts of 2048 tokens, 32 heads of 128, 4 to a key/value head: 31 TFLOP/s of visible
// products (2.8 ms; 4 rows x 4 keys to a thread with the softmax through shared memory
// 3.9 ms), of about 74 that the pipes have: a lane's 12 reads of 16 bytes for 64
// instructions of products keep shared memory as busy as the pipes.
//
// Few rows (8): bound by the memory.  Each warp has 16 of a tile's 64 keys for itself, with
// a maximum, a sum and an o of its own, and loads them by itself: nothing waits for
// another warp until the four are joined at the end of a piece.  K and V leave shared memory
// once.
// 64 contexts of 8000, 8 key/value heads of 128, fp32: 5.3 TB/s (415 us; 510 us
// with the CTA's warps in step and K read by two groups of rows).
#include <math.h>

#include "attend_plan.cuh"
#include "pairs.cuh"
#include "serve.h"

namespace retrace {
namespace {

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

// What a CTA's rows of a piece are.
struct PieceRows {
  int kv_head, G, h0, rows;
};
__device__ __forceinline__ PieceRows piece_rows(const SimtParams& P, const Piece& pc) {
  const int kv_head = pc.head / P.splits, part = pc.head % P.splits, all = P.a.q_heads / P.a.cache.kv_heads;
  const int G = min(P.group, all - part * P.group);
  return PieceRows{kv_head, G, kv_head * all + part * P.group, (pc.i1 - pc.i0) * G};
}

// A key's place in the cache, -1: none, or seen by no row of the unit.
__device__ __forceinline__ long long key_place(const AttendArgs& a, const Piece& pc, int j) {
  if (j > pc.keys.hi || (j < pc.keys.lo && j >= a.sinks)) return -1;
  const int page = page_of(a.cache, pc.b, j / a.cache.page_size);
  return page < 0 ? -1 : page * a.cache.page_stride + (j % a.cache.page_size) * a.cache.slot_stride;
}

// Rows of D elements as fp32, zero beyond D, into rows of shared memory, by kThreads threads.
template <typename T, int DP, int kStride, int kThreads>
__device__ __forceinline__ void load_rows(float* dst, const T* base, const long long* off, int rows, int D, bool vec, int tid) {
  if (vec) {
    constexpr int N = 16 / sizeof(T), kChunks = DP / N;
    for (int i = tid; i < rows * kChunks; i += kThreads) {
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
  for (int i = tid; i < rows * DP; i += kThreads) {
    const int r = i / DP, c = i % DP;
    dst[r * kStride + c] = off[r] >= 0 && c < D ? to_f32(base[off[r] + c]) : 0.f;
  }
}

template <typename T, int DP, int kThreads>
__device__ __forceinline__ void load_queries(float (*q)[DP + 4], const AttendArgs& a, const Piece& pc, const PieceRows& w, int R) {
  const int D = a.cache.head_dim;
  for (int i = threadIdx.x; i < R * DP; i += kThreads) {
    const int r = i / DP, c = i % DP;
    float x = 0.f;
    if (r < w.rows && c < D)
      x = to_f32(static_cast<const T*>(a.q)[(long long)(pc.row0 + pc.i0 + r / w.G) * a.q_token + (w.h0 + r % w.G) * a.q_head + c]);
    q[r][c] = x;
  }
}

template <typename T>
__device__ __forceinline__ T* row_out(const AttendArgs& a, const Piece& pc, const PieceRows& w, int row) {
  return static_cast<T*>(a.out) + (long long)(pc.row0 + pc.i0 + row / w.G) * a.out_token + (w.h0 + row % w.G) * a.out_head;
}
__device__ __forceinline__ float max16(float x) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, o));
  return x;
}
__device__ __forceinline__ float sum16(float x) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
  return x;
}

// ---- many rows -----------------------------------------------------------------
template <int DP, int E>
struct ManyShape {
  // E rows to a thread: 8 lanes' groups of 4, 32 rows, or 16 groups of 8, 128 rows
  static constexpr int kThreads = E == 8 ? 256 : 128, kGroups = kThreads / 16, kRows = kGroups * E;
  struct Shared {
    float k[kKeys][DP + 4];  // + 4: 16-byte reads of consecutive rows fall into different banks
    float v[kKeys][DP];
    float q[kRows][DP + 4];
    float p[kRows][kKeys + 4];
    long long off[2][kKeys];
    long long sum[kThreads / 32];
    PlanStart plan;
  };
  static constexpr int kPerSm = E == 8 ? 1 : sizeof(Shared) <= 75 * 1024 ? 3 : sizeof(Shared) <= 113 * 1024 ? 2 : 1;
};

template <typename T, int DP, int E>
__global__ void __launch_bounds__(ManyShape<DP, E>::kThreads, ManyShape<DP, E>::kPerSm)
    attend_many_kernel(const __grid_constant__ SimtParams P) {
  using Sh = ManyShape<DP, E>;
  constexpr int kThreads = Sh::kThreads, R = Sh::kRows, kKeysEach = kKeys / 16;
  constexpr int kCols = DP / 16, kVec = kCols % 4 == 0 ? 4 : 2, kSteps = kCols / kVec;
  extern __shared__ __align__(16) unsigned char raw[];
  typename Sh::Shared& sm = *reinterpret_cast<typename Sh::Shared*>(raw);
  const AttendArgs& a = P.a;
  const int tid = threadIdx.x, D = a.cache.head_dim, rg = tid / 16, lane = tid % 16;
  pdl_launch_dependents();
  pdl_wait();
  plan_start<kThreads, kKeys>(P.shape, gridDim.x, 1, &sm.plan, sm.sum);
  const PlanStart plan = sm.plan;
  PieceWalk walk;
  walk.start(plan);
  // The two groups of a warp read rows 4 apart, which lie in different banks.
  auto row_of = [&](int r) { return (r & ~3) * Sh::kGroups + rg * 4 + (r & 3); };

  JoinUnit unit{};
  Piece pc;
  while (walk.next<kKeys, true>(P.shape, plan, &pc)) {
    const PieceRows w = piece_rows(P, pc);
    const T* kbase = static_cast<const T*>(a.cache.k) + w.kv_head * a.cache.head_stride;
    const T* vbase = static_cast<const T*>(a.cache.v) + w.kv_head * a.cache.head_stride;
    auto offsets = [&](int k) {  // of tile k of the piece
      if (tid < kKeys && k < pc.k1) sm.off[k & 1][tid] = key_place(a, pc, pc.keys.tile(k) * kKeys + tid);
    };
    auto load = [&](int k, bool values) {
      if (k < pc.k1) {
        if (values)
          load_rows<T, DP, DP, kThreads>(&sm.v[0][0], vbase, sm.off[k & 1], kKeys, D, P.vec, tid);
        else
          load_rows<T, DP, DP + 4, kThreads>(&sm.k[0][0], kbase, sm.off[k & 1], kKeys, D, P.vec, tid);
      }
      cp_async_commit();
    };

    __syncthreads();  // the previous piece's shared memory is free
    offsets(pc.k0);
    load_queries<T, DP, kThreads>(sm.q, a, pc, w, R);
    float2 acc[E][kCols / 2];
    float m[E], l[E];  // l: this lane's keys
#pragma unroll
    for (int r = 0; r < E; ++r) {
      m[r] = -INFINITY;
      l[r] = 0.f;
#pragma unroll
      for (int c = 0; c < kCols / 2; ++c) acc[r][c] = make_float2(0.f, 0.f);
    }
    __syncthreads();
    load(pc.k0, false);
    load(pc.k0, true);

    for (int k = pc.k0; k < pc.k1; ++k) {
      if (k == pc.k0)
        cp_async_wait<1>();  // K of this tile
      else
        cp_async_wait<0>();
      __syncthreads();  // and V of the tile before is free
      if (k > pc.k0) load(k, true);
      offsets(k + 1);
      float2 s[E][kKeysEach];
#pragma unroll
      for (int r = 0; r < E; ++r)
#pragma unroll
        for (int j = 0; j < kKeysEach; ++j) s[r][j] = make_float2(0.f, 0.f);
#pragma unroll 2
      for (int c = 0; c < DP; c += 4) {
        float4 x[kKeysEach];
#pragma unroll
        for (int j = 0; j < kKeysEach; ++j) x[j] = *reinterpret_cast<const float4*>(&sm.k[lane + j * 16][c]);
#pragma unroll
        for (int r = 0; r < E; ++r) {
          const float4 q = *reinterpret_cast<const float4*>(&sm.q[row_of(r)][c]);
#pragma unroll
          for (int j = 0; j < kKeysEach; ++j) {
            s[r][j] = fma2(make_float2(q.x, q.y), make_float2(x[j].x, x[j].y), s[r][j]);
            s[r][j] = fma2(make_float2(q.z, q.w), make_float2(x[j].z, x[j].w), s[r][j]);
          }
        }
      }
      // What a row does not see is replaced, not added to: its bits may be anything.
      const int j0 = pc.keys.tile(k) * kKeys;
      bool there[kKeysEach];
#pragma unroll
      for (int j = 0; j < kKeysEach; ++j) there[j] = sm.off[k & 1][lane + j * 16] >= 0;
#pragma unroll
      for (int r = 0; r < E; ++r) {
        const int row = row_of(r), at = pc.c + pc.i0 + row / w.G;
        const int hi = a.causal ? at : pc.c + pc.n - 1, lo = a.window > 0 ? at - a.window + 1 : 0;
        float x[kKeysEach], top = -INFINITY;
#pragma unroll
        for (int j = 0; j < kKeysEach; ++j) {
          const int key = j0 + lane + j * 16;
          const bool seen = there[j] && key <= hi && (key >= lo || key < a.sinks);
          x[j] = seen ? (s[r][j].x + s[r][j].y) * a.scale : -INFINITY;
          top = fmaxf(top, x[j]);
        }
        const float up = fmaxf(m[r], max16(top)), ref = up == -INFINITY ? 0.f : up, f = expf(m[r] - ref);
        m[r] = up;
        l[r] *= f;
#pragma unroll
        for (int j = 0; j < kKeysEach; ++j) {
          const float e = expf(x[j] - ref);
          l[r] += e;
          sm.p[row][lane + j * 16] = e;
        }
#pragma unroll
        for (int c = 0; c < kCols / 2; ++c) acc[r][c] = mul2(acc[r][c], make_float2(f, f));
      }
      cp_async_wait<0>();  // V of this tile
      __syncthreads();     // and K is free
      load(k + 1, false);
#pragma unroll 2
      for (int j = 0; j < kKeys; j += 4) {
        float4 e[E];
#pragma unroll
        for (int r = 0; r < E; ++r) e[r] = *reinterpret_cast<const float4*>(&sm.p[row_of(r)][j]);
#pragma unroll
        for (int jj = 0; jj < 4; ++jj) {
          float2 x[kCols / 2];
#pragma unroll
          for (int c = 0; c < kSteps; ++c) {
            const float* from = &sm.v[j + jj][(lane + c * 16) * kVec];
            if constexpr (kVec == 4) {
              const float4 y = *reinterpret_cast<const float4*>(from);
              x[c * 2] = make_float2(y.x, y.y);
              x[c * 2 + 1] = make_float2(y.z, y.w);
            } else {
              x[c] = *reinterpret_cast<const float2*>(from);
            }
          }
#pragma unroll
          for (int r = 0; r < E; ++r) {
            const float ee = jj == 0 ? e[r].x : jj == 1 ? e[r].y : jj == 2 ? e[r].z : e[r].w;
#pragma unroll
            for (int c = 0; c < kCols / 2; ++c) acc[r][c] = fma2(make_float2(ee, ee), x[c], acc[r][c]);
          }
        }
      }
    }

    const bool whole = pc.pieces == 1;
    constexpr int kPart = R * (DP + 2);
    float* part = a.partials + ((long long)blockIdx.x * 2 + (pc.k0 == 0 ? 1 : 0)) * kPart;
#pragma unroll
    for (int r = 0; r < E; ++r) {
      const int row = row_of(r);
      const float sum = sum16(l[r]), inv = sum == 0.f ? 0.f : 1.f / sum;
      if (whole) {
        if (row >= w.rows) continue;
        T* out = row_out<T>(a, pc, w, row);
#pragma unroll
        for (int c = 0; c < kCols; ++c) {
          const int col = (lane + c / kVec * 16) * kVec + c % kVec;
          if (col < D) out[col] = from_f32<T>((c % 2 ? acc[r][c / 2].y : acc[r][c / 2].x) * inv);
        }
      } else {  // a part of a unit: rows, maxima and sums to the workspace
#pragma unroll
        for (int c = 0; c < kCols / 2; ++c)
          *reinterpret_cast<float2*>(part + row * DP + (lane + c * 2 / kVec * 16) * kVec + c * 2 % kVec) = acc[r][c];
        if (lane == 0) *reinterpret_cast<float2*>(part + R * DP + row * 2) = make_float2(m[r], sum);
      }
    }
    if (!whole && pc.k0 == 0) unit = JoinUnit{pc.pieces, w.rows, w.rows, pc.row0 + pc.i0, w.h0, w.G, {0, 0}};
  }
  if (tid == 0) a.units[blockIdx.x] = unit;
}

// ---- few rows ------------------------------------------------------------------
template <int DP>
struct FewShape {
  static constexpr int kThreads = 128, kWarps = 4, kRows = 8, kMine = kKeys / kWarps;
  struct Shared {
    float k[kWarps][kMine][DP + 4];  // a warp's keys; at the end its o
    float v[kWarps][kMine][DP];
    float q[kRows][DP + 4];
    float p[kWarps][kRows][kMine + 4];
    float2 stat[kWarps][kRows];  // a warp's maxima and sums
    long long off[kWarps][2][kMine];
    long long sum[kWarps];
    PlanStart plan;
  };
  static constexpr int kPerSm = sizeof(Shared) <= 75 * 1024 ? 3 : 1;
};

template <typename T, int DP>
__global__ void __launch_bounds__(FewShape<DP>::kThreads, FewShape<DP>::kPerSm) attend_few_kernel(const __grid_constant__ SimtParams P) {
  using Sh = FewShape<DP>;
  constexpr int kThreads = Sh::kThreads, R = Sh::kRows, kMine = Sh::kMine, kWarps = Sh::kWarps;
  constexpr int kCols = DP / 32, kVec = kCols % 4 == 0 ? 4 : kCols % 2 == 0 ? 2 : 1, kSteps = kCols / kVec;
  extern __shared__ __align__(16) unsigned char raw[];
  typename Sh::Shared& sm = *reinterpret_cast<typename Sh::Shared*>(raw);
  const AttendArgs& a = P.a;
  const int tid = threadIdx.x, D = a.cache.head_dim, warp = tid / 32, lane = tid % 32;
  const int half = lane / 16, mine = lane % 16;  // of the scores: rows 4 half .. + 3, key `mine` of the warp
  pdl_launch_dependents();
  pdl_wait();
  plan_start<kThreads, kKeys>(P.shape, gridDim.x, 1, &sm.plan, sm.sum);
  const PlanStart plan = sm.plan;
  PieceWalk walk;
  walk.start(plan);

  JoinUnit unit{};
  Piece pc;
  while (walk.next<kKeys, true>(P.shape, plan, &pc)) {
    const PieceRows w = piece_rows(P, pc);
    const T* kbase = static_cast<const T*>(a.cache.k) + w.kv_head * a.cache.head_stride;
    const T* vbase = static_cast<const T*>(a.cache.v) + w.kv_head * a.cache.head_stride;
    auto offsets = [&](int k) {
      if (lane < kMine && k < pc.k1) sm.off[warp][k & 1][lane] = key_place(a, pc, pc.keys.tile(k) * kKeys + warp * kMine + lane);
      __syncwarp();
    };
    auto load = [&](int k, bool values) {
      if (k < pc.k1) {
        if (values)
          load_rows<T, DP, DP, 32>(&sm.v[warp][0][0], vbase, sm.off[warp][k & 1], kMine, D, P.vec, lane);
        else
          load_rows<T, DP, DP + 4, 32>(&sm.k[warp][0][0], kbase, sm.off[warp][k & 1], kMine, D, P.vec, lane);
      }
      cp_async_commit();
    };

    __syncthreads();  // the previous piece's shared memory is free
    offsets(pc.k0);
    load(pc.k0, false);
    load(pc.k0, true);
    load_queries<T, DP, kThreads>(sm.q, a, pc, w, R);
    float acc[R][kCols], m[4], l[4];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int c = 0; c < kCols; ++c) acc[r][c] = 0.f;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      m[r] = -INFINITY;
      l[r] = 0.f;
    }
    __syncthreads();

    for (int k = pc.k0; k < pc.k1; ++k) {
      offsets(k + 1);
      cp_async_wait<1>();  // K of this tile
      __syncwarp();
      float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
      for (int c = 0; c < DP; c += 4) {
        const float4 x = *reinterpret_cast<const float4*>(&sm.k[warp][mine][c]);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float4 q = *reinterpret_cast<const float4*>(&sm.q[half * 4 + r][c]);
          s[r] = fmaf(q.x, x.x, fmaf(q.y, x.y, fmaf(q.z, x.z, fmaf(q.w, x.w, s[r]))));
        }
      }
      const int key = pc.keys.tile(k) * kKeys + warp * kMine + mine;
      const bool there = sm.off[warp][k & 1][mine] >= 0;
      __syncwarp();  // K is free
      load(k + 1, false);
      float f[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = half * 4 + r, at = pc.c + pc.i0 + row / w.G;
        const int hi = a.causal ? at : pc.c + pc.n - 1, lo = a.window > 0 ? at - a.window + 1 : 0;
        // What a row does not see is replaced, not added to: its bits may be anything.
        const bool seen = there && key <= hi && (key >= lo || key < a.sinks);
        const float x = seen ? s[r] * a.scale : -INFINITY;
        const float up = fmaxf(m[r], max16(x)), ref = up == -INFINITY ? 0.f : up;
        f[r] = expf(m[r] - ref);
        m[r] = up;
        const float e = expf(x - ref);
        l[r] = l[r] * f[r] + e;
        sm.p[warp][row][mine] = e;
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float other = __shfl_xor_sync(0xFFFFFFFFu, f[r], 16), f0 = half ? other : f[r], f1 = half ? f[r] : other;
#pragma unroll
        for (int c = 0; c < kCols; ++c) {
          acc[r][c] *= f0;
          acc[4 + r][c] *= f1;
        }
      }
      cp_async_wait<1>();  // V of this tile
      __syncwarp();
#pragma unroll
      for (int j = 0; j < kMine; j += 4) {
        float4 e[R];
#pragma unroll
        for (int r = 0; r < R; ++r) e[r] = *reinterpret_cast<const float4*>(&sm.p[warp][r][j]);
#pragma unroll
        for (int jj = 0; jj < 4; ++jj) {
          float x[kCols];
#pragma unroll
          for (int c = 0; c < kSteps; ++c) {
            const float* from = &sm.v[warp][j + jj][(lane + c * 32) * kVec];
            if constexpr (kVec == 4)
              *reinterpret_cast<float4*>(&x[c * 4]) = *reinterpret_cast<const float4*>(from);
            else if constexpr (kVec == 2)
              *reinterpret_cast<float2*>(&x[c * 2]) = *reinterpret_cast<const float2*>(from);
            else
              x[c] = *from;
          }
#pragma unroll
          for (int r = 0; r < R; ++r) {
            const float ee = jj == 0 ? e[r].x : jj == 1 ? e[r].y : jj == 2 ? e[r].z : e[r].w;
#pragma unroll
            for (int c = 0; c < kCols; ++c) acc[r][c] = fmaf(ee, x[c], acc[r][c]);
          }
        }
      }
      __syncwarp();  // V and the weights are free
      load(k + 1, true);
    }
    cp_async_wait<0>();

    // The four warps' parts, over their keys' shared memory.
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float sum = sum16(l[r]);
      if (mine == 0) sm.stat[warp][half * 4 + r] = make_float2(m[r], sum);
    }
    __syncwarp();
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int c = 0; c < kCols; ++c) sm.k[warp][r][(lane + c / kVec * 32) * kVec + c % kVec] = acc[r][c];
    __syncthreads();
    const bool whole = pc.pieces == 1;
    constexpr int kPart = R * (DP + 2);
    float* part = a.partials + ((long long)blockIdx.x * 2 + (pc.k0 == 0 ? 1 : 0)) * kPart;
    for (int i = tid; i < R * DP; i += kThreads) {
      const int row = i / DP, col = i % DP;
      if (row >= w.rows) break;
      float top = -INFINITY, sum = 0.f, o = 0.f;
#pragma unroll
      for (int x = 0; x < kWarps; ++x) top = fmaxf(top, sm.stat[x][row].x);
#pragma unroll
      for (int x = 0; x < kWarps; ++x) {
        const float2 st = sm.stat[x][row];
        const float g = st.x == -INFINITY ? 0.f : expf(st.x - top);
        sum += st.y * g;
        o += st.x == -INFINITY ? 0.f : sm.k[x][row][col] * g;
      }
      if (whole) {
        if (col < D) row_out<T>(a, pc, w, row)[col] = from_f32<T>(sum == 0.f ? 0.f : o / sum);
      } else {
        part[i] = o;
        if (col == 0) *reinterpret_cast<float2*>(part + R * DP + row * 2) = make_float2(top, sum);
      }
    }
    if (!whole && pc.k0 == 0) unit = JoinUnit{pc.pieces, w.rows, w.rows, pc.row0 + pc.i0, w.h0, w.G, {0, 0}};
  }
  if (tid == 0) a.units[blockIdx.x] = unit;
}

// ---- launches ------------------------------------------------------------------
// A workspace has room for the parts of 192 CTAs of 128 rows.
constexpr int kMaxManyCtas = 192;

template <typename Sh, typename K>
cudaError_t launch(K kernel, SimtParams& p, int DP, cudaStream_t stream, std::atomic<uint64_t>& allowed) {
  constexpr int R = Sh::kRows, most = R == 128 ? kMaxManyCtas : kAttendMaxCtas;
  constexpr size_t smem = sizeof(typename Sh::Shared);
  static_assert(smem <= 227 * 1024, "shared memory of a CTA");
  DeviceInfo dev;
  cudaError_t e = device_info(&dev);
  if (e != cudaSuccess) return e;
  if ((e = allow_shared(kernel, smem, dev, allowed)) != cudaSuccess) return e;
  const int ctas = dev.sm_count * Sh::kPerSm, grid = ctas < most ? ctas : most, heads = p.a.q_heads / p.a.cache.kv_heads;
  p.splits = (heads + R - 1) / R;
  p.group = (heads + p.splits - 1) / p.splits;
  p.shape.kv_heads = p.a.cache.kv_heads * p.splits;
  p.shape.unit_tokens = R / p.group;
  if ((e = launch_dependent(kernel, dim3(grid), dim3(Sh::kThreads), smem, stream, 1u, p)) != cudaSuccess) return e;
  return launch_attend_join(p.a, PartShape{R, DP, 0.f}, grid, stream);
}

template <typename T, int DP, int E>
cudaError_t launch_many(SimtParams& p, cudaStream_t stream) {
  static std::atomic<uint64_t> allowed{0};
  return launch<ManyShape<DP, E>>(attend_many_kernel<T, DP, E>, p, DP, stream, allowed);
}
template <typename T, int DP>
cudaError_t launch_few(SimtParams& p, cudaStream_t stream) {
  static std::atomic<uint64_t> allowed{0};
  return launch<FewShape<DP>>(attend_few_kernel<T, DP>, p, DP, stream, allowed);
}

template <typename T, int DP>
cudaError_t launch_rows(SimtParams& p, cudaStream_t stream) {
  // By the rows that a sequence has on average.  128 rows cost four times what 32 do and less
  // in the end from two thirds of them on: contexts of 2000, 8 heads of 128, 64 / 96 / 128 rows a
  // sequence: in units of 32 1583 / 2257 / 2997 us before the softmax left shared memory, in units
  // of 128 2088 us at 96 and 2240 at 128; at 64 two units of 32 take 1383.
  const long long rows = (long long)p.a.T * (p.a.q_heads / p.a.cache.kv_heads);
  if (rows <= 8ll * p.a.B) return launch_few<T, DP>(p, stream);
  if constexpr (DP <= 128)
    if (rows > 64ll * p.a.B) return launch_many<T, DP, 8>(p, stream);
  return launch_many<T, DP, 4>(p, stream);
}

template <typename T>
cudaError_t launch_typed(SimtParams& p, cudaStream_t stream) {
  const int D = p.a.cache.head_dim;
  return D <= 64   ? launch_rows<T, 64>(p, stream)
         : D <= 96 ? launch_rows<T, 96>(p, stream)
         : D <= 128 ? launch_rows<T, 128>(p, stream)
                    : launch_rows<T, 256>(p, stream);
}

}  // namespace

size_t attend_simt_partial_bytes(int head_dim) {
  const size_t DP = head_dim <= 64 ? 64 : head_dim <= 96 ? 96 : head_dim <= 128 ? 128 : 256;
  const size_t rows = DP <= 128 ? (size_t)kMaxManyCtas * 128 : (size_t)kAttendMaxCtas * 32;
  static_assert(kMaxManyCtas * 128 >= kAttendMaxCtas * 32, "room for either kernel's parts");
  return rows * 2 * (DP + 2) * 4;
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
