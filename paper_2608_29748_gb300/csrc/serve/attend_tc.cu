// Attention over the paged cache on the tensor cores (bf16).
//
// A row is a query token under one query head; the rows of a tile (128, a TMEM lane
// each) share a key/value head.  Per tile of 128 keys a stream computes
//     S = Q K^T        tcgen05.mma, Q and K from shared memory, S in TMEM (fp32)
//     m, p, l          one thread per row: running maximum, p = 2^(s - m), running sum
//     O += P V         tcgen05.mma, P (bf16) from TMEM over S's columns, V from shared
//                      memory as it lies (keys by head dimension), O in TMEM (fp32)
// A CTA runs two streams, so that one's matrix products run during the other's softmax:
// two row tiles over the same key tiles where a unit has more than 128 rows (prompts),
// or the even and the odd key tiles of one row tile (tokens, blocks), joined at the end.
// The maximum that the exponents refer to is the first tile's, and is raised, and O rescaled,
// only where the weights of a row in a tile pass 2^14.
//
// Warps 0 and 2 copy the K and the V tiles into a ring with TMA, a box for each run of
// slots within a page (a warp issues a box in about 120 cycles, so one warp for both was
// the bound with pages of 16); warps 1 and 3 issue the streams' products; warps 4-7 and
// 8-11 are their softmax.
// A tile of keys is 4 D 128 bytes of HBM traffic against 2 x 128 x 128 x D products of a
// tensor core that does 8192 flop a cycle: 1024 of the 2790 cycles that the bytes take
// at D = 128, so tokens and blocks are bound by HBM, and a row tile that is not full costs
// nothing: 64 blocks of 17 tokens over up to 8192, 8 heads of 128, 5.5 TB/s (221 us).  Prompts are
// bound by the chain of products and softmax: four of up to 4096 tokens, 32 heads, 794 TFLOP/s (359 us),
// the tensor core busy for about half of the time (a softmax of 128 x 128 is some 2000
// cycles of its warpgroup, each product 512).  One token over 2048 keys is latency: 18 us with
// the joining kernel.
#include <math.h>

#include "../tc_pair.cuh"
#include "attend_plan.cuh"
#include "pairs.cuh"
#include "serve.h"
#include "tc_ops.cuh"

namespace retrace {
namespace {

constexpr int kThreads = 384;
constexpr int kKeys = 128;  // keys of a tile
constexpr int kRows = 128;  // rows of a tile
constexpr unsigned long long kDrainNs = 20ull * 1000ull * 1000ull;
constexpr int kJoinRows = 32;  // most rows of a unit whose last CTA joins its parts (see `join`)
constexpr float kFar = 8192.f;  // of a reference's exponent (see the softmax)
constexpr int kMasks = 16;  // ring of page masks: more than the tiles between loading and softmax

struct TcParams {
  AttendArgs a;
  AttendShape shape;  // unit_tokens = 2 tile_tokens
  int group;          // query heads of a key/value head
  int tile_tokens;    // tokens of a row tile
  int q_box;          // tokens of a Q box
  FastDivide page_size;
  int kv_box;         // slots of a K or V box: they lie within a page and divide a tile
  float scale2;       // |scale| log2(e)
  int negate;         // scale < 0
  int join;           // parts are joined by the last CTA of a unit, else by a second kernel
};

template <int DP>
struct TcShape {
  static constexpr int kTileBytes = kKeys * DP * 2;
  // K and V tiles have rings of their own, each filled by one warp.  A tile of K is free after
  // its scores, one of V only after the softmax, so V has the odd one.
  static constexpr int kRingK = DP == 64 ? 5 : 2, kRingV = DP == 64 ? 5 : 3;
  static constexpr int kHalves = DP / 64;              // 128-byte columns of a tile
  static constexpr int kHalfBytes = kKeys * 128;
  static constexpr int kVOffset = kRingK * kTileBytes, kQOffset = kVOffset + kRingV * kTileBytes;
  static constexpr int kControl = kQOffset + 2 * kRows * DP * 2;
  static constexpr int kPartRows = 2 * kRows;
  static constexpr int kPart = kPartRows * (DP + 2);  // floats of a part
};

struct Control {
  // A ring's slots.  A wait for a phase by its parity is right only for one who has seen the
  // phase before, so a slot has a `full` barrier per class of tiles (of stream 0, of stream
  // 1, of both), every use of which its waiters see.
  struct Ring {
    uint64_t full[3][5], empty[5];
  } ring[2];  // K, V
  uint64_t q_full[2], q_empty[2];
  uint64_t s_full[2];  // of a stream: S ready and the product with V before it done
  uint64_t p_full[2];  // P written, O rescaled
  // O complete.  Not a phase of s_full: the next piece's first scores follow it with no p_full
  // between them, so that one would complete twice while its waiter is still at the first.  The
  // commits to s_full lie a p_full apart, and those to o_full a piece's p_full, which the softmax
  // gives only after it has seen the phase before.
  uint64_t o_full[2];
  uint64_t issued[2];  // two row tiles: a stream's products of a tile are on their way
  uint64_t done[2];    // after an expired wait: the issued products
  PlanStart plan;
  long long sum[kThreads / 32];
  uint32_t tmem;
  int abort, last;
  PieceWalk walk[2];  // of the softmax streams
  Piece piece[2][2];  // this one and the next
  int more[2][2];
  uint32_t mask[kMasks];  // of a key tile: bit i: box i has a page
  float2 stat[2][kRows];  // m and l of a stream's rows
};

// D[tmem] (+)= A[tmem] * B[smem], bf16 inputs, fp32 accumulation.
__device__ __forceinline__ void tc_mma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc,
                                               uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
      "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// Moves registers from the warpgroup of the copies and products to those of the softmax:
// 128 x 88 + 256 x 208 are the 384 x 168 of the launch.
__device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 88;"); }
__device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 208;"); }
// The four warps of a stream.
__device__ __forceinline__ void stream_barrier(int s) {
  if (s == 0)
    named_barrier<2, kRows>();
  else
    named_barrier<3, kRows>();
}

// Descriptor of V [keys, 64-element columns] as the MN-major operand: rows of 128
// bytes with the 128-byte swizzle; 64-element blocks of the head dimension 16 KB apart
// (leading offset), groups of 8 keys 1024 bytes apart (stride offset).
__device__ __forceinline__ uint64_t sw128_mnmajor_desc(uint32_t saddr) {
  return (uint64_t)((saddr & 0x3FFFFu) >> 4) | (uint64_t)((kKeys * 128) >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 |
         (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
constexpr uint32_t kMajorB = 1u << 16;  // instruction descriptor: B is MN-major

// Bits c of a word of 32 keys: key c is visible iff c <= hi and (c >= lo or c < sinks).
__device__ __forceinline__ uint32_t seen_word(int hi, int lo, int sinks) {
  const uint32_t h = hi < 0 ? 0u : hi >= 31 ? ~0u : (2u << hi) - 1u;
  const uint32_t l = lo <= 0 ? ~0u : lo >= 32 ? 0u : ~0u << lo;
  const uint32_t k = sinks <= 0 ? 0u : sinks >= 32 ? ~0u : (1u << sinks) - 1u;
  return h & (l | k);
}
// Bits of the keys of word w that have a page, from a bit per box of `box` keys.
__device__ __forceinline__ uint32_t page_word(uint32_t boxes, int box, int w) {
  if (box >= 32) return boxes >> (w * 32 / box) & 1u ? ~0u : 0u;
  uint32_t x = 0;
  const uint32_t ones = (1u << box) - 1u;
  for (int i = 0; i < 32 / box; ++i)
    if (boxes >> (w * (32 / box) + i) & 1u) x |= ones << (i * box);
  return x;
}
__device__ __forceinline__ uint32_t boxes_mask(int boxes) { return (1u << boxes) - 1u; }

template <int DP>
__global__ void __launch_bounds__(kThreads, 1)
    attend_tc_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                     const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ TcParams P) {
  using Sh = TcShape<DP>;
  extern __shared__ __align__(1024) uint8_t smem[];
  Control& ct = *reinterpret_cast<Control*>(smem + Sh::kControl);
  volatile int* abort = &ct.abort;
  const uint32_t base = smem_u32(smem);
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  const AttendArgs& a = P.a;

  if (tid == 0) {
    ct.abort = 0;
    // A tile of a ring is free when both streams are through with it; where only one of them
    // uses it, the copying warp counts for the other.
    for (int r = 0; r < 2; ++r)
      for (int s = 0; s < 5; ++s) {
        for (int c = 0; c < 3; ++c) mbar_init(smem_u32(&ct.ring[r].full[c][s]), 1);
        mbar_init(smem_u32(&ct.ring[r].empty[s]), 2);
      }
    for (int s = 0; s < 2; ++s) {
      mbar_init(smem_u32(&ct.q_full[s]), 1);
      mbar_init(smem_u32(&ct.q_empty[s]), 2);  // both streams
      mbar_init(smem_u32(&ct.s_full[s]), 1);
      mbar_init(smem_u32(&ct.p_full[s]), 4);  // one arrival per warp of the stream
      mbar_init(smem_u32(&ct.o_full[s]), 1);
      mbar_init(smem_u32(&ct.issued[s]), 1);
      mbar_init(smem_u32(&ct.done[s]), 1);
    }
    fence_mbar_init();
    tma_prefetch_desc(&tm_q);
    tma_prefetch_desc(&tm_k);
    tma_prefetch_desc(&tm_v);
  }
  if (warp == 2) {
    tmem_alloc(smem_u32(&ct.tmem), 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = ct.tmem;
  pdl_launch_dependents();
  pdl_wait();
  plan_start<kThreads, kKeys>(P.shape, gridDim.x, 2, &ct.plan, ct.sum);
  const PlanStart& plan = ct.plan;
  if (warp < 4) {
    fewer_registers();
    PieceWalk walk;
    walk.start(plan);
    Piece pc;
    bool drain = false;
    if (warp == 0 || warp == 2) {
      // ---- copies of K (warp 0), and of Q and V (warp 2) ----
      const bool keys = warp == 0;
      const CUtensorMap* map = keys ? &tm_k : &tm_v;
      // lane (half, box) loads one box of a tile
      const int boxes = kKeys / P.kv_box, half = lane / 16, box = lane % 16;
      const bool active = box < boxes && half < Sh::kHalves;
      const int box_rows = P.q_box * P.group;
      Control::Ring& ring = ct.ring[keys ? 0 : 1];
      const uint32_t slots = keys ? Sh::kRingK : Sh::kRingV, tiles_at = base + (keys ? 0 : Sh::kVOffset);
      uint32_t tiles = 0, slot = 0, phase = 0, used[2] = {0, 0};
      int turn = 0;
      bool ok = true;
      while (ok && walk.next<kKeys>(P.shape, plan, &pc)) {
        const int nt = pc.k1 - pc.k0, tokens = pc.i1 - pc.i0;
        if (nt == 0) continue;
        const bool two = tokens > P.tile_tokens;
        struct Place {
          int page, slot;
        };
        auto place_of = [&](int k) {  // of this lane's box of the piece's tile k
          Place x{a.cache.num_pages, 0};  // a box without a page lies outside the tensor: zeros
          if (active && k < nt) {
            const int j = pc.keys.tile(pc.k0 + k) * kKeys + box * P.kv_box, i = P.page_size(j);
            const int page = page_of(a.cache, pc.b, i);
            if (page >= 0) x = Place{page, j - i * P.page_size.by};
          }
          return x;
        };
        // looked up two tiles ahead of their copies
        Place now = place_of(0), next = place_of(1);
        if (!keys) {
          // Q: boxes of q_box tokens times the head group, rows in order.  A unit of two row
          // tiles takes both buffers, one of one tile the other one than before.
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            if (!ok || (!two && q != turn)) continue;
            const int t0 = two ? q * P.tile_tokens : 0, n = min(tokens - t0, P.tile_tokens);
            const int q_boxes = (n + P.q_box - 1) / P.q_box;
            ok = warp_wait_all(&ct.q_empty[q], (used[q] & 1u) ^ 1u, abort);
            if (!ok) continue;
            ++used[q];
            const uint32_t bar = smem_u32(&ct.q_full[q]);
            if (lane == 0) mbar_arrive_expect_tx(bar, q_boxes * Sh::kHalves * box_rows * 128);
            __syncwarp();
            for (int i = lane; i < q_boxes * Sh::kHalves; i += 32) {
              const int h = i % Sh::kHalves, x = i / Sh::kHalves;
              tma_load_3d(base + Sh::kQOffset + q * (kRows * DP * 2) + h * Sh::kHalfBytes + x * box_rows * 128, &tm_q, h * 64,
                          pc.head * P.group, pc.row0 + pc.i0 + t0 + x * P.q_box, bar);
            }
          }
          if (!two) turn ^= 1;
        }
        for (int k = 0; k < nt && ok; ++k) {
          const Place after = place_of(k + 2);
          ok = warp_wait_all(&ring.empty[slot], phase ^ 1u, abort);
          if (!ok) break;
          const uint32_t bar = smem_u32(&ring.full[two ? 2 : k & 1][slot]);
          const uint32_t placed = __ballot_sync(0xFFFFFFFFu, active && half == 0 && now.page < a.cache.num_pages);
          if (lane == 0) {
            if (!two) mbar_arrive(smem_u32(&ring.empty[slot]));
            if (keys) ct.mask[tiles % kMasks] = placed;
            mbar_arrive_expect_tx(bar, Sh::kTileBytes);
          }
          __syncwarp();
          if (active)
            tma_load_4d(tiles_at + slot * Sh::kTileBytes + half * Sh::kHalfBytes + box * P.kv_box * 128, map, half * 64, pc.head,
                        now.slot, now.page, bar);
          if (++slot == slots) {
            slot = 0;
            phase ^= 1u;
          }
          ++tiles;
          now = next;
          next = after;
        }
      }
      if (!ok) {
        if (lane == 0) raise_abort(abort, a.status);
        drain = true;
      }
    } else {
      // ---- products of stream s (warps 1 and 3) ----
      constexpr uint32_t kS = idesc_bf16_f32(kRows, kKeys), kPV = idesc_bf16_f32(kRows, DP) | kMajorB;
      const int s = warp >> 1;
      const uint32_t t_s = tmem + s * 128, t_o = tmem + 256 + s * 128;
      uint32_t tiles = 0, used[2] = {0, 0}, np = 0;
      int turn = 0;
      bool ok = true;
      auto wait = [&](uint64_t* bar, uint32_t parity) {
        ok = ok && warp_wait_all(bar, parity, abort);
        return ok;
      };
      uint32_t phases = 0;  // a bit per slot, tiles of this stream or of both, ring
      auto wait_tile = [&](int ring, uint32_t slot, bool two) {
        const uint32_t bit = 1u << (ring * 16 + two * 8 + slot);
        const bool landed = wait(&ct.ring[ring].full[two ? 2 : s][slot], (phases & bit) != 0);
        phases ^= bit;
        return landed;
      };
      auto commit = [&](uint64_t* bar) {
        if (elect_one()) tc_commit(smem_u32(bar));
        __syncwarp();
      };
      auto scores = [&](int q, uint32_t slot) {
        if (elect_one()) {
          const uint64_t qd = sw128_kmajor_desc(base + Sh::kQOffset + q * (kRows * DP * 2));
          const uint64_t kd = sw128_kmajor_desc(base + slot * Sh::kTileBytes);
#pragma unroll
          for (int h = 0; h < Sh::kHalves; ++h)
#pragma unroll
            for (int k = 0; k < 4; ++k)
              tc_mma_bf16(t_s, qd + h * (Sh::kHalfBytes >> 4) + 2 * k, kd + h * (Sh::kHalfBytes >> 4) + 2 * k, kS, h + k > 0);
        }
        __syncwarp();
      };
      // The product of P with a tile of V, which is free after it.
      auto values = [&](uint32_t slot, bool first) {
        tc_fence_after();
        if (elect_one()) {
          const uint64_t vd = sw128_mnmajor_desc(base + Sh::kVOffset + slot * Sh::kTileBytes);
#pragma unroll
          for (int k = 0; k < kKeys / 16; ++k)
            tc_mma_bf16_ts(t_o, t_s + k * 8, vd + k * (2048 >> 4), kPV, !(first && k == 0));
        }
        __syncwarp();
        commit(&ct.ring[1].empty[slot]);
      };
      struct Work {  // of a piece: what the products need of it, looked up a piece ahead
        int nt, two, k0;
        UnitKeys keys;
      };
      bool more = true;
      auto next_work = [&]() {
        Work w{};
        do {
          more = walk.next<kKeys>(P.shape, plan, &pc);
          if (more) w = Work{pc.k1 - pc.k0, pc.i1 - pc.i0 > P.tile_tokens, pc.k0, pc.keys};
        } while (more && w.nt == 0);
        return w;
      };
      uint32_t batches = 0;
      Work next = next_work();
      while (ok && more) {
        const Work w = next;
        const int nt = w.nt;
        const bool two = w.two;
        const int q = two ? s : turn, step = two ? 1 : 2;
        const int first = two ? 0 : s;  // of this stream's tiles: first, first + step, ...
        if (!wait(&ct.q_full[q], used[q]++ & 1u)) break;
        if (two && !wait(&ct.q_full[q ^ 1], used[q ^ 1]++ & 1u)) break;
        if (two && lane == 0) mbar_arrive(smem_u32(&ct.q_empty[q ^ 1]));  // the other stream's
        if (!two) turn ^= 1;
        tc_fence_after();
        int j = first;
        bool landed = false;  // V of the tile before
        for (; j < nt; j += step) {
          const uint32_t k = (tiles + j) % Sh::kRingK, v = (tiles + j) % Sh::kRingV, before = (tiles + j - step) % Sh::kRingV;
          if (!wait_tile(0, k, two)) break;
          if (j > first && !landed && !wait_tile(1, before, two)) break;
          // With two row tiles the streams issue in turn: products that are issued together
          // share the tensor core and end together, and then it waits for both softmaxes.
          if (two && (s == 1 || batches > 0) && !wait(&ct.issued[s ^ 1], (s == 1 ? batches : batches - 1) & 1u)) break;
          if (j > first && !wait(&ct.p_full[s], np++ & 1u)) break;
          if (j > first) values(before, j == first + step);
          // V of a tile at the edge of what the unit sees is there before its scores are: the
          // softmax clears rows of it
          const int j0 = w.keys.tile(w.k0 + j) * kKeys;
          landed = j0 < w.keys.lo || j0 + kKeys - 1 > w.keys.hi;
          if (landed && !wait_tile(1, v, two)) break;
          tc_fence_after();
          scores(q, k);
          if (two) {
            if (lane == 0) mbar_arrive(smem_u32(&ct.issued[s]));
            ++batches;
          }
          commit(&ct.s_full[s]);
          commit(&ct.ring[0].empty[k]);
          if (j == first) next = next_work();
        }
        if (!ok) break;
        if (j > first) {
          commit(&ct.q_empty[q]);
          const uint32_t before = (tiles + j - step) % Sh::kRingV;
          if ((!landed && !wait_tile(1, before, two)) || !wait(&ct.p_full[s], np++ & 1u)) break;
          values(before, j == first + step);
          commit(&ct.o_full[s]);
        } else {
          if (lane == 0) mbar_arrive(smem_u32(&ct.q_empty[q]));  // no tile for this stream
          next = next_work();
        }
        tiles += nt;
      }
      if (!ok) {
        if (lane == 0) raise_abort(abort, a.status);
        volatile int never = 0;
        commit(&ct.done[s]);
        mbar_wait_bounded(smem_u32(&ct.done[s]), 0, &never);
      }
    }
    // After an expired wait: time for this CTA's copies in flight to land.
    if (drain) {
      const unsigned long long t0 = global_ns();
      while (global_ns() - t0 < kDrainNs) __nanosleep(1000);
    }
    __syncwarp();
  } else {
    more_registers();
    // ---- softmax: stream s, one thread per row ----
    const int s = warp >= 8, row = tid & 127;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t t_s = tmem + lanes + s * 128, t_o = tmem + lanes + 256 + s * 128;
    const int G = P.group, D = a.cache.head_dim;
    const float sl = P.scale2;
    const uint32_t all_boxes = boxes_mask(kKeys / P.kv_box);
    uint32_t ns = 0, no = 0, tiles = 0;
    JoinUnit unit{};
    bool ok = true;
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      if (ok && !warp_wait_all(bar, parity, abort)) {
        ok = false;
        if (lane == 0) raise_abort(abort, a.status);
      }
    };
    // The part of a unit of few rows is written: the last CTA of the unit to come here joins
    // the parts, in the order of the CTAs' ranges.
    auto join_parts = [&](const Piece& pc) {
      __threadfence();
      named_barrier<1, 256>();
      if (tid == 128) ct.last = !*abort && atomicAdd(a.tickets + pc.first_cta, 1u) == (uint32_t)(pc.pieces - 1);
      named_barrier<1, 256>();
      if (ct.last) {
        __threadfence();
        if (tid == 128) a.tickets[pc.first_cta] = 0u;
        constexpr int kLanes = DP / 4;  // threads of a row
        const int col = (tid - 128) % kLanes * 4, rows = (pc.i1 - pc.i0) * G;
        for (int r = (tid - 128) / kLanes; r < rows; r += 256 / kLanes) {
          float top = -INFINITY, sum = 0.f;
          float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
          for (int i = 0; i < pc.pieces; ++i) {
            const float* from = a.partials + ((long long)(pc.first_cta + i) * 2 + (i == 0 ? 1 : 0)) * Sh::kPart;
            const float2 st = __ldcg(reinterpret_cast<const float2*>(from + Sh::kPartRows * DP + r * 2));
            const float4 y = __ldcg(reinterpret_cast<const float4*>(from + r * DP + col));
            const bool any = st.x != -INFINITY;
            const float up = fmaxf(top, st.x), f = any ? exp2_fast((top - up) * sl) : 1.f, g = any ? exp2_fast((st.x - up) * sl) : 0.f;
            top = up;
            sum = sum * f + st.y * g;
            o.x = o.x * f + y.x * g;
            o.y = o.y * f + y.y * g;
            o.z = o.z * f + y.z * g;
            o.w = o.w * f + y.w * g;
          }
          const float inv = sum == 0.f ? 0.f : 1.f / sum;
          if (col < D)
            *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.out) + (long long)(pc.row0 + pc.i0 + r / G) * a.out_token +
                                      (pc.head * G + r % G) * (long long)a.out_head + col) =
                make_uint2(pack_bf16x2(o.x * inv, o.y * inv), pack_bf16x2(o.z * inv, o.w * inv));
        }
      }
      named_barrier<1, 256>();  // `last` has been read
    };
    // Where this thread's row goes, the tile's first token given.
    auto row_out = [&](const Piece& pc, int t0) {
      return static_cast<__nv_bfloat16*>(a.out) + (long long)(pc.row0 + pc.i0 + t0 + row / G) * a.out_token +
             (pc.head * G + row % G) * (long long)a.out_head;
    };
    // One thread of the stream walks, a piece ahead; the pieces stay in shared memory.
    const bool walker = row == kRows - 32;
    if (walker) {
      ct.walk[s].start(plan);
      ct.more[s][0] = ct.walk[s].next<kKeys, true>(P.shape, plan, &ct.piece[s][0]);
    }
    for (int np = 0;; np ^= 1) {
      stream_barrier(s);
      if (!ct.more[s][np]) break;
      if (walker) ct.more[s][np ^ 1] = ct.walk[s].next<kKeys, true>(P.shape, plan, &ct.piece[s][np ^ 1]);
      const Piece& pc = ct.piece[s][np];
      const int nt = pc.k1 - pc.k0, tokens = pc.i1 - pc.i0;
      const bool two = tokens > P.tile_tokens;
      const int t0 = two ? s * P.tile_tokens : 0;                                       // first token of this stream's tile
      const int rows = (two && s == 1 ? tokens - P.tile_tokens : min(tokens, P.tile_tokens)) * G;
      const bool valid = row < rows, busy = (row & ~31) < rows;                          // this row, this warp
      const int p = pc.c + pc.i0 + t0 + row / G;
      const int hi = !valid ? -1 : a.causal ? p : pc.c + pc.n - 1, lo = a.window > 0 ? p - a.window + 1 : 0;
      if (nt == 0) {  // nothing is visible
        if (valid && (two || s == 0) && ok) {
          __nv_bfloat16* out = row_out(pc, t0);
          for (int c = 0; c < D; c += 8) *reinterpret_cast<uint4*>(out + c) = make_uint4(0u, 0u, 0u, 0u);
        }
        continue;
      }
      float m = -INFINITY;                // of the raw scores
      float2 l = make_float2(0.f, 0.f);  // the sum of 2^((score - m) sl), in two parts
      int done = 0;
      const UnitKeys keys = pc.keys;
      const int k0 = pc.k0;
      for (int j = two ? 0 : s; j < nt; j += two ? 1 : 2) {
        // what is known of the tile before its scores are there
        const int j0 = keys.tile(k0 + j) * kKeys;
        const bool edge = j0 < keys.lo || j0 + kKeys - 1 > keys.hi;
        // A row of the tile that holds no token is left as it is: nothing reads what it gives.
        const bool in_sight = __all_sync(0xFFFFFFFFu, !valid || (j0 + kKeys - 1 <= hi && (j0 >= lo || j0 + kKeys <= a.sinks)));
        wait(&ct.s_full[s], ns++ & 1u);
        if (!ok) break;
        tc_fence_after();
        const uint32_t pages = ct.mask[(tiles + j) % kMasks];
        const bool masked = !in_sight || pages != all_boxes;
        // A row of V that no row of the unit sees holds anything, and 0 times that need not
        // be 0: cleared before the product (V of such a tile landed before its scores were
        // issued).
        if (edge) {
          const uint32_t slot = (tiles + j) % Sh::kRingV;
          const int key = j0 + row;
          if (key > keys.hi || (key < keys.lo && key >= a.sinks)) {
#pragma unroll
            for (int h = 0; h < Sh::kHalves; ++h)
#pragma unroll
              for (int c = 0; c < 8; ++c)  // the lanes of a warp begin at different banks
                *reinterpret_cast<uint4*>(smem + Sh::kVOffset + slot * Sh::kTileBytes + h * Sh::kHalfBytes + row * 128 + ((c + row) & 7) * 16) =
                    make_uint4(0u, 0u, 0u, 0u);
          }
          fence_proxy_async_shared();
        }
        if (busy) {
          // Half of the row at a time, in a loop: less code, which a lone warp would wait for.
#pragma unroll 1
          for (int half = 0; half < 2; ++half) {
            float v[64];
            tmem_ld32(t_s + half * 64, v);
            tmem_ld32(t_s + half * 64 + 32, v + 32);
            tmem_wait_ld();
            if (P.negate) {
#pragma unroll
              for (int c = 0; c < 64; ++c) v[c] = -v[c];
            }
            if (masked) {
#pragma unroll
              for (int w = 0; w < 2; ++w) {
                const int k0 = j0 + 64 * half + 32 * w;
                const uint32_t see = seen_word(hi - k0, lo - k0, a.sinks - k0) & page_word(pages, P.kv_box, 2 * half + w);
                if (__all_sync(0xFFFFFFFFu, !valid || see == ~0u)) continue;
#pragma unroll
                for (int c = 0; c < 32; ++c)
                  if (!(see >> c & 1u)) v[32 * w + c] = -INFINITY;
              }
            }
            auto top_of = [&]() {
              float t[4];
#pragma unroll
              for (int i = 0; i < 4; ++i) t[i] = max3(v[i], v[4 + i], v[8 + i]);
#pragma unroll
              for (int c = 12; c < 60; c += 8)
#pragma unroll
                for (int i = 0; i < 4; ++i) t[i] = max3(t[i], v[c + i], v[c + 4 + i]);
              return max3(max3(t[0], t[1], t[2]), max3(t[3], v[60], v[61]), fmaxf(v[62], v[63]));
            };
            if (__any_sync(0xFFFFFFFFu, valid && m == -INFINITY)) {  // nothing seen so far
              const float top = top_of();
              if (m == -INFINITY) m = top;
            }
            // The weights refer to a maximum of before, without looking for this one.  Where their
            // sum in a row shows that one may have grown past 2^14, and only there, the maximum is
            // taken, what was summed so far rescaled, and this half done again.
            // A row whose reference is far from zero takes its maximum at once and subtracts it from the
            // scores.  The rounding of m sl is at most 2^-12 of an exponent below that, less than what a
            // weight loses in bf16; with scores of 2^30 it is some 2^5, and weights that are past 2^14 only
            // through it stay so whatever maximum they refer to.
            float2 sum[2];
            bool moved = false;
            for (;;) {
              const float ref = m == -INFINITY || moved ? 0.f : -m * sl;
              const float2 sl2 = make_float2(sl, sl), ref2 = make_float2(ref, ref);
              sum[0] = sum[1] = make_float2(0.f, 0.f);
#pragma unroll
              for (int c = 0; c < 64; c += 32) {
                uint32_t x[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                  float2 y = fma2(make_float2(v[c + 2 * i], v[c + 2 * i + 1]), sl2, ref2);
                  y.x = exp2_fast(y.x);
                  y.y = exp2_fast(y.y);
                  sum[i & 1] = add2(sum[i & 1], y);
                  x[i] = pack_bf16x2(y.x, y.y);
                }
                tmem_st16(t_s + half * 32 + c / 2, x);
              }
              sum[0] = add2(sum[0], sum[1]);
              const bool raise = valid && (sum[0].x + sum[0].y > 16384.f || fabsf(ref) >= kFar);
              if (!__any_sync(0xFFFFFFFFu, raise)) break;
              tmem_wait_st();
              // By a whole power of two where the maximum is near, so that weights that are in bf16
              // already stay the same numbers.  (Far from zero it need not be one: there a score's own
              // rounding is worth more than a weight's.)
              float f = 1.f;
              if (raise) {
                const float top = fmaxf(m, top_of()), steps = ceilf((top - m) * sl);
                const bool near = fabsf(top) * sl < kFar;
                f = !near ? exp2_fast((m - top) * sl) : steps < 126.f ? __int_as_float((127 - (int)steps) << 23) : 0.f;
                m = near ? m + __fdividef(steps, sl) : top;
              }
              l.x *= f;
              l.y *= f;
              if (done > 0) {
#pragma unroll
                for (int c = 0; c < DP; c += 8) {
                  float o[8];
                  tmem_ld8(t_o + c, o);
                  tmem_wait_ld();
#pragma unroll
                  for (int i = 0; i < 8; ++i) o[i] *= f;
                  tmem_st8(t_o + c, o);
                }
              }
              if (half == 1) {  // the weights of the first half
#pragma unroll
                for (int c = 0; c < 32; c += 8) {
                  float x[8];
                  tmem_ld8(t_s + c, x);
                  tmem_wait_ld();
#pragma unroll
                  for (int i = 0; i < 8; ++i) {
                    const uint32_t w = __float_as_uint(x[i]);
                    x[i] = __uint_as_float(pack_bf16x2(bf16_lo(w) * f, bf16_hi(w) * f));
                  }
                  tmem_st8(t_s + c, x);
                }
              }
              if (valid && !moved && fabsf(m) * sl >= kFar) {  // no weight of this half is above 1 now
                moved = true;
#pragma unroll
                for (int c = 0; c < 64; ++c) v[c] -= m;
              }
            }
            l = add2(l, sum[0]);
          }
          tmem_wait_st();
        }
        ++done;
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&ct.p_full[s]));
      }
      if (done && ok) {  // O is complete
        wait(&ct.o_full[s], no++ & 1u);
        tc_fence_after();
      }
      tiles += nt;

      const float sum_l = l.x + l.y;
      __nv_bfloat16* out = row_out(pc, two ? s * P.tile_tokens : 0);
      const bool whole = pc.pieces == 1;
      float* part = a.partials + ((long long)blockIdx.x * 2 + (pc.k0 == 0 ? 1 : 0)) * Sh::kPart;
      // Columns [c0, c1) of this thread's row: into the output, or into the part.
      auto put = [&](int c, const float (&o)[32], float inv) {
        if (!valid || !ok) return;
        if (whole) {
#pragma unroll
          for (int i = 0; i < 32; i += 8) {
            if (c + i >= D) break;
            uint4 x;
            x.x = pack_bf16x2(o[i] * inv, o[i + 1] * inv);
            x.y = pack_bf16x2(o[i + 2] * inv, o[i + 3] * inv);
            x.z = pack_bf16x2(o[i + 4] * inv, o[i + 5] * inv);
            x.w = pack_bf16x2(o[i + 6] * inv, o[i + 7] * inv);
            *reinterpret_cast<uint4*>(out + c + i) = x;
          }
        } else {
          float* to = part + ((two ? s * kRows : 0) + row) * DP + c;
#pragma unroll
          for (int i = 0; i < 32; i += 4) *reinterpret_cast<float4*>(to + i) = make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]);
        }
      };
      auto put_stat = [&](float mm, float ll) {
        if (valid && !whole && ok)
          *reinterpret_cast<float2*>(part + Sh::kPartRows * DP + ((two ? s * kRows : 0) + row) * 2) = make_float2(mm, ll);
      };
      if (two) {
        const float inv = sum_l == 0.f ? 0.f : 1.f / sum_l;
        if (busy && ok) {
#pragma unroll
          for (int c = 0; c < DP; c += 32) {
            float o[32];
            tmem_ld32(t_o + c, o);
            tmem_wait_ld();
            put(c, o, inv);
          }
        }
        put_stat(m, sum_l);
      } else {
        // The two streams hold parts of the same rows: each joins half of the columns.
        ct.stat[s][row] = make_float2(done ? m : -INFINITY, sum_l);
        tc_fence_before();
        named_barrier<1, 256>();
        tc_fence_after();
        const float2 x0 = ct.stat[0][row], x1 = ct.stat[1][row];
        const float top = fmaxf(x0.x, x1.x);
        const float f0 = x0.x == -INFINITY ? 0.f : exp2_fast((x0.x - top) * sl);
        const float f1 = x1.x == -INFINITY ? 0.f : exp2_fast((x1.x - top) * sl);
        const float sum = x0.y * f0 + x1.y * f1, inv = sum == 0.f ? 0.f : 1.f / sum;
        if (busy && ok) {
#pragma unroll
          for (int c = 0; c < DP / 2; c += 32) {
            const int col = s * (DP / 2) + c;
            float o[32], y[32];
            tmem_ld32(tmem + lanes + 256 + col, o);
            if (nt > 1) tmem_ld32(tmem + lanes + 384 + col, y);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] = nt > 1 ? o[i] * f0 + y[i] * f1 : o[i] * f0;
            put(col, o, inv);
          }
        }
        if (s == 0) put_stat(top, sum);
        tc_fence_before();
        named_barrier<1, 256>();  // both are through with O and the statistics
        tc_fence_after();
      }
      if (whole) continue;

      if (P.join) {
        join_parts(pc);
        continue;
      }
      if (pc.k0 == 0)
        unit = JoinUnit{pc.pieces, tokens * G, min(tokens, P.tile_tokens) * G, pc.row0 + pc.i0, pc.head * G, G, {0, 0}};
    }
    if (!P.join && tid == 128) a.units[blockIdx.x] = unit;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 2) tmem_dealloc(tmem, 512);
}

template <int DP>
cudaError_t launch(TcParams& p, const DeviceInfo& dev, cudaStream_t stream) {
  using Sh = TcShape<DP>;
  const AttendArgs& a = p.a;
  const retrace_kv_cache& c = a.cache;
  CUtensorMap mq, mk, mv;
  {
    const long long dims[3] = {c.head_dim, a.q_heads, a.T}, strides[3] = {1, a.q_head, a.q_token};
    const int box[3] = {64, p.group, p.q_box};
    if (!encode(&mq, a.q, 3, dims, strides, box)) return cudaErrorInvalidValue;
  }
  {
    const long long dims[4] = {c.head_dim, c.kv_heads, c.page_size, c.num_pages};
    const long long strides[4] = {1, c.head_stride, c.slot_stride, c.page_stride};
    const int box[4] = {64, 1, p.kv_box, 1};
    if (!encode(&mk, c.k, 4, dims, strides, box) || !encode(&mv, c.v, 4, dims, strides, box)) return cudaErrorInvalidValue;
  }
  constexpr size_t smem = Sh::kControl + sizeof(Control);
  static_assert(smem <= 227 * 1024, "shared memory of a CTA");
  static std::atomic<uint64_t> allowed{0};
  cudaError_t e = allow_shared(attend_tc_kernel<DP>, smem, dev, allowed);
  if (e != cudaSuccess) return e;
  const int grid = dev.sm_count < kAttendMaxTcCtas ? dev.sm_count : kAttendMaxTcCtas;
  e = launch_dependent(attend_tc_kernel<DP>, dim3(grid), dim3(kThreads), smem, stream, 1u, mq, mk, mv, p);
  if (e != cudaSuccess) return e;
  return p.join ? cudaSuccess : launch_attend_join(a, PartShape{Sh::kPartRows, DP, p.scale2}, grid, stream);
}

}  // namespace

// Every shape that fits, single tokens too, which fill few rows of a tile: 220 of them, 8 heads
// of 128 over up to 1000 keys 163 us, on the CUDA cores 464; up to 79 keys 74 and 93.  (256
// tokens, heads of 64 over up to 79 keys: 71 and 66, over up to 250 95 and 146.)
bool attend_tc_supported(const AttendArgs& a) {
  const retrace_kv_cache& c = a.cache;
  const int G = a.q_heads / c.kv_heads;
  auto whole = [](long long x) { return x % 8 == 0; };
  auto stride = [&](long long x, int extent) { return extent <= 1 || (x > 0 && whole(x)); };
  return c.dtype == RETRACE_BF16 && c.head_dim <= 128 && c.head_dim % 8 == 0 && c.page_size % 8 == 0 && c.num_pages > 0 &&
         G * (8 / gcd(G, 8)) <= kRows && stride(a.q_token, a.T) && stride(a.q_head, a.q_heads) &&
         stride(c.page_stride, c.num_pages) && stride(c.slot_stride, c.page_size) && stride(c.head_stride, c.kv_heads) &&
         whole(a.out_token) && whole(a.out_head) &&
         (((uintptr_t)a.q | (uintptr_t)a.out | (uintptr_t)c.k | (uintptr_t)c.v) & 15u) == 0;
}

size_t attend_tc_partial_bytes(int head_dim) {
  if (head_dim > 128) return 0;
  return (size_t)kAttendMaxTcCtas * 2 * (head_dim <= 64 ? TcShape<64>::kPart : TcShape<128>::kPart) * 4;
}

cudaError_t launch_attend_tc(const AttendArgs& a, cudaStream_t stream) {
  DeviceInfo dev;
  const cudaError_t e = device_info(&dev);
  if (e != cudaSuccess) return e;
  TcParams p{};
  p.a = a;
  const retrace_kv_cache& c = a.cache;
  p.group = a.q_heads / c.kv_heads;
  p.q_box = 8 / gcd(p.group, 8);  // boxes of whole 8-row groups of the swizzle
  p.tile_tokens = kRows / (p.group * p.q_box) * p.q_box;
  p.kv_box = gcd(c.page_size, kKeys);
  const float s = a.scale == 0.f ? 1e-30f : a.scale;  // 2^(1e-30 s) is 1, and -inf stays -inf
  p.scale2 = fminf(fabsf(s) * 1.4426950408889634f, 3.0e38f);
  p.negate = s < 0.f;
  p.shape.q_start = a.q_start;
  p.shape.cache_len = a.cache_len;
  p.shape.B = a.B;
  p.shape.T = a.T;
  p.shape.uniform = a.q_start ? 0 : a.T / a.B;
  p.page_size = FastDivide::of(c.page_size);
  p.shape.kv_heads = c.kv_heads;
  p.shape.causal = a.causal;
  p.shape.window = a.window;
  p.shape.sinks = a.sinks;
  p.shape.places = c.max_pages * c.page_size;
  p.shape.unit_tokens = 2 * p.tile_tokens;
  // Where units of few rows are shared by two or three CTAs, the last one joins the parts
  // and spares a launch; more parts, or larger ones, are read by the whole device in a second
  // kernel.  Tokens over a window of 1024 keys, 2048 units: 186 us here, 201 with it; 500
  // keys, 512 units: 43 / 51; one token over 2048 keys, 8 units of nine parts: 21.0 / 18.2.
  p.join = !a.q_start && (long long)p.shape.uniform * p.group <= kJoinRows && 2ll * a.B * c.kv_heads >= dev.sm_count;
  return c.head_dim <= 64 ? launch<64>(p, dev, stream) : launch<128>(p, dev, stream);
}

}  // namespace retrace
