// Attention over a cache in 8 bits on the tensor cores (bf16 queries).
//
// The keys are on the M side: per tile of 128 keys and up to 72 rows (query tokens times the
// heads of a group) a CTA computes, all products in 8 bits with fp32 accumulation,
//     S^T = K Q^T      [keys, rows]: K as it lies in the cache; a query is the sum of two e4m3 numbers
//                      (its leading 4 bits and the other 4, times 2^-4), in columns of their own;
//     t = scale S 2^ke, p = 2^(t + ve - m), l += p 2^-ve       a key's exponents ke and ve are its
//                      thread's: one thread per key and half of the rows;
//     O^T += V^T P^T   [head dim, rows]: V as it lies; a weight is the sum of three e5m2 numbers of 3
//                      bits each, in columns of their own.
// e5m2 is the upper byte of an fp16 number, so the first two parts of a weight are bytes of it and of
// what is left, and the last, times 2^5, is rounded: 9 bits in all, where a bf16 weight has 8, or multiples
// of 2^-21.  m is chosen so that the largest weight of a row's first tile is 2^4, and raised (O and l
// rescaled) when one passes 2^15; so a weight is off by at most 2^-9 of it or 2^-26 of the row's largest.
// Nothing is converted but the queries, once, and the weights: keys and values go from HBM to shared
// memory to the tensor core, 256 D bytes a tile, 1400 cycles of an SM's share of HBM at D = 128.  The
// products are 4 (2 rows + 3 rows) cycles at D = 128, shared memory moves some 1100 cycles' worth at
// 72 rows, and the softmax does 128 rows exponentials: with few rows on the N side all of
// it scales with the rows that there are.
//
// Warps 0 and 1 copy K, 2 and 3 V (TMA boxes of the slots of a page, dealt out by turns); warp 4 issues
// the scores' products, warp 5 those with V; warps 6 and 7 take the queries apart, a piece ahead.  The softmax has groups of four
// warps, a thread to a key.  Up to 32 rows, two groups take the even and the odd tiles, each
// with references, sums and an O of its own, joined at the end: a tile's way through a group is
// latency, twice what its bytes take.  For 72 rows three groups have 24 rows each of every tile.
#include <math.h>

#include "attend_plan.cuh"
#include "fp8.cuh"
#include "pairs.cuh"
#include "tc_ops.cuh"

namespace retrace {
namespace {

constexpr int kKeys = 128;  // keys of a tile
constexpr unsigned long long kDrainNs = 20ull * 1000ull * 1000ull;
constexpr int kInfoTiles = 16;  // ring of tiles' units: more than the tiles between loading and softmax
constexpr int kMostBoxes = 16;  // of a tile: pages of 8 slots
constexpr int kBase = 256;      // threads before the softmax's
constexpr float kFirstTop = 4.f, kMostTop = 15.f;
constexpr float kNone = 1e30f;     // in place of the reference of a row that has seen nothing
constexpr float kFar = 4194304.f;  // 2^22: references up to it are whole numbers, and sums of two are exact

struct TcParams {
  AttendArgs a;
  AttendShape shape;  // unit_tokens: of a row tile
  int group;          // query heads of a key/value head
  FastDivide by_group, page_size;
  int kv_box;   // slots of a box: they lie within a page and divide a tile
  float scale2;  // scale log2(e)
};

// R rows to a thread of the softmax, in chunks of 16 (the last may be of 8).  Two streams (`kStreams`
// 2): a group has every other tile and all rows; one: the groups share the rows of every tile.
template <int DP, int R>
struct TcShape {
  static constexpr int kStreams = R == 24 ? 1 : 2, kGroups = R == 24 ? 3 : 2;
  static constexpr int kThreads = kBase + 128 * kGroups;
  static constexpr int kRows = kStreams == 2 ? R : R * kGroups;
  static constexpr int kBuffers = 2 * kStreams;  // of S and P
  static constexpr int kChunks = (R + 15) / 16;
  __host__ __device__ static constexpr int rows_of(int chunk) { return R - 16 * chunk < 16 ? R - 16 * chunk : 16; }
  // Columns of S: 2 a row, the two parts of a chunk's queries side by side, group after group.
  static constexpr int kSGroup = 2 * R, kSColumns = kStreams == 2 ? kSGroup : kSGroup * kGroups;
  // Columns of O (and of P): 3 a row; all groups' first chunks, then all second ones.
  static constexpr int kShare = kStreams == 2 ? 1 : kGroups;
  __host__ __device__ static constexpr int o_column(int group, int chunk) {
    return 48 * kShare * chunk + 3 * rows_of(chunk) * (kStreams == 2 ? 0 : group);
  }
  static constexpr int kOColumns = (3 * R * kShare + 15) / 16 * 16;
  static_assert(kSColumns % 16 == 0 && kOColumns <= 256, "columns of a product");
  static constexpr int kOAt = kBuffers * kSColumns;
  static_assert(kOAt + kStreams * kOColumns <= 512, "columns of TMEM");
  // Registers of a thread: the launch's, and what the softmax takes of the others'.
  static constexpr int kFewer = kGroups == 3 ? 56 : 64, kMore = kGroups == 3 ? 120 : 192;
  static_assert(kBase * kFewer + 128 * kGroups * kMore <= kThreads * (65536 / kThreads / 8 * 8), "registers of a CTA");

  static constexpr int kTileBytes = kKeys * DP;
  static constexpr int kPAtoms = (kOColumns + 127) / 128;  // 128-byte columns of P
  static constexpr int kPBytes = kPAtoms * kKeys * 128;
  static constexpr int kQBytes = (kSColumns * DP + 1023) / 1024 * 1024;
  static constexpr int kControlBytes = 12 * 1024;
  static constexpr int kRoom = (227 * 1024 - kControlBytes - kBuffers * kPBytes - 2 * kQBytes) / kTileBytes;
  static constexpr int kRingV = (kRoom + 1) / 2 < 8 ? (kRoom + 1) / 2 : 8, kRingK = kRoom / 2 < 8 ? kRoom / 2 : 8;
  static_assert(kRingK >= 3 && kRingV >= kBuffers, "tiles in flight");
  static constexpr int kVAt = kRingK * kTileBytes, kPAt = kVAt + kRingV * kTileBytes, kQAt = kPAt + kBuffers * kPBytes;
  static constexpr int kControl = kQAt + 2 * kQBytes;
  static constexpr int kPart = kRows * (DP + 2);  // floats of a part
};

// A box's keys: scores are multiplied by k and k / 16, weights are 2^(.. + v), sums take them times inv.
struct BoxUnits {
  float k, v, inv;
  int there;  // has a page
};

template <int R>
struct Control {
  uint64_t full[2][8], empty[2][8];  // rings of K and V
  uint64_t q_full[2], q_empty[2];
  uint64_t s_full[4];   // scores ready
  uint64_t p_full[4];   // weights written, the scores' buffer read
  uint64_t pv_done[4];  // the product with V done
  uint64_t done[2];     // after an expired wait: the issued products
  PlanStart plan;
  long long sum[(kBase + 384) / 32];
  uint32_t tmem;
  int abort;
  PieceWalk walk[3];  // of the softmax groups
  Piece piece[3][2];  // this one and the next
  int more[3][2];
  BoxUnits units[kInfoTiles][kMostBoxes];
  alignas(16) float factor[2][72];  // of a row: scale log2(e) times its queries' unit
  long long out[2][72];             // where a row goes, elements
  // Of a group's rows: what is added to exponents (minus the reference), and, where that is far from
  // zero, added to the difference; how the reference moves; at the end the factors of the streams' O.
  alignas(16) float minus[3][R], rest[3][R], move[3][R];
  alignas(16) float scale[3][R];
  float part[3][4][R];  // per warp: a row's maximum, or sum
};

// ---- instructions -------------------------------------------------------------
// D[tmem] (+)= A[smem] * B[smem], 8-bit inputs, fp32 accumulation.
__device__ __forceinline__ void tc_mma_8bit(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
      "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// kind::f8f6f4: fp32 accumulator (bits 4-5 = 1); formats of A (7-9) and B (10-12): e4m3 0, e5m2 1; A and B
// MN-major (15, 16); N >> 3 (17-22), M >> 4 (24-28).
__host__ __device__ constexpr uint32_t idesc_8bit(int N, bool values) {
  return (1u << 4) | ((uint32_t)(N >> 3) << 17) | ((128u >> 4) << 24) | (values ? 1u << 10 | 1u << 15 | 1u << 16 : 0u);
}
// Rows of DP bytes with the swizzle of their width, 8 rows a group; `lead`: from one column of DP (of P: 128)
// bytes to the next, for an MN-major operand.
template <int kWidth>
__device__ __forceinline__ uint64_t rows_desc(uint32_t saddr, uint32_t lead) {
  constexpr uint64_t mode = kWidth == 128 ? 2 : 4;
  return (uint64_t)((saddr & 0x3FFFFu) >> 4) | (uint64_t)(lead >> 4) << 16 | (uint64_t)((kWidth * 8) >> 4) << 32 | (uint64_t)1 << 46 | mode << 61;
}

template <int N>
__device__ __forceinline__ void tmem_load(uint32_t at, float* v) {
  uint32_t* r = reinterpret_cast<uint32_t*>(v);
  if constexpr (N == 32) {
    tmem_ld32(at, v);
  } else if constexpr (N == 16) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
                   "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(at)
                 : "memory");
  } else if constexpr (N == 8) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(at)
                 : "memory");
  } else {
    static_assert(N == 4, "4, 8, 16 or 32 columns");
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
  }
}
__device__ __forceinline__ void tmem_store4(uint32_t at, const float* v) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1,%2,%3,%4};" ::"r"(at), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]) : "memory");
}
// Rows (N of them) over the lanes of a warp by `join`: each step halves the rows that a lane has.  Lane i
// ends with row i % N, in v[0].
template <int N, typename Join>
__device__ __forceinline__ void join_lanes(float* v, int lane, Join&& join) {
#pragma unroll
  for (int o = N / 2; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < o; ++i) {
      const bool upper = lane & o;
      const float other = __shfl_xor_sync(0xFFFFFFFFu, upper ? v[i] : v[i + o], o);
      v[i] = join(upper ? v[i + o] : v[i], other);
    }
#pragma unroll
  for (int o = N; o < 32; o <<= 1) v[0] = join(v[0], __shfl_xor_sync(0xFFFFFFFFu, v[0], o));
}
// A group's agreement on whether any of its threads says so.
__device__ __forceinline__ bool any_of_group(int group, bool mine) {
  uint32_t p = mine;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %0, 0;\n\t"
      "barrier.cta.red.or.pred q, %1, 128, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "+r"(p)
      : "r"(2 + group)
      : "memory");
  return p != 0;
}
__device__ __forceinline__ void group_barrier(int group) { asm volatile("bar.sync %0, 128;" ::"r"(2 + group) : "memory"); }

// Registers from the copies, products and queries to the softmax.
template <int kCount>
__device__ __forceinline__ void fewer_registers() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kCount));
}
template <int kCount>
__device__ __forceinline__ void more_registers() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kCount));
}

__device__ __forceinline__ uint32_t halves(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t minus_halves(uint32_t a, uint32_t b) {
  const __half2 h = __hsub2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t times_32(uint32_t a) {
  const __half2 h = __hmul2(*reinterpret_cast<const __half2*>(&a), __float2half2_rn(32.f));
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t to_e5m2x2(uint32_t h) {
  __half2_raw r;
  r.x = (unsigned short)(h & 0xFFFFu);
  r.y = (unsigned short)(h >> 16);
  return __nv_cvt_halfraw2_to_fp8x2(r, __NV_SATFINITE, __NV_E5M2);
}
// The three parts of four weights, none negative, a byte each; the third times 2^5.
__device__ __forceinline__ void take_apart(const float (&w)[4], uint32_t& first, uint32_t& second, uint32_t& third) {
  const uint32_t a = halves(w[0], w[1]), b = halves(w[2], w[3]);
  const uint32_t a1 = minus_halves(a, a & 0xFF00FF00u), b1 = minus_halves(b, b & 0xFF00FF00u);
  const uint32_t a2 = minus_halves(a1, a1 & 0xFF00FF00u), b2 = minus_halves(b1, b1 & 0xFF00FF00u);
  first = __byte_perm(a, b, 0x7531);
  second = __byte_perm(a1, b1, 0x7531);
  third = to_e5m2x2(times_32(a2)) | to_e5m2x2(times_32(b2)) << 16;
}

template <int I>
struct Index {
  static constexpr int value = I;
};
template <int N, int I = 0, typename F>
__device__ __forceinline__ void each_chunk(F&& f) {
  if constexpr (I < N) {
    f(Index<I>{});
    each_chunk<N, I + 1>(f);
  }
}

template <int DP, int R>
__global__ void __launch_bounds__(TcShape<DP, R>::kThreads, 1)
    attend_fp8_tc_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                         const __grid_constant__ TcParams P) {
  using Sh = TcShape<DP, R>;
  constexpr int kThreads = Sh::kThreads, kBuffers = Sh::kBuffers;
  static_assert(sizeof(Control<R>) <= Sh::kControlBytes, "room of the control block");
  extern __shared__ __align__(1024) uint8_t smem[];
  Control<R>& ct = *reinterpret_cast<Control<R>*>(smem + Sh::kControl);
  volatile int* abort = &ct.abort;
  const uint32_t base = smem_u32(smem);
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  const AttendArgs& a = P.a;

  if (tid == 0) {
    ct.abort = 0;
    for (int r = 0; r < 2; ++r)
      for (int s = 0; s < 8; ++s) {
        mbar_init(smem_u32(&ct.full[r][s]), 2);  // two copying warps
        mbar_init(smem_u32(&ct.empty[r][s]), 1);
      }
    for (int s = 0; s < 2; ++s) {
      mbar_init(smem_u32(&ct.done[s]), 1);
      mbar_init(smem_u32(&ct.q_full[s]), 2);
      mbar_init(smem_u32(&ct.q_empty[s]), 1 + 4 * Sh::kGroups);  // the products, and the softmax warps
    }
    for (int s = 0; s < 4; ++s) {
      mbar_init(smem_u32(&ct.s_full[s]), 1);
      mbar_init(smem_u32(&ct.p_full[s]), 4 * Sh::kGroups / Sh::kStreams);  // the warps that have the tile
      mbar_init(smem_u32(&ct.pv_done[s]), 1);
    }
    fence_mbar_init();
    tma_prefetch_desc(&tm_k);
    tma_prefetch_desc(&tm_v);
  }
  if (warp == 4) {
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
  if (warp < 8) {
    fewer_registers<Sh::kFewer>();
    PieceWalk walk;
    walk.start(plan);
    Piece pc;
    bool ok = true, drain = false;
    if (warp < 4) {
      // ---- copies of K (warps 0, 1) and V (2, 3): every other box each ----
      // Lane (tile, box) looks up and copies a box of each of a batch of tiles.  What it reads for
      // the next batch is not used before the present one has been copied: the warp would wait for it.
      const int ring = warp / 2, turn = warp % 2;
      const bool keys = ring == 0;
      const CUtensorMap* map = keys ? &tm_k : &tm_v;
      const int boxes = kKeys / P.kv_box, mine = (boxes + 1 - turn) / 2;
      const int batch = min(32 / max(mine, 1), 8), my_tile = mine > 0 ? lane / mine : 32, box = mine > 0 ? lane % mine * 2 + turn : 0;
      const uint32_t slots = keys ? Sh::kRingK : Sh::kRingV, tiles_at = base + (keys ? 0 : Sh::kVAt);
      uint32_t tiles = 0, slot = 0, phase = 0;
      struct Lookup {
        int slot;          // within the page
        bool listed;       // the table has an entry for it
        const int32_t* at;
      };
      auto lookup = [&](int k) {  // of this lane's box of tile k + my_tile of the piece
        Lookup x{0, false, a.cache.page_table};
        k += my_tile;
        if (my_tile < batch && k < pc.k1 - pc.k0) {
          const int j = pc.keys.tile(pc.k0 + k) * kKeys + box * P.kv_box, i = P.page_size(j);
          x.slot = j - i * P.page_size.by;
          x.listed = i < a.cache.max_pages;
          if (x.listed) x.at += pc.b * a.cache.table_stride + i;
        }
        return x;
      };
      while (ok && walk.next<kKeys>(P.shape, plan, &pc)) {
        const int nt = pc.k1 - pc.k0;
        if (nt == 0) continue;
        Lookup now = lookup(0);
        int page = now.listed ? *now.at : -1;
        for (int k = 0; k < nt && ok; k += batch) {
          // a box without a page lies outside the tensor: zeros
          if (page < 0 || page >= a.cache.num_pages) page = a.cache.num_pages;
          const bool there = page < a.cache.num_pages;
          int ke = 0, ve = 0;
          if (keys && there) {
            const long long at = page * a.exp_page + pc.head * a.exp_head;
            ke = a.k_exp[at];
            ve = a.v_exp[at];
          }
          const Lookup next = lookup(k + batch);
          const int next_page = next.listed ? *next.at : -1;
          for (int t = 0; t < min(batch, nt - k); ++t) {
            ok = warp_wait_quick(&ct.empty[ring][slot], phase ^ 1u, abort);
            if (!ok) break;
            const uint32_t bar = smem_u32(&ct.full[ring][slot]);
            const bool active = my_tile == t;
            if (keys && active)
              ct.units[tiles % kInfoTiles][box] = there ? BoxUnits{power_of_two(clamp_exponent(ke)), (float)clamp_exponent(ve), power_of_two(-clamp_exponent(ve)), 1}
                                                        : BoxUnits{1.f, 0.f, 1.f, 0};
            __syncwarp();
            if (lane == 0) mbar_arrive_expect_tx(bar, mine * P.kv_box * DP);
            __syncwarp();
            if (active)
              tma_load_4d(tiles_at + slot * Sh::kTileBytes + box * P.kv_box * DP, map, 0, pc.head, now.slot, page, bar);
            if (++slot == slots) {
              slot = 0;
              phase ^= 1u;
            }
            ++tiles;
          }
          now = next;
          page = next_page;
        }
      }
      drain = !ok;
    } else if (warp == 4 || warp == 5) {
      // ---- products: scores (warp 4) and O (warp 5) ----
      // Issuing a tile's products and commits takes some 500 cycles of a warp; one warp for both had
      // 1100 a tile, and was the bound with few rows.
      const bool values = warp == 5;
      uint32_t tiles = 0, pieces = 0;
      auto wait = [&](uint64_t* bar, uint32_t parity) {
        ok = ok && warp_wait_quick(bar, parity, abort);
        return ok;
      };
      while (ok && walk.next<kKeys>(P.shape, plan, &pc)) {
        const int nt = pc.k1 - pc.k0;
        if (nt == 0) continue;
        const uint32_t q = pieces & 1u;
        if (!values) {
          constexpr uint32_t kDesc = idesc_8bit(Sh::kSColumns, false);
          if (!wait(&ct.q_full[q], pieces >> 1 & 1u)) break;
          for (int i = 0; i < nt; ++i) {
            const uint32_t g = tiles + i, b = g % kBuffers, slot = g % Sh::kRingK;
            if (!wait(&ct.full[0][slot], g / Sh::kRingK & 1u)) break;
            if (g >= kBuffers && !wait(&ct.p_full[b], (g / kBuffers & 1u) ^ 1u)) break;  // S has been read
            tc_fence_after();
            if (elect_one()) {
              const uint64_t kd = rows_desc<DP>(base + slot * Sh::kTileBytes, 16), qd = rows_desc<DP>(base + Sh::kQAt + q * Sh::kQBytes, 16);
#pragma unroll
              for (int k = 0; k < DP / 32; ++k) tc_mma_8bit(tmem + b * Sh::kSColumns, kd + 2 * k, qd + 2 * k, kDesc, k > 0);
              tc_commit(smem_u32(&ct.s_full[b]));
              tc_commit(smem_u32(&ct.empty[0][slot]));
            }
            __syncwarp();
          }
          if (!ok) break;
          if (elect_one()) tc_commit(smem_u32(&ct.q_empty[q]));
          __syncwarp();
        } else {
          constexpr uint32_t kDesc = idesc_8bit(Sh::kOColumns, true);
          for (int i = 0; i < nt; ++i) {
            const uint32_t g = tiles + i, b = g % kBuffers, slot = g % Sh::kRingV;
            if (!wait(&ct.full[1][slot], g / Sh::kRingV & 1u) || !wait(&ct.p_full[b], g / kBuffers & 1u)) break;
            tc_fence_after();
            if (elect_one()) {
              // 64 columns of the head dimension fill half of M: the other half is the same again
              const uint64_t vd = rows_desc<DP>(base + Sh::kVAt + slot * Sh::kTileBytes, 0);
              const uint64_t pd = rows_desc<128>(base + Sh::kPAt + b * Sh::kPBytes, kKeys * 128);
              const uint32_t t_o = tmem + Sh::kOAt + i % Sh::kStreams * Sh::kOColumns;
#pragma unroll
              for (int k = 0; k < kKeys / 32; ++k)
                tc_mma_8bit(t_o, vd + k * (32 * DP >> 4), pd + k * (32 * 128 >> 4), kDesc, i >= Sh::kStreams || k > 0);
              tc_commit(smem_u32(&ct.pv_done[b]));
              tc_commit(smem_u32(&ct.empty[1][slot]));
            }
            __syncwarp();
          }
          if (!ok) break;
        }
        ++pieces;
        tiles += nt;
      }
      if (!ok) {
        volatile int never = 0;
        if (elect_one()) tc_commit(smem_u32(&ct.done[values]));
        __syncwarp();
        mbar_wait_bounded(smem_u32(&ct.done[values]), 0, &never);
      }
    } else {
      // ---- queries: rows of 128 or 64 bytes, each a sum of two e4m3 numbers times its row's unit ----
      constexpr int kEach = DP / 32;  // elements of a lane
      const int D = a.cache.head_dim;
      uint32_t pieces = 0;
      while (ok && walk.next<kKeys>(P.shape, plan, &pc)) {
        if (pc.k1 == pc.k0) continue;
        const uint32_t buffer = pieces & 1u;
        ok = warp_wait_quick(&ct.q_empty[buffer], (pieces >> 1 & 1u) ^ 1u, abort);
        if (!ok) break;
        ++pieces;
        const int rows = (pc.i1 - pc.i0) * P.group;
        uint8_t* to = smem + Sh::kQAt + buffer * Sh::kQBytes;
        for (int r0 = warp - 6; r0 < Sh::kRows; r0 += 2 * 4) {
          // four rows' loads at a time
          uint32_t raw[4][kEach / 2];
          int token[4], head[4];
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const int r = r0 + 2 * u;
            token[u] = P.by_group(r);
            head[u] = r - token[u] * P.group;
            token[u] += pc.row0 + pc.i0;
            head[u] += pc.head * P.group;
#pragma unroll
            for (int e = 0; e < kEach / 2; ++e) raw[u][e] = 0u;
            if (r < rows && lane * kEach < D) {
              const __nv_bfloat16* from = static_cast<const __nv_bfloat16*>(a.q) + token[u] * a.q_token + head[u] * a.q_head + lane * kEach;
              if constexpr (kEach == 4)
                *reinterpret_cast<uint2*>(raw[u]) = *reinterpret_cast<const uint2*>(from);
              else
                raw[u][0] = *reinterpret_cast<const uint32_t*>(from);
            }
          }
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const int r = r0 + 2 * u;
            if (r >= Sh::kRows) break;
            // magnitudes as whole numbers: infinities and NaN are the largest
            uint32_t most = 0u;
#pragma unroll
            for (int e = 0; e < kEach / 2; ++e) most = max(most, max(raw[u][e] & 0x7FFFu, raw[u][e] >> 16 & 0x7FFFu));
            const uint32_t top = __reduce_max_sync(0xFFFFFFFFu, most) << 16;
            // the least exponent with top <= 448 times its power of two; a row with an infinity or a
            // NaN is NaN throughout, as its scores are
            const int e = min(max((int)(top >> 23) - 127 - 8 + ((top & 0x7FFFFFu) > 0x600000u), -120), 120);
            const float down = power_of_two(-e);
            const bool nan = top >= 0x7F800000u;
            uint32_t lead = 0u, rest = 0u;
#pragma unroll
            for (int i = 0; i < kEach / 2; ++i) {
              const float x = bf16_lo(raw[u][i]) * down, y = bf16_hi(raw[u][i]) * down;
              const uint32_t c = to_e4m3x2(x, y);
              const float2 f = e4m3_floats(c);
              lead |= c << (16 * i);
              rest |= to_e4m3x2((x - f.x) * 16.f, (y - f.y) * 16.f) << (16 * i);
            }
            if (nan) lead = 0x7F7F7F7Fu;
            // the columns of the row's two parts
            const int group = r / R, in = r % R, chunk = in / 16, c = in % 16, size = min(16, R - 16 * chunk);
#pragma unroll
            for (int part = 0; part < 2; ++part) {
              const int n = group * Sh::kSGroup + 32 * chunk + part * size + c, at = lane * kEach;
              const int chunk16 = DP == 128 ? (at / 16) ^ (n & 7) : (at / 16) ^ (n >> 1 & 3);
              uint8_t* dst = to + n * DP + chunk16 * 16 + at % 16;
              if constexpr (kEach == 4)
                *reinterpret_cast<uint32_t*>(dst) = part ? rest : lead;
              else
                *reinterpret_cast<uint16_t*>(dst) = (uint16_t)(part ? rest : lead);
            }
            if (lane == 0) {
              ct.factor[buffer][r] = r < rows ? P.scale2 * power_of_two(e) : 0.f;
              ct.out[buffer][r] = token[u] * a.out_token + head[u] * a.out_head;
            }
          }
        }
        fence_proxy_async_shared();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&ct.q_full[buffer]));
      }
    }
    if (!ok && lane == 0) raise_abort(abort, a.status);
    // After an expired wait: time for this CTA's copies in flight to land.
    if (drain) {
      const unsigned long long t0 = global_ns();
      while (global_ns() - t0 < kDrainNs) __nanosleep(1000);
    }
    __syncwarp();
  } else {
    more_registers<Sh::kMore>();
    // ---- softmax: group h, one thread per key ----
    constexpr bool kTwo = Sh::kStreams == 2;
    const int h = (warp - kBase / 32) / 4, key = tid & 127, quarter = warp & 3, r0 = kTwo ? 0 : h * R;
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
    const uint32_t t_o = tmem + lanes + Sh::kOAt + (kTwo ? h * Sh::kOColumns : 0);
    const int D = a.cache.head_dim, G = P.group;
    uint32_t tiles = 0, pieces = 0;
    JoinUnit unit{};
    bool ok = true;
    // After an expired wait a warp goes on without waiting, and writes nothing: the warps of a group meet
    // at the same barriers all the same.
    auto wait = [&](uint64_t* bar, uint32_t parity) {
      if (ok && !warp_wait_quick(bar, parity, abort)) {
        ok = false;
        if (lane == 0) raise_abort(abort, a.status);
      }
    };
    // One thread of the group walks, a piece ahead; the pieces stay in shared memory.
    const bool walker = key == 96;
    if (walker) {
      ct.walk[h].start(plan);
      ct.more[h][0] = ct.walk[h].template next<kKeys, true>(P.shape, plan, &ct.piece[h][0]);
    }
    for (int np = 0;; np ^= 1) {
      group_barrier(h);
      if (!ct.more[h][np]) break;
      if (walker) ct.more[h][np ^ 1] = ct.walk[h].template next<kKeys, true>(P.shape, plan, &ct.piece[h][np ^ 1]);
      const Piece& pc = ct.piece[h][np];
      const int nt = pc.k1 - pc.k0, rows = (pc.i1 - pc.i0) * G;
      if (nt == 0) {  // nothing is visible
        for (int i = h * 128 + key; i < Sh::kRows * D; i += 128 * Sh::kGroups) {
          const int r = i / D, token = P.by_group(r);
          if (r < rows)
            static_cast<__nv_bfloat16*>(a.out)[(long long)(pc.row0 + pc.i0 + token) * a.out_token +
                                               (pc.head * G + r - token * G) * (long long)a.out_head + i % D] = __float2bfloat16_rn(0.f);
        }
        continue;
      }
      const uint32_t buffer = pieces & 1u;
      wait(&ct.q_full[buffer], pieces >> 1 & 1u);
      ++pieces;
      const float* factor = ct.factor[buffer] + r0;
      // A row of the tile that holds no token refers to a number that no weight comes near.
      if (key < R) {
        ct.minus[h][key] = r0 + key < rows ? kNone : -kNone;
        ct.rest[h][key] = 0.f;
      }
      group_barrier(h);
      float2 l[R / 2];  // sums of this thread's keys
#pragma unroll
      for (int i = 0; i < R / 2; ++i) l[i] = make_float2(0.f, 0.f);
      bool far = false;  // some row's reference is far from zero
      const UnitKeys keys = pc.keys;
      const int first = pc.c + pc.i0, k0 = pc.k0;  // position of the unit's first token
      const bool idle = r0 >= rows;

      for (int j = kTwo ? h : 0; j < nt; j += Sh::kStreams) {
        // what is known of the tile before its scores are there
        const uint32_t g = tiles + j, b = g % kBuffers;
        const int j0 = keys.tile(k0 + j) * kKeys, at = j0 + key;
        const bool edge = j0 < keys.lo || j0 + kKeys - 1 > keys.hi;
        // The key is seen by the rows [from, to).
        int from = 0, to = rows;
        if (a.causal && at > first) from = (at - first) * G;
        if (a.window > 0 && at >= a.sinks && at - first + a.window < P.shape.unit_tokens)
          to = max(at - first + a.window, 0) * G;
        if (at > keys.hi) to = 0;
        from -= r0;
        to -= r0;
        wait(&ct.s_full[b], g / kBuffers & 1u);
        if (g >= kBuffers) wait(&ct.pv_done[b], (g / kBuffers & 1u) ^ 1u);  // the weights' buffer is free
        tc_fence_after();
        const BoxUnits u = ct.units[g % kInfoTiles][key / P.kv_box];
        if (!u.there) to = from = -1000;
        // A row of V that no row of the unit sees holds anything, and 0 times that need not be 0:
        // cleared before the product.
        if (edge && (kTwo || h == 0)) {
          // (the slot's phase before is over: its product was issued before the one waited for above)
          wait(&ct.full[1][g % Sh::kRingV], g / Sh::kRingV & 1u);
          if (at > keys.hi || (at < keys.lo && at >= a.sinks)) {
            uint8_t* v = smem + Sh::kVAt + (g % Sh::kRingV) * Sh::kTileBytes + key * DP;
#pragma unroll
            for (int c = 0; c < DP / 16; ++c)  // the lanes begin at different banks
              *reinterpret_cast<uint4*>(v + ((c + 2 * key) % (DP / 16)) * 16) = make_uint4(0u, 0u, 0u, 0u);
          }
        }
        if (!idle) {
          const bool masked = !__all_sync(0xFFFFFFFFu, from <= 0 && to >= min(rows - r0, R));
          const uint32_t t_s = tmem + lanes + b * Sh::kSColumns + (kTwo ? 0 : h * Sh::kSGroup);
          const float2 sixteenth = make_float2(0.0625f, 0.0625f), unit2 = make_float2(u.k, u.k), v2 = make_float2(u.v, u.v);
          float y[R];  // exponents of the weights
          auto hide = [&]() {
            if (!masked) return;
#pragma unroll
            for (int r = 0; r < R; ++r)
              if (r < from || r >= to) y[r] = -INFINITY;
          };
          // Scores in the keys' units, two rows at a time: f(row, scores).
          auto scores = [&](auto&& f) {
            float s[2 * R];
            each_chunk<Sh::kChunks>([&](auto chunk) {
              constexpr int c = decltype(chunk)::value;
              tmem_load<2 * Sh::rows_of(c)>(t_s + 32 * c, s + 32 * c);
            });
            tmem_wait_ld();
            each_chunk<Sh::kChunks>([&](auto chunk) {
              constexpr int c = decltype(chunk)::value, n = Sh::rows_of(c);
#pragma unroll
              for (int i = 0; i < n; i += 2) {
                const float2 x = fma2(make_float2(s[32 * c + n + i], s[32 * c + n + i + 1]), sixteenth, make_float2(s[32 * c + i], s[32 * c + i + 1]));
                f(16 * c + i, mul2(x, unit2));
              }
            });
            hide();
          };
          auto put = [&](int r, const float2& x) {
            y[r] = x.x;
            y[r + 1] = x.y;
          };
          auto two = [](const float* p) { return *reinterpret_cast<const float2*>(p); };
          // The product with the factor rounded before the reference is taken off, for references far from
          // zero; `fresh`: rows that have none keep their exponents.
          auto exact = [&](bool fresh) {
            scores([&](int r, const float2& x) {
              float2 ref = two(ct.minus[h] + r);
              if (fresh && ref.x == kNone) ref.x = 0.f;
              if (fresh && ref.y == kNone) ref.y = 0.f;
              put(r, add2(add2(add2(mul2(x, two(factor + r)), ref), v2), two(ct.rest[h] + r)));
            });
          };
          auto exponents = [&]() {
            if (far)
              exact(false);
            else
              scores([&](int r, const float2& x) { put(r, add2(fma2(x, two(factor + r), two(ct.minus[h] + r)), v2)); });
          };
          // The rows' maxima, to ct.part.
          auto maxima = [&]() {
            each_chunk<Sh::kChunks>([&](auto chunk) {
              constexpr int c = decltype(chunk)::value, n = Sh::rows_of(c);
              float v[n];
#pragma unroll
              for (int i = 0; i < n; ++i) v[i] = y[16 * c + i];
              join_lanes<n>(v, lane, [](float p, float q) { return fmaxf(p, q); });
              if (lane < n) ct.part[h][quarter][16 * c + lane] = v[0];
            });
            group_barrier(h);
          };
          auto most_of = [&](int r) { return fmaxf(fmaxf(ct.part[h][0][r], ct.part[h][1][r]), fmaxf(ct.part[h][2][r], ct.part[h][3][r])); };

          // The first tile sets the references.  After it a weight may outgrow its own, or a row may see
          // its first keys: then, too, the rows' maxima over the tile, new references (whole numbers,
          // so that they are the same however often they move), and what was summed so far in the new unit.
          const bool fresh = j < Sh::kStreams;
          bool raise = fresh;
          if (!fresh) {
            exponents();
            float top = -INFINITY;
#pragma unroll
            for (int r = 0; r < R; r += 2) top = max3(top, y[r], y[r + 1]);
            raise = any_of_group(h, top > kMostTop);
          }
          if (raise) {
            exact(true);
            maxima();
            float old = 0.f, old_rest = 0.f, now = 0.f, now_rest = 0.f, move = 0.f;
            bool pending = false;
            if (key < R) {
              old = now = ct.minus[h][key];
              old_rest = now_rest = ct.rest[h][key];
              const float most = most_of(key), by = floorf(kFirstTop - most);
              if (old == kNone ? most > -INFINITY : most > kMostTop) {
                const float from_zero = old == kNone ? 0.f : old;
                if (fabsf(from_zero) >= kFar) {
                  now_rest = old_rest + by;
                  move = by;
                } else if (fabsf(from_zero + by) < kFar) {
                  now = from_zero + by;
                  move = by;
                } else {  // the maximum itself, and what is left of it over the tile
                  now = from_zero - most;
                  pending = true;
                }
                ct.minus[h][key] = now;
                ct.rest[h][key] = now_rest;
              }
              ct.move[h][key] = move;
            }
            const bool again = any_of_group(h, pending);
            if (again) {
              exact(false);
              maxima();
              if (pending) {
                now_rest = floorf(kFirstTop - most_of(key));
                ct.rest[h][key] = now_rest;
              }
              far = true;
            }
            if (key < R) ct.scale[h][key] = old == kNone ? 0.f : exp2_fast((now - old) + (now_rest - old_rest));
            group_barrier(h);
            if (!fresh) {
#pragma unroll
              for (int r = 0; r < R; r += 2) l[r / 2] = mul2(l[r / 2], two(ct.scale[h] + r));
              const uint32_t before = g - Sh::kStreams;
              wait(&ct.pv_done[before % kBuffers], before / kBuffers & 1u);
              tc_fence_after();
              each_chunk<Sh::kChunks>([&](auto chunk) {
                constexpr int c = decltype(chunk)::value, n = Sh::rows_of(c);
#pragma unroll
                for (int part = 0; part < 3; ++part) {
                  float o[n];
                  const uint32_t column = t_o + Sh::o_column(h, c) + part * n;
                  tmem_load<n>(column, o);
                  tmem_wait_ld();
#pragma unroll
                  for (int i = 0; i < n; ++i) o[i] *= ct.scale[h][16 * c + i];
#pragma unroll
                  for (int i = 0; i < n; i += 4) tmem_store4(column + i, o + i);
                }
              });
              tmem_wait_st();
            }
            if (again) {
              exact(false);
            } else {
#pragma unroll
              for (int r = 0; r < R; r += 2) put(r, add2(make_float2(y[r], y[r + 1]), two(ct.move[h] + r)));
            }
          }

          uint8_t* weights = smem + Sh::kPAt + b * Sh::kPBytes + key * 128;
          const float2 inv2 = make_float2(u.inv, u.inv);
          each_chunk<Sh::kChunks>([&](auto chunk) {
            constexpr int c = decltype(chunk)::value, n = Sh::rows_of(c);
            uint32_t w[3 * n / 4];
#pragma unroll
            for (int i = 0; i < n; i += 4) {
              float e[4];
#pragma unroll
              for (int k = 0; k < 4; ++k) e[k] = exp2_fast(y[16 * c + i + k]);
              l[(16 * c + i) / 2] = fma2(make_float2(e[0], e[1]), inv2, l[(16 * c + i) / 2]);
              l[(16 * c + i) / 2 + 1] = fma2(make_float2(e[2], e[3]), inv2, l[(16 * c + i) / 2 + 1]);
              take_apart(e, w[i / 4], w[n / 4 + i / 4], w[2 * (n / 4) + i / 4]);
            }
            const int column = Sh::o_column(h, c);
#pragma unroll
            for (int i = 0; i < 3; ++i) {
              const int x = column + i * n;
              uint8_t* to_w = weights + x / 128 * (kKeys * 128) + ((x % 128 / 16) ^ (key & 7)) * 16 + x % 16;
              if constexpr (n == 16)
                *reinterpret_cast<uint4*>(to_w) = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
              else
                *reinterpret_cast<uint2*>(to_w) = make_uint2(w[2 * i], w[2 * i + 1]);
            }
          });
        }
        fence_proxy_async_shared();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&ct.p_full[b]));
      }
      tiles += nt;

      // The rows' sums over the group's threads.
      each_chunk<Sh::kChunks>([&](auto chunk) {
        constexpr int c = decltype(chunk)::value, n = Sh::rows_of(c);
        float v[n];
#pragma unroll
        for (int i = 0; i < n; ++i) v[i] = i % 2 ? l[8 * c + i / 2].y : l[8 * c + i / 2].x;
        join_lanes<n>(v, lane, [](float p, float q) { return p + q; });
        if (lane < n) ct.part[h][quarter][16 * c + lane] = v[0];
      });
      if constexpr (kTwo)
        named_barrier<1, 256>();
      else
        group_barrier(h);
      const bool whole = pc.pieces == 1;
      float* part = a.partials + ((long long)blockIdx.x * 2 + (pc.k0 == 0 ? 1 : 0)) * Sh::kPart;
      auto sum_of = [&](int s, int r) { return (ct.part[s][0][r] + ct.part[s][1][r]) + (ct.part[s][2][r] + ct.part[s][3][r]); };
      if (key < R) {
        // What O is multiplied by, so that it refers to `top`: to a number, where minus and rest are two.
        const float m = -(ct.minus[h][key] + ct.rest[h][key]);
        float sum = sum_of(h, key), top = m, f;
        if constexpr (kTwo) {  // the larger reference for both streams
          const float other = -(ct.minus[h ^ 1][key] + ct.rest[h ^ 1][key]), other_sum = sum_of(h ^ 1, key);
          const bool mine = ct.minus[h][key] != kNone, theirs = ct.minus[h ^ 1][key] != kNone;
          top = !theirs ? m : !mine ? other : fmaxf(m, other);
          f = mine ? exp2_fast(-((ct.minus[h][key] + top) + ct.rest[h][key])) : 0.f;
          sum = sum * f + other_sum * (theirs ? exp2_fast(-((ct.minus[h ^ 1][key] + top) + ct.rest[h ^ 1][key])) : 0.f);
        } else {
          f = exp2_fast(-((ct.minus[h][key] + top) + ct.rest[h][key]));
          sum *= f;
        }
        ct.scale[h][key] = whole ? (sum == 0.f ? 0.f : f / sum) : f;
        if (!whole && ok && r0 + key < rows && (!kTwo || h == 0))
          *reinterpret_cast<float2*>(part + Sh::kRows * DP + (r0 + key) * 2) = make_float2(sum == 0.f ? -INFINITY : top, sum);
      }
      if constexpr (kTwo)
        named_barrier<1, 256>();
      else
        group_barrier(h);
      // O is complete
      if (ok) {
        const uint32_t last = tiles - 1;
        wait(&ct.pv_done[last % kBuffers], last / kBuffers & 1u);
        tc_fence_after();
      }
      // `key` is the lane, the element of the head; row r of x[i] goes out.
      auto put_rows = [&](int from, const float* x, int n) {
#pragma unroll
        for (int i = 0; i < n; ++i) {
          const int r = from + i;
          if (r >= rows || key >= DP) break;
          if (!whole)
            part[r * DP + key] = x[i];
          else if (key < D)
            static_cast<__nv_bfloat16*>(a.out)[ct.out[buffer][r] + key] = __float2bfloat16_rn(x[i]);
        }
      };
      if constexpr (kTwo) {
        // half of the rows to each group, from both streams' O (the second has none where there was one tile)
        constexpr int n = R / 2, c = R == 32 ? 16 : R;  // rows of a chunk
        const int from = h * n;
        if (ok && from < rows) {
          float x[n];
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            if (s == 1 && nt == 1) break;
            float o[3 * n];
            const uint32_t column = tmem + lanes + Sh::kOAt + s * Sh::kOColumns + (R == 32 ? 48 * h : from);
#pragma unroll
            for (int p = 0; p < 3; ++p) tmem_load<n>(column + p * c, o + p * n);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < n; ++i) {
              const float f = ct.scale[s][from + i], y = o[i] + (o[n + i] + o[2 * n + i] * 0.03125f);
              x[i] = s == 0 ? (f == 0.f ? 0.f : y * f) : (f == 0.f ? x[i] : fmaf(y, f, x[i]));
            }
          }
          put_rows(from, x, n);
        }
        tc_fence_before();
        named_barrier<1, 256>();  // both are through with O
        tc_fence_after();
      } else if (ok) {
        each_chunk<Sh::kChunks>([&](auto chunk) {
          constexpr int c = decltype(chunk)::value, n = Sh::rows_of(c);
          if (r0 + 16 * c >= rows) return;
          float o[3 * n];
#pragma unroll
          for (int p = 0; p < 3; ++p) tmem_load<n>(t_o + Sh::o_column(h, c) + p * n, o + p * n);
          tmem_wait_ld();
#pragma unroll
          for (int i = 0; i < n; ++i) o[i] = (o[i] + (o[n + i] + o[2 * n + i] * 0.03125f)) * ct.scale[h][16 * c + i];
          put_rows(r0 + 16 * c, o, n);
        });
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&ct.q_empty[buffer]));
      if (!whole && h == 0 && pc.k0 == 0) unit = JoinUnit{pc.pieces, rows, rows, pc.row0 + pc.i0, pc.head * G, G, {0, 0}};
    }
    if (tid == kBase) a.units[blockIdx.x] = unit;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 4) tmem_dealloc(tmem, 512);
}

template <int DP, int R>
cudaError_t launch(TcParams& p, const DeviceInfo& dev, cudaStream_t stream) {
  using Sh = TcShape<DP, R>;
  const AttendArgs& a = p.a;
  const retrace_kv_cache& c = a.cache;
  p.shape.unit_tokens = Sh::kRows / p.group;
  CUtensorMap mk, mv;
  const long long dims[4] = {c.head_dim, c.kv_heads, c.page_size, c.num_pages};
  const long long strides[4] = {1, c.head_stride, c.slot_stride, c.page_stride};
  const int box[4] = {DP, 1, p.kv_box, 1};
  const CUtensorMapSwizzle swizzle = DP == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B;
  // A row of a head is all that lies together: what L2 would fetch beyond it is another head's.
  const CUtensorMapL2promotion promotion = DP == 128 ? CU_TENSOR_MAP_L2_PROMOTION_L2_128B : CU_TENSOR_MAP_L2_PROMOTION_L2_64B;
  if (!encode(&mk, c.k, 4, dims, strides, box, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, swizzle, promotion) ||
      !encode(&mv, c.v, 4, dims, strides, box, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, swizzle, promotion))
    return cudaErrorInvalidValue;
  constexpr size_t smem = Sh::kControl + sizeof(Control<R>);
  static_assert(smem <= 227 * 1024, "shared memory of a CTA");
  static std::atomic<uint64_t> allowed{0};
  cudaError_t e = allow_shared(attend_fp8_tc_kernel<DP, R>, smem, dev, allowed);
  if (e != cudaSuccess) return e;
  const int grid = dev.sm_count < kAttendMaxTcCtas ? dev.sm_count : kAttendMaxTcCtas;
  e = launch_dependent(attend_fp8_tc_kernel<DP, R>, dim3(grid), dim3(Sh::kThreads), smem, stream, 1u, mk, mv, p);
  if (e != cudaSuccess) return e;
  return launch_attend_join(a, PartShape{Sh::kRows, DP, 1.f}, grid, stream);
}

template <int DP>
cudaError_t launch_rows(TcParams& p, const DeviceInfo& dev, cudaStream_t stream) {
  // By the rows that a sequence has on average; a group of query heads is never divided.
  const long long rows = (long long)p.a.T * p.group, B = p.a.B;
  if (p.group <= 8 && rows <= 8 * B) return launch<DP, 8>(p, dev, stream);
  if (p.group <= 16 && rows <= 16 * B) return launch<DP, 16>(p, dev, stream);
  if (p.group <= 32 && rows <= 32 * B) return launch<DP, 32>(p, dev, stream);
  return launch<DP, 24>(p, dev, stream);
}

}  // namespace

bool attend_fp8_tc_supported(const AttendArgs& a) {
  const retrace_kv_cache& c = a.cache;
  auto whole = [](long long x, int n) { return x % n == 0; };
  auto stride = [&](long long x, int extent) { return extent <= 1 || (x > 0 && whole(x, 16)); };
  return a.dtype == RETRACE_BF16 && c.head_dim <= 128 && whole(c.head_dim, 4) && whole(c.page_size, 8) && c.num_pages > 0 &&
         a.q_heads / c.kv_heads <= 72 && stride(c.page_stride, c.num_pages) && stride(c.slot_stride, c.page_size) &&
         stride(c.head_stride, c.kv_heads) && whole(a.q_token, 4) && whole(a.q_head, 4) && ((uintptr_t)a.q & 7u) == 0 &&
         (((uintptr_t)c.k | (uintptr_t)c.v) & 15u) == 0;
}

size_t attend_fp8_tc_partial_bytes(int head_dim) {
  if (head_dim > 128) return 0;
  return (size_t)kAttendMaxTcCtas * 2 * (head_dim <= 64 ? TcShape<64, 24>::kPart : TcShape<128, 24>::kPart) * 4;
}

cudaError_t launch_attend_fp8_tc(const AttendArgs& a, cudaStream_t stream) {
  DeviceInfo dev;
  const cudaError_t e = device_info(&dev);
  if (e != cudaSuccess) return e;
  TcParams p{};
  p.a = a;
  const retrace_kv_cache& c = a.cache;
  p.group = a.q_heads / c.kv_heads;
  p.by_group = FastDivide::of(p.group);
  p.page_size = FastDivide::of(c.page_size);
  p.kv_box = gcd(c.page_size, kKeys);
  p.scale2 = a.scale * 1.4426950408889634f;
  p.shape.q_start = a.q_start;
  p.shape.cache_len = a.cache_len;
  p.shape.B = a.B;
  p.shape.T = a.T;
  p.shape.uniform = a.q_start ? 0 : a.T / a.B;
  p.shape.kv_heads = c.kv_heads;
  p.shape.causal = a.causal;
  p.shape.window = a.window;
  p.shape.sinks = a.sinks;
  p.shape.places = c.max_pages * c.page_size;
  return c.head_dim <= 64 ? launch_rows<64>(p, dev, stream) : launch_rows<128>(p, dev, stream);
}

}  // namespace retrace
