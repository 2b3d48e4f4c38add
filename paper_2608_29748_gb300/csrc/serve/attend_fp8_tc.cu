// Attention over a cache in 8 bits on the tensor cores (bf16 queries).
//
// The keys are on the M side: per tile of 128 keys and up to 72 rows (query tokens times the
// heads of a group) a CTA computes, all products in 8 bits with fp32 accumulation,
//     S^T = K Q^T      [keys, rows]: K as it lies in the cache; a query is the sum of two e4m3 numbers
//                      (its leading 4 bits and the other 4), products of their own into the same sum;
//     t = scale S 2^ke, p = 2^(t + ve - m), l += p 2^-ve       a key's exponents ke and ve (from the
//                      unit that O counts in) are its thread's: one thread per key and 8 to 32 rows;
//     O^T += V^T P^T   [head dim, rows]: V as it lies; a weight is the sum of three e5m2 numbers of 3
//                      bits each, in columns of their own.
// e5m2 is the upper byte of an fp16 number, so the first part of a weight is a byte of it and the second
// a byte of what is left, times 4; the last, times 32, is rounded: down to 2^-13 off by at most 2^-9 and 2^-11
// of it (two roundings), and by 2^-21.8 below.  m puts the largest weight of a row's first tile at 2^3 to 2^4 and is
// raised, O and l rescaled, when a weight passes 2^15: so that is 2^-24 of the row's largest.  (From few keys, a window's
// sinks, m could be set lower, as larger scores may follow: window-tokens took 83 us with up to 2^7.  But sinks are
// kept because they have most of the weight, and what is lost of the others below them counts: 3 % of all weight under
// one sink 12.5 above 8192 equal scores.  Instead a window's sinks come last: 96 us, 107 with the sinks first.  At 2^7
// more rows are raised later: block-16k 424 us where 2^4 takes 377.)
// One page in a much larger unit would push all other pages' weights out of that range, whatever it holds: one
// rejected token of huge values makes such a page.  So the product has the pages within 2^3 of the unit that O counts in
// (2^-24 becomes 2^-18 at its ends); it moves to where most pages of a tile are.  The keys of others count in sums of their
// own, in fp32 on the CUDA cores, a column of TMEM to a row.  64 blocks of 17 over 4096, 32 / 8 heads of 128: 183 us, with one
// page apart in each sequence 240, one in each tile 860; all pages anywhere within 2^17 1690.  Tiles of the second kind, which
// also look for pages that are missing, have code of their own: inside the usual tile's it made that slower
// (window-tokens, sinks first, 106 -> 123 us).
// Nothing is converted but the queries, once, and the weights: keys and values go from HBM to shared
// memory to the tensor core, 256 D bytes a tile, 1400 cycles of an SM's share of HBM at D = 128.  The
// products are 4 (2 rows + 3 rows) cycles at D = 128, shared memory moves some 1100 cycles' worth at
// 72 rows, and the softmax does 128 rows exponentials: with few rows on the N side all of
// it scales with the rows that there are.
// A tile of D = 128 and 16-slot pages takes an SM 705 ns with 4 or 8 rows, 730 with 16, 750 with 32 (7.0 to 6.6 TB/s:
// bound by HBM), 980 ns with 48 and 1155 with 68 (4.3 TB/s): there the issue slots are 52 % taken and the tensor
// cores 27 %; a third of the warps' time is the chain of a tile (scores from TMEM, the group's agreement, exponentials,
// parts) without another one to fill it.  A unit costs 2.7 us (4 to 16 rows), 4.6 us (32) or 7 us (48, 68) besides its tiles.
//
// Warps of a CTA: copies of K and of V (TMA boxes of the slots of a page), the products, the queries
// (taken apart a piece ahead), and the softmax in groups of four warps, a thread to a key.  Up to 32
// rows a CTA has one group, and an SM two CTAs: a tile's way through the softmax, and the beginning
// and end of a piece, are latencies, and the other CTA works meanwhile.  Up to 72 rows three groups
// have 24 rows each, an SM one CTA, and the products two warps, the queries four.
//
// CTAs take the heads one after another, all sequences under each: then a sequence's heads, whose rows
// of 128 bytes lie side by side, are read by several CTAs at about the same time, and not by one in turn.
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
constexpr float kFirstTop = 4.f, kMostTop = 15.f;
constexpr float kNone = 3.402823466e38f;  // in place of the reference of a row that has seen nothing
constexpr float kFar = 4194304.f;         // 2^22: references up to it are whole numbers, and sums of two are exact
// Exponents of 2^10 and more lose places of a weight.  From 2^28 on what the rounding left is not counted: neighbouring
// scores are 32 apart there.
constexpr float kLarge = 1024.f, kHuge = 268435456.f;
// A factor times the largest unit of keys would leave fp32, and a score of zero times that is no number: the factor is
// multiplied by last.
constexpr float kLargeFactor = 1.2e24f;  // 2^80
constexpr int kNoPage = -1000;  // in place of a box's exponent
// Values whose exponent is within [unit - kBelow, unit + kAbove] are in the product.
constexpr int kBelow = 3, kAbove = 3;

struct TcParams {
  AttendArgs a;
  AttendShape shape;  // unit_tokens: of a row tile
  int group;          // query heads of a key/value head
  FastDivide by_group, page_size;
  int kv_box;   // slots of a box: they lie within a page and divide a tile
  float scale2;  // scale log2(e)
};

// R rows to a thread of the softmax, in chunks of 16 (the last may be of 8).
template <int DP, int R>
struct TcShape {
  static constexpr int kGroups = R == 24 ? 3 : 1;
  static constexpr bool kFew = kGroups == 1;
  static constexpr int kPerSm = kFew ? 2 : 1;
  static constexpr int kProducts = kFew ? 1 : 2, kQueries = kFew ? 1 : 4;   // warps
  static constexpr int kBase = kFew ? 128 : 256;                            // threads before the softmax's
  static constexpr int kThreads = kBase + 128 * kGroups;
  static constexpr int kRows = R * kGroups;
  static constexpr int kChunks = (R + 15) / 16;
  __host__ __device__ static constexpr int rows_of(int chunk) { return R - 16 * chunk < 16 ? R - 16 * chunk : 16; }
  // Columns of S: one a row, group after group, to a whole number of 16.
  static constexpr int kSColumns = (kRows + 15) / 16 * 16;
  // Columns of O (and of P): 3 a row; all groups' first chunks, then all second ones.
  __host__ __device__ static constexpr int o_column(int group, int chunk) { return 48 * kGroups * chunk + 3 * rows_of(chunk) * group; }
  static constexpr int kOColumns = (3 * kRows + 15) / 16 * 16;
  static_assert(kSColumns <= 256 && kOColumns <= 256, "columns of a product");
  static constexpr int kOAt = 2 * kSColumns, kTmem = 512 / kPerSm;
  static constexpr int kApartAt = kOAt + kOColumns;  // a column a row: what is not in the product
  static_assert(kApartAt + kRows <= kTmem, "columns of TMEM");
  // Registers of a thread: what the softmax takes of the others' of the launch.
  static constexpr int kFewer = kFew ? 64 : 56, kMore = kFew ? 192 : 120;
  static_assert(kBase * kFewer + 128 * kGroups * kMore <= kThreads * (65536 / (kThreads * kPerSm) / 8 * 8), "registers of a CTA");

  static constexpr int kTileBytes = kKeys * DP;
  static constexpr int kPWidth = kOColumns == 96 ? 32 : kOColumns > 64 ? 128 : kOColumns > 32 ? 64 : 32;  // bytes of a key's columns of P side by side
  static constexpr int kPBytes = (kOColumns + kPWidth - 1) / kPWidth * kKeys * kPWidth;
  static constexpr int kQPart = kSColumns * DP, kQBytes = (2 * kQPart + 1023) / 1024 * 1024;
  static constexpr int kControlBytes = kFew ? 7 * 1024 : 12 * 1024;
  static constexpr int kRoom = ((kFew ? 113 : 227) * 1024 - kControlBytes - 2 * kPBytes - 2 * kQBytes) / kTileBytes;
  static constexpr int kRingV = (kRoom + 1) / 2 < 8 ? (kRoom + 1) / 2 : 8, kRingK = kRoom / 2 < 8 ? kRoom / 2 : 8;
  static_assert(kRingK >= 2 && kRingV >= 2, "tiles in flight");
  static constexpr int kVAt = kRingK * kTileBytes, kPAt = kVAt + kRingV * kTileBytes, kQAt = kPAt + 2 * kPBytes;
  static constexpr int kControl = kQAt + 2 * kQBytes;
  static constexpr int kPart = kRows * (DP + 2);  // floats of a part
};

// A box's keys: scores are multiplied by k, values by 2^v.  Where no row sees the box, or it has no page, v is kNoPage.
struct BoxUnits {
  float k;
  int v;
};

template <int R, int kGroups>
struct Control {
  uint64_t full[2][8], empty[2][8];  // rings of K and V
  uint64_t q_full[2], q_empty[2];
  uint64_t s_full[2];   // scores ready
  uint64_t p_full[2];   // weights written, the scores' buffer read
  uint64_t pv_done[2];  // the product with V done, the weights' buffer free
  uint64_t done[2];     // after an expired wait: the issued products
  PlanStart plan;
  long long sum[20];
  uint32_t tmem;
  int abort;
  Piece piece[2];  // of the softmax, with its queries
  int more[2];     // 0: no piece, the end
  BoxUnits units[kInfoTiles][kMostBoxes];
  int2 span[kInfoTiles];  // largest and smallest v of the tile's boxes that are seen; the latter kNoPage if one has no page
  int large[2][4];     // some factor of a query warp's rows is
  alignas(16) float factor[2][R * kGroups];   // scale log2(e) times a row's unit
  long long out[2][R * kGroups];              // where a row goes, elements
  // Of a group's rows: what is added to exponents (minus the reference), and, where that is far from
  // zero, added to the difference; how the reference moves; what sums, and at the end O, are multiplied by.
  alignas(16) float minus[kGroups][R], rest[kGroups][R], move[kGroups][R], scale[kGroups][R];
  float part[kGroups][4][R];  // per warp: a row's maximum, or sum; of four keys: their weights
  uint32_t others[kGroups];   // boxes that are not in the product
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
// Rows of kWidth bytes with the swizzle of their width, 8 rows a group; `lead`: from one column of kWidth
// bytes to the next, for an MN-major operand.
template <int kWidth>
__device__ __forceinline__ uint64_t rows_desc(uint32_t saddr, uint32_t lead) {
  constexpr uint64_t mode = kWidth == 128 ? 2 : kWidth == 64 ? 4 : 6;
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
template <int kBy>
__device__ __forceinline__ uint32_t times(uint32_t a) {
  const __half2 h = __hmul2(*reinterpret_cast<const __half2*>(&a), __float2half2_rn((float)kBy));
  return *reinterpret_cast<const uint32_t*>(&h);
}
// Four fp16 numbers to e5m2, to the nearest, a byte each.
__device__ __forceinline__ uint32_t to_e5m2x4(uint32_t a, uint32_t b) {
  uint32_t y;
  asm("{\n\t.reg .b16 lo, hi;\n\t"
      "cvt.rn.satfinite.e5m2x2.f16x2 lo, %1;\n\t"
      "cvt.rn.satfinite.e5m2x2.f16x2 hi, %2;\n\t"
      "mov.b32 %0, {lo, hi};\n\t}"
      : "=r"(y)
      : "r"(a), "r"(b));
  return y;
}
// The three parts of four weights, none negative, a byte each; the second times 4, the third times 32.
__device__ __forceinline__ void take_apart(const float2& w0, const float2& w1, uint32_t& first, uint32_t& second, uint32_t& third) {
  const uint32_t a = halves(w0.x, w0.y), b = halves(w1.x, w1.y);
  const uint32_t a1 = times<4>(minus_halves(a, a & 0xFF00FF00u)), b1 = times<4>(minus_halves(b, b & 0xFF00FF00u));
  const uint32_t a2 = minus_halves(a1, a1 & 0xFF00FF00u), b2 = minus_halves(b1, b1 & 0xFF00FF00u);
  first = __byte_perm(a, b, 0x7531);
  second = __byte_perm(a1, b1, 0x7531);
  third = to_e5m2x4(times<8>(a2), times<8>(b2));
}

__device__ __forceinline__ void st_shared(uint32_t at, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
__device__ __forceinline__ void st_shared(uint32_t at, uint32_t x, uint32_t y) {
  asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(at), "r"(x), "r"(y) : "memory");
}

// The tiles of a unit in this kernel's order: the window's first, then the sinks'.  The first tile sets the references, and
// sinks show few keys.
__device__ __forceinline__ int tile_of(const UnitKeys& keys, int k) {
  const int window = keys.count - keys.sink_tiles;
  return k < window ? keys.first + k : k - window;
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
__global__ void __launch_bounds__(TcShape<DP, R>::kThreads, TcShape<DP, R>::kPerSm)
    attend_fp8_tc_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                         const __grid_constant__ TcParams P) {
  using Sh = TcShape<DP, R>;
  using Ct = Control<R, Sh::kGroups>;
  constexpr int kThreads = Sh::kThreads, kBase = Sh::kBase, kProducts = Sh::kProducts, kQueries = Sh::kQueries;
  static_assert(sizeof(Ct) <= Sh::kControlBytes, "room of the control block");
  extern __shared__ __align__(1024) uint8_t smem[];
  Ct& ct = *reinterpret_cast<Ct*>(smem + Sh::kControl);
  volatile int* abort = &ct.abort;
  const uint32_t base = smem_u32(smem);
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  const AttendArgs& a = P.a;

  if (tid == 0) {
    ct.abort = 0;
    for (int r = 0; r < 2; ++r)
      for (int s = 0; s < 8; ++s) {
        mbar_init(smem_u32(&ct.full[r][s]), 1);
        mbar_init(smem_u32(&ct.empty[r][s]), 1);
      }
    for (int s = 0; s < 2; ++s) {
      mbar_init(smem_u32(&ct.done[s]), 1);
      mbar_init(smem_u32(&ct.q_full[s]), kQueries);
      mbar_init(smem_u32(&ct.q_empty[s]), 1 + 4 * Sh::kGroups);  // the products, and the softmax warps
      mbar_init(smem_u32(&ct.s_full[s]), 1);
      mbar_init(smem_u32(&ct.p_full[s]), 4 * Sh::kGroups);
      mbar_init(smem_u32(&ct.pv_done[s]), 1);
    }
    fence_mbar_init();
    tma_prefetch_desc(&tm_k);
    tma_prefetch_desc(&tm_v);
  }
  if (warp == 3) {
    tmem_alloc(smem_u32(&ct.tmem), Sh::kTmem);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = ct.tmem;
  pdl_launch_dependents();
  pdl_wait();
  plan_start<kThreads, kKeys, true>(P.shape, gridDim.x, 2, &ct.plan, ct.sum);
  const PlanStart& plan = ct.plan;
  if (warp < kBase / 32) {
    fewer_registers<Sh::kFewer>();
    PieceWalk walk;
    walk.start(plan);
    Piece pc;
    bool ok = true, drain = false;
    if (warp < 2) {
      // ---- copies of K (warp 0) and V (1) ----
      // Lane (tile, box) looks up and copies a box of each of a batch of tiles.  A batch's pages are read
      // two batches ahead of its copies, their exponents one, whether it is of the same piece or not:
      // the warp never waits for what it has just asked for.
      const bool keys = warp == 0;
      const CUtensorMap* map = keys ? &tm_k : &tm_v;
      const int boxes = kKeys / P.kv_box, batch = min(32 / boxes, 8), my_tile = lane / boxes, box = lane % boxes;
      const uint32_t slots = keys ? Sh::kRingK : Sh::kRingV, tiles_at = base + (keys ? 0 : Sh::kVAt);
      uint32_t tiles = 0, slot = 0, phase = 0;
      struct Batch {
        int count;       // tiles; 0: no more
        int head, slot;  // slot: within the page
        int page;
        int ke, ve;
        bool seen;  // by a row of the unit
      };
      int nt = 0, k = 0;
      auto pages = [&]() {  // of the next batch
        Batch x{0, 0, 0, -1, 0, 0, false};
        while (k >= nt) {
          if (!walk.next<kKeys, false, true>(P.shape, plan, &pc)) return x;
          nt = pc.k1 - pc.k0;
          k = 0;
        }
        x.count = min(batch, nt - k);
        x.head = pc.head;
        if (my_tile < x.count) {
          const int j = tile_of(pc.keys, pc.k0 + k + my_tile) * kKeys + box * P.kv_box, i = P.page_size(j);
          x.slot = j - i * P.page_size.by;
          x.seen = j <= pc.keys.hi && (j + P.kv_box > pc.keys.lo || j < a.sinks);
          if (i < a.cache.max_pages) x.page = a.cache.page_table[pc.b * a.cache.table_stride + i];
        }
        k += batch;
        return x;
      };
      auto exponents = [&](Batch& x) {
        // a box without a page lies outside the tensor: zeros
        if (x.page < 0 || x.page >= a.cache.num_pages) x.page = a.cache.num_pages;
        if (keys && x.page < a.cache.num_pages) {
          const long long at = x.page * a.exp_page + x.head * a.exp_head;
          x.ke = a.k_exp[at];
          x.ve = a.v_exp[at];
        }
      };
      Batch now = pages();
      exponents(now);
      Batch next = pages();
      while (ok && now.count > 0) {
        exponents(next);
        const Batch after = pages();
        for (int t = 0; t < now.count; ++t) {
          ok = warp_wait_quick(&ct.empty[!keys][slot], phase ^ 1u, abort);
          if (!ok) break;
          const uint32_t bar = smem_u32(&ct.full[!keys][slot]);
          const bool active = my_tile == t;
          if (keys) {
            const bool there = active && now.page < a.cache.num_pages;
            const int v = there && now.seen ? clamp_exponent(now.ve) : kNoPage;
            if (active) ct.units[tiles % kInfoTiles][box] = BoxUnits{there ? power_of_two(clamp_exponent(now.ke)) : 1.f, v};
            const int hi = __reduce_max_sync(0xFFFFFFFFu, max(v, -kMostExponent));
            const int lo = __reduce_min_sync(0xFFFFFFFFu, active && now.seen ? v : kMostExponent);
            if (lane == 0) ct.span[tiles % kInfoTiles] = make_int2(hi, lo);
          }
          __syncwarp();
          if (lane == 0) mbar_arrive_expect_tx(bar, Sh::kTileBytes);
          __syncwarp();
          if (active)
            tma_load_4d(tiles_at + slot * Sh::kTileBytes + box * P.kv_box * DP, map, 0, now.head, now.slot, now.page, bar);
          if (++slot == slots) {
            slot = 0;
            phase ^= 1u;
          }
          ++tiles;
        }
        now = next;
        next = after;
      }
      drain = !ok;
    } else if (warp < 2 + kProducts) {
      // ---- products: scores (the first warp) and O (the second), or both (of one) ----
      // Issuing a tile's products and commits takes a warp some 1100 cycles for both.
      const bool does_scores = warp == 2, does_values = warp == 1 + kProducts;
      uint32_t tiles = 0, pieces = 0;
      auto wait = [&](uint64_t* bar, uint32_t parity) {
        ok = ok && warp_wait_quick(bar, parity, abort);
        return ok;
      };
      auto scores = [&](int i) {
        constexpr uint32_t kDesc = idesc_8bit(Sh::kSColumns, false);
        const uint32_t g = tiles + i, b = g & 1u, slot = g % Sh::kRingK;
        if (!wait(&ct.full[0][slot], g / Sh::kRingK & 1u)) return;
        // The product of two tiles ago is done: S has been read and the weights' buffer is free.  (A warp that
        // issues both has issued it before, and a commit waits for all that was issued before it.)
        if (kProducts == 2 && g >= 2 && !wait(&ct.pv_done[b], (g >> 1 & 1u) ^ 1u)) return;
        tc_fence_after();
        if (elect_one()) {
          const uint64_t kd = rows_desc<DP>(base + slot * Sh::kTileBytes, 16), qd = rows_desc<DP>(base + Sh::kQAt + (pieces & 1u) * Sh::kQBytes, 16);
#pragma unroll
          for (int k = 0; k < DP / 16; ++k) {  // the queries' leading parts, then what is left of them
            const int at = k % (DP / 32), part = k / (DP / 32);
            tc_mma_8bit(tmem + b * Sh::kSColumns, kd + 2 * at, qd + part * (Sh::kQPart >> 4) + 2 * at, kDesc, k > 0);
          }
          tc_commit(smem_u32(&ct.s_full[b]));
          tc_commit(smem_u32(&ct.empty[0][slot]));
        }
        __syncwarp();
      };
      auto values = [&](int i) {
        constexpr uint32_t kDesc = idesc_8bit(Sh::kOColumns, true);
        const uint32_t g = tiles + i, b = g & 1u, slot = g % Sh::kRingV;
        if (!wait(&ct.full[1][slot], g / Sh::kRingV & 1u) || !wait(&ct.p_full[b], g >> 1 & 1u)) return;
        tc_fence_after();
        if (elect_one()) {
          // 64 columns of the head dimension fill half of M: the other half is the same again
          const uint64_t vd = rows_desc<DP>(base + Sh::kVAt + slot * Sh::kTileBytes, 0);
          const uint64_t pd = rows_desc<Sh::kPWidth>(base + Sh::kPAt + b * Sh::kPBytes, kKeys * Sh::kPWidth);
#pragma unroll
          for (int k = 0; k < kKeys / 32; ++k)
            tc_mma_8bit(tmem + Sh::kOAt, vd + k * (32 * DP >> 4), pd + k * (32 * Sh::kPWidth >> 4), kDesc, i + k > 0);
          tc_commit(smem_u32(&ct.pv_done[b]));
          tc_commit(smem_u32(&ct.empty[1][slot]));
        }
        __syncwarp();
      };
      while (ok && walk.next<kKeys, false, true>(P.shape, plan, &pc)) {
        const int nt = pc.k1 - pc.k0;
        if (nt == 0) continue;
        if (does_scores && !wait(&ct.q_full[pieces & 1u], pieces >> 1 & 1u)) break;
        if constexpr (kProducts == 1) {
          scores(0);
          if (nt > 1) scores(1);
          for (int i = 0; i < nt && ok; ++i) {
            values(i);
            if (ok && i + 2 < nt) scores(i + 2);
          }
        } else {
          for (int i = 0; i < nt && ok; ++i)
            if (does_scores)
              scores(i);
            else
              values(i);
        }
        if (!ok) break;
        if (does_scores) {
          if (elect_one()) tc_commit(smem_u32(&ct.q_empty[pieces & 1u]));
          __syncwarp();
        }
        ++pieces;
        tiles += nt;
      }
      if (!ok) {
        volatile int never = 0;
        if (elect_one()) tc_commit(smem_u32(&ct.done[does_values]));
        __syncwarp();
        mbar_wait_bounded(smem_u32(&ct.done[does_values]), 0, &never);
      }
    } else {
      // ---- queries: rows of 128 or 64 bytes, each a sum of two e4m3 numbers times a unit ----
      // A lane has 16 elements of a row.
      constexpr int kLanes = DP / 16, kAtOnce = 32 / kLanes;
      constexpr int kSteps = (Sh::kRows + kQueries * kAtOnce - 1) / (kQueries * kAtOnce);
      const int which = warp - 2 - kProducts, D = a.cache.head_dim, col = lane % kLanes * 16;
      for (uint32_t pieces = 0;; ++pieces) {
        bool more;
        int rows;
        while ((more = walk.next<kKeys, true, true>(P.shape, plan, &pc))) {
          rows = (pc.i1 - pc.i0) * P.group;
          if (pc.k1 > pc.k0) break;
          for (int i = which * 32 + lane; i < rows * D; i += 32 * kQueries) {  // nothing is visible
            const int r = i / D, token = P.by_group(r);
            static_cast<__nv_bfloat16*>(a.out)[(long long)(pc.row0 + pc.i0 + token) * a.out_token +
                                               (pc.head * P.group + r - token * P.group) * (long long)a.out_head + i % D] = __float2bfloat16_rn(0.f);
          }
        }
        const uint32_t buffer = pieces & 1u;
        ok = warp_wait_quick(&ct.q_empty[buffer], (pieces >> 1 & 1u) ^ 1u, abort);
        if (!ok) break;
        if (lane == 0 && which == 0) {
          ct.piece[buffer] = pc;
          ct.more[buffer] = more;
        }
        if (!more) {
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&ct.q_full[buffer]));
          break;
        }
        uint8_t* to = smem + Sh::kQAt + buffer * Sh::kQBytes;
        auto row_of = [&](int step) { return (step * kQueries + which) * kAtOnce + lane / kLanes; };
        // Where the two parts of this lane's elements of row r go.
        auto place = [&](int r) { return to + r * DP + ((col / 16) ^ (DP == 128 ? r & 7 : r >> 1 & 3)) * 16; };
        // The row's largest magnitude, as bits: infinities and NaN are the largest.
        auto top_of = [&](const uint4 (&raw)[2]) {
          constexpr uint32_t kMagnitude = 0x7FFF7FFFu;
          uint32_t most = 0u;
#pragma unroll
          for (int i = 0; i < 2; ++i)
            most = __vmaxu2(__vmaxu2(most, __vmaxu2(raw[i].x & kMagnitude, raw[i].y & kMagnitude)), __vmaxu2(raw[i].z & kMagnitude, raw[i].w & kMagnitude));
#pragma unroll
          for (int o = 1; o < kLanes; o <<= 1) most = __vmaxu2(most, __shfl_xor_sync(0xFFFFFFFFu, most, o));
          return max(most & 0xFFFFu, most >> 16) << 16;
        };
        // The least exponent with a magnitude <= 448 times its power of two.
        auto exponent_of = [](uint32_t t) { return min(max((int)(t >> 23) - 127 - 8 + ((t & 0x7FFFFFu) > 0x600000u), -120), 120); };
        // A row's unit is its own: in a larger row's, 2^6 above it, elements 2^-5 of the row's largest would be
        // off by 2^-7 of themselves, and what a token gets would depend on what else is in its unit.
        bool large = false;
#pragma unroll 1
        for (int step = 0; step < kSteps; ++step) {
          const int r = row_of(step), token = P.by_group(r);
          uint4 raw[2] = {make_uint4(0u, 0u, 0u, 0u), make_uint4(0u, 0u, 0u, 0u)};
          const __nv_bfloat16* from = static_cast<const __nv_bfloat16*>(a.q) + (long long)(pc.row0 + pc.i0 + token) * a.q_token +
                                      (pc.head * P.group + r - token * P.group) * a.q_head + col;
          if (r < rows && col < D) raw[0] = *reinterpret_cast<const uint4*>(from);
          if (r < rows && col + 8 < D) raw[1] = *reinterpret_cast<const uint4*>(from + 8);
          const uint32_t top = top_of(raw);
          const int e = exponent_of(top);
          const float down = power_of_two(-e);
          uint32_t lead[4], rest[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t w[2] = {i == 0 ? raw[0].x : i == 1 ? raw[0].z : i == 2 ? raw[1].x : raw[1].z,
                                   i == 0 ? raw[0].y : i == 1 ? raw[0].w : i == 2 ? raw[1].y : raw[1].w};
            lead[i] = rest[i] = 0u;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const float x = bf16_lo(w[k]) * down, y = bf16_hi(w[k]) * down;
              const uint32_t c = to_e4m3x2(x, y);
              const float2 f = e4m3_floats(c);
              lead[i] |= c << (16 * k);
              rest[i] |= to_e4m3x2(x - f.x, y - f.y) << (16 * k);
            }
            if (top >= 0x7F800000u) lead[i] = 0x7F7F7F7Fu;  // an infinity or a NaN: NaN throughout, as its scores are
          }
          if (r < Sh::kRows) {
            uint8_t* at = place(r);
            *reinterpret_cast<uint4*>(at) = make_uint4(lead[0], lead[1], lead[2], lead[3]);
            *reinterpret_cast<uint4*>(at + Sh::kQPart) = make_uint4(rest[0], rest[1], rest[2], rest[3]);
            if (col == 0) {
              const float factor = fminf(fmaxf(P.scale2 * power_of_two(e), -kNone), kNone);
              ct.factor[buffer][r] = factor;
              large |= fabsf(factor) >= kLargeFactor;
              ct.out[buffer][r] = (pc.row0 + pc.i0 + token) * a.out_token + (pc.head * P.group + r - token * P.group) * a.out_head;
            }
          }
        }
        large = __any_sync(0xFFFFFFFFu, large);
        if (lane == 0) ct.large[buffer][which] = large;
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
    const int h = (warp - kBase / 32) / 4, key = tid & 127, quarter = warp & 3, r0 = h * R;
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
    const uint32_t t_o = tmem + lanes + Sh::kOAt, t_apart = tmem + lanes + Sh::kApartAt + r0;
    // This key's weights, with the swizzle of its row: a column of 16 bytes is one exclusive or away.
    const uint32_t my_weights = (base + Sh::kPAt + key * Sh::kPWidth) ^
                                (Sh::kPWidth == 128 ? key & 7 : Sh::kPWidth == 64 ? key >> 1 & 3 : key >> 2 & 1) * 16;
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
    for (;;) {
      const uint32_t buffer = pieces & 1u;
      const Piece& pc = ct.piece[buffer];
      wait(&ct.q_full[buffer], pieces >> 1 & 1u);
      const bool more = ok && ct.more[buffer];
      const int rows = more ? (pc.i1 - pc.i0) * G : 0;
      // A row of the tile that holds no token refers to a number that no weight comes near.
      if (key < R) {
        ct.minus[h][key] = r0 + key < rows ? kNone : -kNone;
        ct.rest[h][key] = 0.f;
      }
      // (after an expired wait the group leaves together)
      if (any_of_group(h, !more)) break;
      const int nt = pc.k1 - pc.k0;
      ++pieces;
      const float* factor = ct.factor[buffer] + r0;
      float2 l[R / 2];  // sums of this thread's keys
#pragma unroll
      for (int i = 0; i < R / 2; ++i) l[i] = make_float2(0.f, 0.f);
      bool far = false;  // some row's reference is far from zero, or its factor large
#pragma unroll
      for (int i = 0; i < kQueries; ++i) far |= ct.large[buffer][i] != 0;
      int o_unit = 0;      // O counts in 2^o_unit
      bool apart = false;  // something was not in the product
      const UnitKeys keys = pc.keys;
      const int first = pc.c + pc.i0, k0 = pc.k0;  // position of the unit's first token
      const bool idle = r0 >= rows;
      const int my_box = key / P.kv_box;
      // The tiles that begin in this range: not after the first token's last key less a tile, not before
      // the last token's first key.
      const int inner_hi = min(keys.hi, a.causal ? first : pc.c + pc.n - 1) - (kKeys - 1);
      const int inner_lo = a.window > 0 ? pc.c + pc.i1 - a.window : 0;

      // A tile; false: it needs care, and nothing has been done with it.
      auto tile = [&](auto care, int j) {
        constexpr bool kCare = decltype(care)::value;
        const uint32_t g = tiles + j, b = g & 1u;
        const int j0 = tile_of(keys, k0 + j) * kKeys;
        const bool inner = j0 >= inner_lo && j0 <= inner_hi;  // every row sees every key that has a page
        // Else the key is seen by the rows [from, to).
        int from = 0, to = R;
        if (!inner) {
          const int at = j0 + key;
          to = rows;
          if (a.causal && at > first) from = (at - first) * G;
          if (a.window > 0 && at >= a.sinks && at - first + a.window < P.shape.unit_tokens)
            to = max(at - first + a.window, 0) * G;
          if (at > keys.hi) to = 0;
          from -= r0;
          to -= r0;
        }
        wait(&ct.s_full[b], g >> 1 & 1u);
        tc_fence_after();
        const bool fresh = j == 0;
        const BoxUnits u = ct.units[g % kInfoTiles][my_box];
        const int2 span = ct.span[g % kInfoTiles];
        int now_unit = fresh ? span.x : o_unit;
        const bool wide = span.x > now_unit + kAbove || span.y < now_unit - kBelow;
        bool hides = !inner;
        uint32_t others = 0u;  // boxes that are not in the product
        if (kCare && wide) {
          // No row sees a key without a page (its score is zero times the query, which need not be a number).
          if (span.y == kNoPage) {
            hides = true;
            if (u.v == kNoPage) to = 0;
          }
          // The unit that most boxes fit; this one, if it is one of several.
          const int v = lane < kKeys / P.kv_box ? ct.units[g % kInfoTiles][lane].v : kNoPage;
          auto fitting = [&](int x) { return __ballot_sync(0xFFFFFFFFu, v != kNoPage && v <= x + kAbove && v >= x - kBelow); };
          uint32_t in = fitting(now_unit);
          for (int i = 0; i < kKeys / P.kv_box; ++i) {
            const int x = __shfl_sync(0xFFFFFFFFu, v, i);
            const uint32_t then = fitting(x);
            if (__popc(then) > __popc(in)) {
              in = then;
              now_unit = x;
            }
          }
          others = __ballot_sync(0xFFFFFFFFu, v != kNoPage) & ~in;
        }
        // Exponents of this key's weights: they are in the product as they are then, so that it counts in 2^now_unit.
        const int above = u.v - now_unit, shift = above <= kAbove ? max(above, -2 * kMostExponent) : 0;
        // A row of V that no row of the unit sees holds anything, and 0 times that need not be 0:
        // cleared before the product.
        const bool clears = !inner && h == 0 && (j0 < keys.lo || j0 + kKeys - 1 > keys.hi);
        // (the slot's phase before is over: the scores of this tile waited for a later product)
        if (clears || (kCare && others != 0u)) wait(&ct.full[1][g % Sh::kRingV], g / Sh::kRingV & 1u);
        if (clears) {
          const int at = j0 + key;
          if (at > keys.hi || (at < keys.lo && at >= a.sinks)) {
            uint8_t* v = smem + Sh::kVAt + (g % Sh::kRingV) * Sh::kTileBytes + key * DP;
#pragma unroll
            for (int c = 0; c < DP / 16; ++c)  // the lanes begin at different banks
              *reinterpret_cast<uint4*>(v + ((c + 2 * key) % (DP / 16)) * 16) = make_uint4(0u, 0u, 0u, 0u);
          }
        }
        if (!idle) {
          const uint32_t t_s = tmem + lanes + b * Sh::kSColumns + r0;
          const float2 unit2 = make_float2(u.k, u.k), shift2 = make_float2((float)shift, (float)shift);
          float y[R];  // exponents of the weights, then the weights
          auto hide = [&]() {
            if (!hides) return;
#pragma unroll
            for (int r = 0; r < R; ++r)
              if (r < from || r >= to) y[r] = -INFINITY;
          };
          // Scores, four rows at a time: f(row, two of them, two of them).
          auto scores = [&](auto&& f) {
            float s[R];
            each_chunk<Sh::kChunks>([&](auto chunk) {
              constexpr int c = decltype(chunk)::value;
              tmem_load<Sh::rows_of(c)>(t_s + 16 * c, s + 16 * c);
            });
            tmem_wait_ld();
#pragma unroll
            for (int r = 0; r < R; r += 4) f(r, make_float2(s[r], s[r + 1]), make_float2(s[r + 2], s[r + 3]));
            hide();
          };
          auto put = [&](int r, const float2& p, const float2& q) {
            y[r] = p.x;
            y[r + 1] = p.y;
            y[r + 2] = q.x;
            y[r + 3] = q.y;
          };
          struct Four {
            float2 p, q;
          };
          auto four = [](const float* from) {
            const float4 x = *reinterpret_cast<const float4*>(from);
            return Four{make_float2(x.x, x.y), make_float2(x.z, x.w)};
          };
          // For references far from zero: the product with the factor rounded, the reference taken off, and then
          // what the rounding left added.  `fresh`: rows without a reference keep their exponents.
          auto exact = [&](bool fresh) {
            auto one = [&](const float2& x, const float2& factor, float2 ref, const float2& rest) {
              if (fresh) {
                if (ref.x == kNone) ref.x = 0.f;
                if (ref.y == kNone) ref.y = 0.f;
              }
              const float2 t = mul2(x, unit2), m = mul2(t, factor);
              float2 left = fma2(t, factor, make_float2(-m.x, -m.y));
              if (fabsf(ref.x) >= kHuge) left.x = 0.f;
              if (fabsf(ref.y) >= kHuge) left.y = 0.f;
              return add2(add2(add2(m, ref), left), add2(shift2, rest));
            };
            scores([&](int r, const float2& x0, const float2& x1) {
              const Four factors = four(factor + r), rest = four(ct.rest[h] + r), ref = four(ct.minus[h] + r);
              put(r, one(x0, factors.p, ref.p, rest.p), one(x1, factors.q, ref.q, rest.q));
            });
          };
          auto exponents = [&]() {
            if (far)
              exact(false);
            else
              scores([&](int r, const float2& x0, const float2& x1) {
                const Four factors = four(factor + r), ref = four(ct.minus[h] + r);
                put(r, add2(fma2(x0, mul2(factors.p, unit2), ref.p), shift2), add2(fma2(x1, mul2(factors.q, unit2), ref.q), shift2));
              });
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
          // So does another unit of the values; and a tile that needs care, or has boxes that are not in the product, comes
          // by here, because the group agrees on it: after an expired wait its warps may have read different units.
          bool raise = fresh;
          if (!fresh) {
            exponents();
            float top = -INFINITY;
#pragma unroll
            for (int r = 0; r < R; r += 2) top = max3(top, y[r], y[r + 1]);
            // (the weights do not wait for the answer: exponents are worked out again where they move)
#pragma unroll
            for (int r = 0; r < R; ++r) y[r] = exp2_fast(y[r]);
            raise = any_of_group(h, top > kMostTop || (kCare ? now_unit != o_unit || others != 0u : wide));
          }
          bool some_apart = false;
          if (__builtin_expect(raise, false)) {
            if (key == 0) ct.others[h] = kCare ? others : wide;
            if (fresh && !far)
              scores([&](int r, const float2& x0, const float2& x1) {
                const Four factors = four(factor + r);
                put(r, fma2(x0, mul2(factors.p, unit2), shift2), fma2(x1, mul2(factors.q, unit2), shift2));
              });
            else
              exact(true);
            maxima();
            some_apart = ct.others[h] != 0u;
            if (!kCare && some_apart) {
              group_barrier(h);  // all have read it
              return false;
            }
            float old = 0.f, old_rest = 0.f, now = 0.f, now_rest = 0.f, move = 0.f;
            bool pending = false;
            if (key < R) {
              old = now = ct.minus[h][key];
              old_rest = now_rest = ct.rest[h][key];
              const float most = most_of(key), by = floorf(kFirstTop - most);
              if (old == kNone ? most > -INFINITY : most > kMostTop) {
                const float from_zero = old == kNone ? 0.f : old;
                if (fabsf(from_zero) >= kFar && fabsf(old_rest + by) < kFar) {
                  now_rest = old_rest + by;
                  move = by;
                } else if (fabsf(from_zero) < kFar && fabsf(from_zero + by) < kFar) {
                  now = from_zero + by;
                  move = by;
                } else {  // the maximum itself, and what is left of it over the tile
                  now = (from_zero + old_rest) - most;
                  now_rest = 0.f;
                  pending = true;
                }
                ct.minus[h][key] = now;
                ct.rest[h][key] = now_rest;
              }
              ct.move[h][key] = move;
            }
            const bool again = any_of_group(h, pending || fabsf(move) >= kLarge);
            if (again) {
              far = true;
              // (a maximum that moves by more than its own places takes another turn)
              for (int turn = 0;; ++turn) {
                exact(false);
                maxima();
                if (pending) {
                  const float most = most_of(key);
                  pending = fabsf(most) >= kFar && turn < 2;
                  if (pending)
                    ct.minus[h][key] = now -= most;
                  else
                    ct.rest[h][key] = now_rest = floorf(kFirstTop - most);
                }
                if (!any_of_group(h, pending)) break;
              }
            }
            if (key < R) ct.scale[h][key] = old == kNone ? 0.f : exp2_fast((now - old) + (now_rest - old_rest));
            group_barrier(h);
            if (!fresh) {
#pragma unroll
              for (int r = 0; r < R; r += 2) l[r / 2] = mul2(l[r / 2], *reinterpret_cast<const float2*>(ct.scale[h] + r));
              const float carry = kCare ? power_of_two(o_unit - now_unit) : 1.f;
              const uint32_t before = g - 1;
              wait(&ct.pv_done[before & 1u], before >> 1 & 1u);
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
                  for (int i = 0; i < n; ++i) o[i] *= ct.scale[h][16 * c + i] * carry;
#pragma unroll
                  for (int i = 0; i < n; i += 4) tmem_store4(column + i, o + i);
                }
              });
              if (kCare && apart)
#pragma unroll 1
                for (int r = 0; r < R; r += 8) {
                  float o[8];
                  tmem_load<8>(t_apart + r, o);
                  tmem_wait_ld();
#pragma unroll
                  for (int i = 0; i < 8; ++i) o[i] *= ct.scale[h][r + i];
                  tmem_store4(t_apart + r, o);
                  tmem_store4(t_apart + r + 4, o + 4);
                }
              tmem_wait_st();
            }
            if (again) {
              exact(false);
            } else {
#pragma unroll
              for (int r = 0; r < R; r += 4) {
                const Four move = four(ct.move[h] + r);
                put(r, add2(make_float2(y[r], y[r + 1]), move.p), add2(make_float2(y[r + 2], y[r + 3]), move.q));
              }
            }
#pragma unroll
            for (int r = 0; r < R; ++r) y[r] = exp2_fast(y[r]);
          }

          const uint32_t weights = my_weights + b * Sh::kPBytes;
          const float inv = power_of_two(-shift);
          const float2 inv2 = make_float2(inv, inv);
          auto put_weights = [&](auto chunk, const uint32_t* w) {
            constexpr int c = decltype(chunk)::value, n = Sh::rows_of(c);
            const int column = Sh::o_column(h, c);
#pragma unroll
            for (int i = 0; i < 3; ++i) {
              const int x = column + i * n;
              const uint32_t at_w = (weights ^ (uint32_t)(x % Sh::kPWidth / 16 * 16)) + x / Sh::kPWidth * (kKeys * Sh::kPWidth) + x % 16;
              if constexpr (n == 16)
                st_shared(at_w, w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
              else
                st_shared(at_w, w[2 * i], w[2 * i + 1]);
            }
          };
          each_chunk<Sh::kChunks>([&](auto chunk) {
            constexpr int c = decltype(chunk)::value, n = Sh::rows_of(c);
            uint32_t w[3 * n / 4];
#pragma unroll
            for (int i = 0; i < n; i += 4) {
              const float2 p = make_float2(y[16 * c + i], y[16 * c + i + 1]), q = make_float2(y[16 * c + i + 2], y[16 * c + i + 3]);
              l[(16 * c + i) / 2] = fma2(p, inv2, l[(16 * c + i) / 2]);
              l[(16 * c + i) / 2 + 1] = fma2(q, inv2, l[(16 * c + i) / 2 + 1]);
              take_apart(p, q, w[i / 4], w[n / 4 + i / 4], w[2 * (n / 4) + i / 4]);
            }
            put_weights(chunk, w);
          });

          // Keys that are not in the product, four at a time: their weights through shared memory, and this thread's
          // element of their values, in fp32.
          if (kCare && some_apart) {
            if (ct.others[h] >> my_box & 1u)
              each_chunk<Sh::kChunks>([&](auto chunk) {
                const uint32_t none[12] = {};
                put_weights(chunk, none);
              });
            if (!apart) {
              const float zero[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
              for (int r = 0; r < R; r += 4) tmem_store4(t_apart + r, zero);
              tmem_wait_st();
              apart = true;
            }
            const uint8_t* values = smem + Sh::kVAt + (g % Sh::kRingV) * Sh::kTileBytes;
            const int element = key % DP;
#pragma unroll 1
            for (uint32_t left = ct.others[h]; left != 0u; left &= left - 1u) {
              const int box = __ffs(left) - 1;
              const float value_unit = power_of_two(ct.units[g % kInfoTiles][box].v);
#pragma unroll 1
              for (int four_at = box * P.kv_box; four_at < (box + 1) * P.kv_box; four_at += 4) {
                if (key / 4 == four_at / 4) {
#pragma unroll
                  for (int r = 0; r < R; ++r) ct.part[h][key % 4][r] = y[r] * inv;
                }
                group_barrier(h);
                float v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  const int k = four_at + i, at = j0 + k;
                  const bool seen = at <= keys.hi && (at >= keys.lo || at < a.sinks);
                  const uint32_t code = values[k * DP + ((element / 16) ^ (DP == 128 ? k & 7 : k >> 1 & 3)) * 16 + element % 16];
                  v[i] = seen ? e4m3_floats(code).x * value_unit : 0.f;
                }
#pragma unroll 1
                for (int r = 0; r < R; r += 8) {
                  float o[8];
                  tmem_load<8>(t_apart + r, o);
                  tmem_wait_ld();
#pragma unroll
                  for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int x = 0; x < 8; ++x) o[x] += ct.part[h][i][r + x] * v[i];
                  tmem_store4(t_apart + r, o);
                  tmem_store4(t_apart + r + 4, o + 4);
                }
                tmem_wait_st();
                group_barrier(h);
              }
            }
          }
        }
        o_unit = now_unit;
        fence_proxy_async_shared();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&ct.p_full[b]));
        return true;
      };
      int j = 0;
      while (j < nt && tile(Index<0>{}, j)) ++j;
      for (; j < nt; ++j) tile(Index<1>{}, j);
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
      group_barrier(h);
      const bool whole = pc.pieces == 1;
      float* part = a.partials + ((long long)blockIdx.x * 2 + (pc.k0 == 0 ? 1 : 0)) * Sh::kPart;
      auto sum_of = [&](int s, int r) { return (ct.part[s][0][r] + ct.part[s][1][r]) + (ct.part[s][2][r] + ct.part[s][3][r]); };
      if (key < R) {
        // What O is multiplied by, so that it refers to m: to a number, where minus and rest are two.
        const float m = -(ct.minus[h][key] + ct.rest[h][key]);
        const float f = exp2_fast(-((ct.minus[h][key] + m) + ct.rest[h][key])), sum = sum_of(h, key) * f;
        ct.scale[h][key] = (whole ? (sum == 0.f ? 0.f : f / sum) : f) * power_of_two(o_unit);
        if (!whole && ok && r0 + key < rows)
          *reinterpret_cast<float2*>(part + Sh::kRows * DP + (r0 + key) * 2) = make_float2(sum == 0.f ? -INFINITY : m, sum);
      }
      group_barrier(h);
      // O is complete
      if (ok) {
        const uint32_t last = tiles - 1;
        wait(&ct.pv_done[last & 1u], last >> 1 & 1u);
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
      if (ok) {
        each_chunk<Sh::kChunks>([&](auto chunk) {
          constexpr int c = decltype(chunk)::value, n = Sh::rows_of(c);
          if (r0 + 16 * c >= rows) return;
          float o[3 * n];
#pragma unroll
          for (int p = 0; p < 3; ++p) tmem_load<n>(t_o + Sh::o_column(h, c) + p * n, o + p * n);
          tmem_wait_ld();
#pragma unroll
          for (int i = 0; i < n; ++i) o[i] = o[i] + (o[n + i] * 0.25f + o[2 * n + i] * 0.03125f);
          if (apart) {
            const float down = power_of_two(-o_unit);
            tmem_load<n>(t_apart + 16 * c, o + n);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < n; ++i) o[i] += o[n + i] * down;
          }
#pragma unroll
          for (int i = 0; i < n; ++i) o[i] *= ct.scale[h][16 * c + i];
          put_rows(r0 + 16 * c, o, n);
        });
      }
      if (!whole && h == 0 && pc.k0 == 0) unit = JoinUnit{pc.pieces, rows, rows, pc.row0 + pc.i0, pc.head * G, G, {0, 0}};
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&ct.q_empty[buffer]));
    }
    if (tid == kBase) a.units[blockIdx.x] = unit;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 3) tmem_dealloc(tmem, Sh::kTmem);
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
  constexpr size_t smem = Sh::kControl + sizeof(Control<R, Sh::kGroups>);
  static_assert(smem <= (Sh::kFew ? 113 : 227) * 1024, "shared memory of a CTA");
  static std::atomic<uint64_t> allowed{0};
  cudaError_t e = allow_shared(attend_fp8_tc_kernel<DP, R>, smem, dev, allowed);
  if (e != cudaSuccess) return e;
  const int grid = Sh::kPerSm * (dev.sm_count < kAttendMaxTcCtas ? dev.sm_count : kAttendMaxTcCtas);
  static_assert(2 * kAttendMaxTcCtas <= kAttendMaxCtas, "entries of the CTAs");
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
  return a.dtype == RETRACE_BF16 && c.head_dim <= 128 && whole(c.head_dim, 8) && whole(c.page_size, 8) && c.num_pages > 0 &&
         a.q_heads / c.kv_heads <= 72 && stride(c.page_stride, c.num_pages) && stride(c.slot_stride, c.page_size) &&
         stride(c.head_stride, c.kv_heads) && whole(a.q_token, 8) && whole(a.q_head, 8) &&
         (((uintptr_t)a.q | (uintptr_t)c.k | (uintptr_t)c.v) & 15u) == 0;
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
  p.scale2 = std::min(std::max(a.scale * 1.4426950408889634f, -kNone), kNone);  // finite, as scale is
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
