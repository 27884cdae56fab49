// Attention of packed chunks or draft trees with a window, over a bf16 cache or one of e4m3 codes with a scale for each block of slots and head.
//
//   out[t] = sum_j softmax_j(z[t, j]) v[j],  z = scale * q[t].k[j],  over the slots j that token t sees.
//
// Planner and merge are those of chunk.cu.  So is the structure of the tile kernel in this file: a cluster of two CTAs works on two neighbouring
// query tiles of 128 rows over the same K/V tiles, with MMAs of 256 rows (cta_group::2) for which each CTA holds half of every
// K tile (64 keys) and of every V tile (64 of 128 columns); three score buffers in tensor memory, two softmax groups of four warps that take
// alternate steps and share one reference per row, P in place of its scores.  What differs:
//
// The plan leaves out K/V tiles between the sinks and the window of a unit, and rows mask what is left of the gap (and a tree's rows what is
// not on their path) in tensor memory, on tiles that some row does not see whole.
//
// Codes come through a ring of their own and are widened to fp16 (exactly) into the swizzled tiles that the MMAs read, by four warps between
// the copies and the MMAs: each CTA widens its halves, 16 K numbers a step.  Scales stay in fp32, outside of the products: the scores of 16 keys
// take ks * scale as their factor, and the maximum is taken over z + log2 vs, so that 2^(z + log2 vs - m) is the weight of
// the codes themselves and fits fp16 whatever the scales are; the row sum divides by vs again.  Query rows are multiplied by a power of two, so that they fit
// fp16 as well, and the scores by its inverse.  A warp brings the scales of each step's 128 keys.
#include "window.cuh"

namespace eagle {

namespace {

using namespace tc;

constexpr int kSBufs = 3;                // score buffers in tensor memory; step g uses buffer g % 3
constexpr uint32_t kTmemCols = 512;      // S0 S1 S2 | O; P (packed, 64 columns) overwrites the front of its S
constexpr uint32_t kColO = 384;
constexpr float kRescaleThreshold = 8.0f;   // log2 units: the accumulator is rescaled when the row maximum outgrows its reference by more
constexpr int kPolyStride = 2;           // bf16: one pair of exponentials in so many is a polynomial on the FMA pipe (measured in chunk.cu)
constexpr int kGroups = kChunkTile / 16; // groups of 16 keys in a tile, the smallest block

template <int D, bool CODES>
struct Roles {
  // two softmax groups of four warps; the widening warps (codes); copies; a relay (bf16: V tiles that have landed; codes: scales); two
  // MMA issuers (the second CTA's pass on what its widening warps have done)
  static constexpr int kConv = 8, kProducer = CODES ? 12 : 8, kRelay = kProducer + 1, kQK = kProducer + 2, kPV = kProducer + 3;
  static constexpr int kThreads = 32 * (kPV + 1);
};

template <int D, bool CODES>
struct Smem {
  static constexpr int kKSlots = CODES ? 3 : 5, kVSlots = CODES ? 3 : 4;     // rings of half tiles that the MMAs read
  static constexpr int kKStages = 4, kVStages = 3;           // and of half tiles of codes
  // (the two warps that widen K tiles take every other step each, those of V likewise)
  static_assert(!CODES || (kKStages % 2 == 0 && kVStages == kVSlots), "a stage belongs to one warp, or its tile's turn tells its uses apart");
  static constexpr int kFactors = 5;                         // items whose rows' factors are kept: the MMAs are three steps ahead of the softmax, the widening two items ahead of them
  static constexpr int kSlabs = D / 64;                      // 64 16-bit numbers = one 128-byte swizzled row
  static constexpr int kQSlab = 128 * 128, kQBytes = kSlabs * kQSlab;
  static constexpr int kKSlab = 64 * 128, kKBytes = kSlabs * kKSlab;     // half a K tile: 64 keys
  static constexpr int kVBytes = 128 * D;                    // half a V tile: 128 keys x D / 2 columns
  static constexpr int kKCodes = 64 * D, kVCodes = 128 * D / 2;
  static constexpr int kQ = 0;                               // two query tiles: the current item's and the next one's
  static constexpr int kK = 2 * kQBytes;
  static constexpr int kV = kK + kKSlots * kKBytes;
  static constexpr int kKC = kV + kVSlots * kVBytes;
  static constexpr int kVC = kKC + (CODES ? kKStages * kKCodes : 0);
  static constexpr int kTag = kVC + (CODES ? kVStages * kVCodes : 0);        // uint64 [128 rows]: step number | reference maximum
  static constexpr int kLfin = kTag + 128 * 8;               // uint64 [2][128 rows]: item number | row sum on its way to the output, by items in turn
  static constexpr int kFactor = kLfin + 2 * 128 * 8;        // uint64 [kFactors][128 rows]: item number | the row's factor
  static constexpr int kScale = kFactor + (CODES ? kFactors * 128 * 8 : 0);  // float4 [kSBufs][kGroups]: ks * scale, log2 vs, 1 / vs
  static constexpr int kBar = kScale + (CODES ? kSBufs * kGroups * 16 : 0);
  static constexpr int kNumBars = CODES ? 2 * (kKStages + kVStages) + 3 * (kKSlots + kVSlots) + 8 + 3 * kSBufs + 1 : 2 * (kKSlots + 2) + 3 * kVSlots + 3 * kSBufs + 1;
  static constexpr int kMisc = (kBar + 8 * kNumBars + 15) / 16 * 16;         // tensor-memory base, abort flag, wait limit (8 bytes)
  static constexpr int kBytes = kMisc + 16;
  static_assert(kBytes <= 227 * 1024, "shared memory of an SM");
};

// The same places in both CTAs.  ready (first CTA only): a tile can be read by the MMAs, in both CTAs; full, done (codes): the second CTA's half has been widened,
// which one of its idle warps passes on; empty: the MMAs have finished with the slot (both CTAs).
template <int D, bool CODES>
struct Bars {
  using S = Smem<D, CODES>;
  uint32_t base;
  static constexpr uint32_t kVAt = 2 * S::kKSlots, kQAt = kVAt + 3 * S::kVSlots, kSAt = kQAt + 4, kCAt = kSAt + 3 * kSBufs + 1;
  static constexpr uint32_t kKStageAt = kCAt + S::kKSlots + 4, kVStageAt = kKStageAt + 2 * S::kKStages;
  __device__ __forceinline__ uint32_t at(uint32_t i) const { return base + 8u * i; }
  __device__ __forceinline__ uint32_t k_ready(uint32_t i) const { return at(i); }
  __device__ __forceinline__ uint32_t k_empty(uint32_t i) const { return at(S::kKSlots + i); }
  __device__ __forceinline__ uint32_t v_full(uint32_t i) const { return at(kVAt + i); }                  // bf16: the half has landed; codes: it has been widened
  __device__ __forceinline__ uint32_t v_ready(uint32_t i) const { return at(kVAt + S::kVSlots + i); }
  __device__ __forceinline__ uint32_t v_empty(uint32_t i) const { return at(kVAt + 2 * S::kVSlots + i); }
  __device__ __forceinline__ uint32_t q_ready(uint32_t i) const { return at(kQAt + i); }
  __device__ __forceinline__ uint32_t q_empty(uint32_t i) const { return at(kQAt + 2 + i); }
  __device__ __forceinline__ uint32_t s_full(uint32_t i) const { return at(kSAt + i); }                  // scores of a step (both CTAs)
  __device__ __forceinline__ uint32_t p_full(uint32_t i) const { return at(kSAt + kSBufs + i); }         // its probabilities (first CTA only)
  __device__ __forceinline__ uint32_t o_done(uint32_t i) const { return at(kSAt + 2 * kSBufs + i); }     // its PV has finished (both CTAs)
  __device__ __forceinline__ uint32_t o_free() const { return at(kSAt + 3 * kSBufs); }                   // an item's accumulators have been read (first CTA only)
  // codes alone
  __device__ __forceinline__ uint32_t k_done(uint32_t i) const { return at(kCAt + i); }
  __device__ __forceinline__ uint32_t q_full(uint32_t i) const { return at(kCAt + S::kKSlots + i); }     // a query tile has landed
  __device__ __forceinline__ uint32_t q_done(uint32_t i) const { return at(kCAt + S::kKSlots + 2 + i); }
  __device__ __forceinline__ uint32_t kc_full(uint32_t i) const { return at(kKStageAt + i); }
  __device__ __forceinline__ uint32_t kc_empty(uint32_t i) const { return at(kKStageAt + S::kKStages + i); }
  __device__ __forceinline__ uint32_t vc_full(uint32_t i) const { return at(kVStageAt + i); }
  __device__ __forceinline__ uint32_t vc_empty(uint32_t i) const { return at(kVStageAt + S::kVStages + i); }
};

__device__ __forceinline__ uint4 load_shared(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void store_shared(uint32_t addr, const uint4& v) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
// Sixteen codes as two vectors of eight fp16 numbers.
__device__ __forceinline__ void widen_codes(const uint4& c, uint4& lo, uint4& hi) {
  half_of_codes(c.x, lo.x, lo.y);
  half_of_codes(c.y, lo.z, lo.w);
  half_of_codes(c.z, hi.x, hi.y);
  half_of_codes(c.w, hi.z, hi.w);
}

template <int D, bool PAGED, bool CODES, bool STALL>       // (STALL: of the test hook, as in chunk.cu)
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(Roles<D, CODES>::kThreads, 1)
window_attn_kernel(ChunkParams p, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                   const __grid_constant__ CUtensorMap map_q) {
  using S = Smem<D, CODES>;
  using R = Roles<D, CODES>;
  constexpr int kKSlots = S::kKSlots, kVSlots = S::kVSlots;
  extern __shared__ __align__(1024) unsigned char smem[];
  const uint32_t sbase = smem_u32(smem);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = cluster_rank();
  if (sbase & 1023u) {   // the swizzled tiles need a 1024-byte aligned base; uniform over the launch
    if (tid == 0) report_status(p.status, EAGLE_ERR_DEVICE);
    return;
  }
  Bars<D, CODES> B;
  B.base = sbase + S::kBar;
  volatile uint32_t* s_tmem = reinterpret_cast<volatile uint32_t*>(smem + S::kMisc);
  volatile int* s_abort = reinterpret_cast<volatile int*>(smem + S::kMisc + 4);

  if (tid == 0) {
    prefetch_map(&map_k);
    prefetch_map(&map_v);
    prefetch_map(&map_q);
    for (int i = 0; i < kKSlots; ++i) { mbar_init(B.k_ready(i), CODES ? 2 : 1); mbar_init(B.k_empty(i), 1); }
    for (int i = 0; i < kVSlots; ++i) { mbar_init(B.v_full(i), 1); mbar_init(B.v_ready(i), 2); mbar_init(B.v_empty(i), 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(B.q_ready(i), CODES ? 3 : 1); mbar_init(B.q_empty(i), 1); }
    for (int i = 0; i < kSBufs; ++i) {
      mbar_init(B.s_full(i), CODES ? 2 : 1);       // (codes: the step's scales as well)
      mbar_init(B.p_full(i), 8);           // a group's four warps, in both CTAs
      mbar_init(B.o_done(i), 1);
    }
    mbar_init(B.o_free(), 8);
    if constexpr (CODES) {
      for (int i = 0; i < kKSlots; ++i) mbar_init(B.k_done(i), 1);
      for (int i = 0; i < 2; ++i) { mbar_init(B.q_full(i), 1); mbar_init(B.q_done(i), 2); }
      for (int i = 0; i < S::kKStages; ++i) { mbar_init(B.kc_full(i), 1); mbar_init(B.kc_empty(i), 1); }
      for (int i = 0; i < S::kVStages; ++i) { mbar_init(B.vc_full(i), 1); mbar_init(B.vc_empty(i), 1); }
    }
    *s_abort = 0;
    *reinterpret_cast<volatile unsigned long long*>(smem + S::kMisc + 8) = p.wait_limit_ns;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  for (int i = tid; i < (CODES ? 3 + S::kFactors : 3) * 128; i += R::kThreads)
    reinterpret_cast<volatile unsigned long long*>(smem + S::kTag)[i] = ~0ull;      // (kLfin and kFactor too) no step and no item has this number
  if (warp == R::kQK) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(sbase + S::kMisc), "r"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  fence_before();
  __syncthreads();
  cluster_sync();                          // both CTAs' barriers exist before either is arrived at from across
  fence_after();
  const uint32_t tmem = *s_tmem;

  launch_dependents();
  wait_for_prerequisites();                // the plan is there
  const int4 mine = p.work.cta[blockIdx.x >> 1];         // whole units first, then this pair's share of the rest
  const int n_items = mine.y + mine.w;
  struct Item {
    int b, g, part, start, n, L, t0, t1, slot;
  };
  auto item = [&](int i) {
    const int4* at = reinterpret_cast<const int4*>(p.work.items + (i < mine.y ? mine.x + i : mine.z + (i - mine.y)));
    const int4 a = at[0], b = at[1];
    return Item{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w, at[2].x};
  };
  auto span_of = [&](const Item& it) { return chunk_span(p, it.L, it.part * p.ut); };

  if (warp >= R::kConv) {
    if (warp == R::kProducer) {
      // =========================================================================== copies
      // Order: K(0), K(1), K(2), then V(g), K(g + 3), g counting this pair's steps over all items (the score MMA runs up to three
      // steps ahead of the PV MMA); an item's query tile goes with its first K tile.  Each CTA's producer fetches its own halves.  bf16: K
      // and query tiles report to the first CTA's barrier, V tiles to the relay of their own CTA; codes: all report to the widening warps of their
      // own.  A lane per box (a page, or a 64-column half); the page of a lane's next box is looked up while the box before it is on its way.
      struct Cursor {
        Item it;
        ChunkSpan span;
        int i, tile, end;
        int y, page;                         // this lane's next box: row in its page (or in the sequence), page (or sequence)
        bool valid, fresh;
        bool wrong;                          // some entry of the item was outside the pool
      };
      constexpr int kKLanes = CODES ? 1 : S::kSlabs;       // lanes to a K box's rows
      const int k_rows = PAGED ? min(p.page_size, 64) : 64, v_rows = PAGED ? min(p.page_size, kChunkTile) : kChunkTile;
      const int k_r0 = (lane / kKLanes) * k_rows, v_r0 = lane * v_rows, half = static_cast<int>(rank);
      auto advance = [&](Cursor& c, bool is_v) {        // to the next K/V tile of the work list
        c.fresh = false;
        if (++c.tile >= c.end) {
          if (PAGED && c.wrong) p.work.bad_page[c.it.b] = 1;
          c.wrong = false;
          for (++c.i; c.i < n_items; ++c.i) {
            c.it = item(c.i);
            if (c.it.t1 > c.it.t0) break;
          }
          if (c.i >= n_items) {
            c.valid = false;
            return;
          }
          c.span = span_of(c.it);
          c.tile = c.it.t0;
          c.end = c.it.t1;
          c.fresh = true;
        }
        const int r0 = is_v ? v_r0 : k_r0, key = c.span.tile(c.tile) * kChunkTile + (is_v ? 0 : half * 64) + r0;
        c.y = key;
        c.page = c.it.b;
        if (PAGED && r0 < (is_v ? kChunkTile : 64)) {
          // a box past the sequence's last page fetches that page again (its rows are masked), so that a tile's byte count never changes
          const int last = (c.it.L + c.it.n - 1) >> p.page_shift, pi = key >> p.page_shift;
          c.page = __ldg(p.block_table + static_cast<size_t>(c.it.b) * p.max_pages + c.span.page(pi < last ? pi : last, p.page_shift));
          c.y = key & (p.page_size - 1);
        }
      };
      // an entry outside the pool reads page 0, and marks its sequence when the item ends (the merge kernel reports it and zeroes the rows)
      auto place = [&](Cursor& c) {
        const bool wrong = PAGED && static_cast<uint32_t>(c.page) >= static_cast<uint32_t>(p.num_pages);
        c.wrong |= wrong;
        return (wrong ? 0 : c.page) * p.Hkv + c.it.g;
      };
      const uint32_t to_first = map_to_rank(sbase, 0) - sbase;       // added to a barrier's address: the first CTA's
      bool ok = true;
      Ring<CODES ? S::kKStages : kKSlots> kr;
      Ring<CODES ? S::kVStages : kVSlots> vr;
      uint32_t q_items = 0;
      Cursor ck, cv;
      ck.i = cv.i = -1;
      ck.tile = ck.end = cv.tile = cv.end = 0;
      ck.valid = cv.valid = true;
      ck.wrong = cv.wrong = false;
      // One loop, so that the code of a step stands here once: n = -4 looks up the first tiles, from -3 on a K tile is asked for, from 0 on V(n) before it.
      [[maybe_unused]] int keys = 0, values = 0;                     // tiles issued
#pragma unroll 1
      for (int n = -4; ok; ++n) {
        if (n >= 0) {
          if (!cv.valid) break;
          if constexpr (STALL) {
            if (values++ >= p.stall_after_tiles) break;
          }
          const uint32_t full = CODES ? B.vc_full(vr.slot) : B.v_full(vr.slot);
          ok = mbar_wait_warp(CODES ? B.vc_empty(vr.slot) : B.v_empty(vr.slot), vr.par ^ 1u, s_abort);
          if (!ok) break;
          if (lane == 0) mbar_expect_tx(full, CODES ? S::kVCodes : S::kVBytes);
          __syncwarp();
          if (v_r0 < kChunkTile) {
            if constexpr (CODES) tma_load_3d(sbase + S::kVC + vr.slot * S::kVCodes + v_r0 * 64, &map_v, half * 64, cv.y, place(cv), full);
            else tma_load_3d(sbase + S::kV + vr.slot * S::kVBytes + v_r0 * D, &map_v, half * (D / 2), cv.y, place(cv), full);
          }
          vr.step();
        }
        if (n == -4 || n >= 0) advance(cv, true);
        if (!ck.valid) continue;
        if (n >= -3) {
          if constexpr (STALL) {
            if (keys++ >= p.stall_after_tiles) continue;
          }
          if (ck.fresh) {
            // box of TPT tokens x G heads x 64 columns: rows land in (token, head) order; rows of the next sequence (or zeros past
            // the tensor) that come along are computed and never written
            const uint32_t qb = q_items & 1u;
            ok = mbar_wait_warp(B.q_empty(qb), ((q_items >> 1) & 1u) ^ 1u, s_abort);
            if (!ok) break;
            if (lane == 0) {
              if constexpr (CODES) mbar_expect_tx(B.q_full(qb), S::kSlabs * p.tpt * p.G * 128);
              else if (rank == 0) mbar_expect_tx(B.q_ready(qb), 2 * S::kSlabs * p.tpt * p.G * 128);
#pragma unroll
              for (int sl = 0; sl < S::kSlabs; ++sl) {
                const uint32_t dst = sbase + S::kQ + qb * S::kQBytes + sl * S::kQSlab;
                const int token = ck.it.start + (2 * ck.it.part + half) * p.tpt;
                if constexpr (CODES) tma_load_3d(dst, &map_q, sl * 64, ck.it.g * p.G, token, B.q_full(qb));
                else tma_load_3d_pair(dst, &map_q, sl * 64, ck.it.g * p.G, token, B.q_ready(qb) + to_first);
              }
            }
            ++q_items;
          }
          if constexpr (CODES) {
            ok = mbar_wait_warp(B.kc_empty(kr.slot), kr.par ^ 1u, s_abort);
            if (!ok) break;
            if (lane == 0) mbar_expect_tx(B.kc_full(kr.slot), S::kKCodes);
            __syncwarp();
            if (k_r0 < 64) tma_load_3d(sbase + S::kKC + kr.slot * S::kKCodes + k_r0 * 128, &map_k, 0, ck.y, place(ck), B.kc_full(kr.slot));
          } else {
            ok = mbar_wait_warp(B.k_empty(kr.slot), kr.par ^ 1u, s_abort);
            if (!ok) break;
            if (lane == 0 && rank == 0) mbar_expect_tx(B.k_ready(kr.slot), 2 * S::kKBytes);
            const int sl = lane % S::kSlabs;
            if (k_r0 < 64)
              tma_load_3d_pair(sbase + S::kK + kr.slot * S::kKBytes + sl * S::kKSlab + k_r0 * 128, &map_k, sl * 64, ck.y, place(ck),
                               B.k_ready(kr.slot) + to_first);
          }
          kr.step();
        }
        advance(ck, false);
      }
    } else if (warp == R::kRelay) {
      bool ok = true;
      uint32_t steps = 0, items = 0;
      if constexpr (CODES) {
        // =========================================================================== scales
        // Four steps at a time, a lane per step and group of 16 keys, and one round of four ahead: pages are looked up two rounds before their
        // scales are handed on, scales are read one round before.  A step's entries are free when the PV of the step three before has
        // finished, as its score buffer is.  Groups that the unit sees nothing of take 1, whatever their blocks hold.
        const int sub = lane >> 3, group = lane & 7;
        Item at;
        ChunkSpan span = {};
        int at_i = -1, tile = 0;
        at.t1 = 0;
        struct Round {
          int found;                                       // steps in it
          int g, row, page;                                // of this lane's step: KV head, slot in its page, page; row < 0: nothing to read
        };
        auto look_up = [&]() {
          Round r = {0, 0, -1, 0};
#pragma unroll 1
          for (int j = 0; j < 4; ++j) {
            if (++tile >= at.t1) {
              for (++at_i; at_i < n_items; ++at_i) {
                at = item(at_i);
                if (at.t1 > at.t0) break;
              }
              if (at_i >= n_items) {
                at.t1 = 0;
                break;
              }
              span = span_of(at);
              tile = at.t0;
              ++items;
            }
            ++r.found;
            if (j == sub) {
              const int key = span.tile(tile) * kChunkTile + group * 16;
              if (key < at.L + at.n && span.sees_some(key, 16)) {
                r.g = at.g;
                r.row = key;
                r.page = at.b;
                if (PAGED) {
                  r.page = __ldg(p.block_table + static_cast<size_t>(at.b) * p.max_pages + (key >> p.page_shift));
                  r.row = key & (p.page_size - 1);
                }
              }
            }
          }
          return r;
        };
        auto read = [&](const Round& r, float& ks, float& vs) {
          ks = vs = 1.f;
          if (r.row >= 0 && (!PAGED || static_cast<uint32_t>(r.page) < static_cast<uint32_t>(p.num_pages))) {
            const long long place = (static_cast<long long>(r.page) * p.Hkv + r.g) * p.head_blocks + (r.row >> p.block_shift);
            ks = __ldg(p.k_scale + place);
            vs = __ldg(p.v_scale + place);
          }
        };
        Round now = {0, 0, -1, 0}, next = now;
        float ks = 1.f, vs = 1.f;
#pragma unroll 1
        do {
          const Round later = look_up();
          float ks_next, vs_next;
          read(next, ks_next, vs_next);
          if (beyond_range(vs) > kScaleRange) report_status(p.status, EAGLE_ERR_SCALE);
          const uint4 entry = make_uint4(__float_as_uint(ks * p.scale_log2), __float_as_uint(fast_log2(vs)), __float_as_uint(fast_rcp(vs)), 0u);
#pragma unroll 1
          for (int j = 0; j < now.found && ok; ++j, ++steps) {
            const uint32_t sb = steps % kSBufs;
            if (steps >= kSBufs) ok = mbar_wait_warp(B.o_done(sb), ((steps / kSBufs) & 1u) ^ 1u, s_abort);
            if (!ok) break;
            if (j == sub) store_shared(sbase + S::kScale + (sb * kGroups + group) * 16, entry);
            __syncwarp();
            if (lane == 0) mbar_arrive(B.s_full(sb));
          }
          now = next;
          next = later;
          ks = ks_next;
          vs = vs_next;
        } while (now.found + next.found > 0 && ok);
      } else {
        // =========================================================================== V tiles that have landed
        // Values of slots that the unit does not see may be anything, and 0 * garbage must not reach O: they are zeroed here before the first
        // CTA's issuer hears of the tile.
        Ring<kVSlots> vr;
        const uint32_t to_first = map_to_rank(sbase, 0) - sbase;
        for (int i = 0; i < n_items && ok; ++i) {
          const Item it = item(i);
          const ChunkSpan span = span_of(it);
          items += it.t1 > it.t0 ? 1u : 0u;
          for (int t = it.t0; t < it.t1; ++t, ++steps, vr.step()) {
            ok = mbar_wait_warp(B.v_full(vr.slot), vr.par, s_abort);
            if (!ok) break;
            const int key0 = span.tile(t) * kChunkTile, in_use = it.L + it.n;
            if (key0 + kChunkTile > in_use || !span.sees_all(key0, kChunkTile)) {
              for (int j = lane; j < kChunkTile * (D / 16); j += 32) {     // whole rows of D bytes, so the swizzle does not matter
                const int key = key0 + j / (D / 16);
                if (key >= in_use || !span.sees(key)) *reinterpret_cast<uint4*>(smem + S::kV + vr.slot * S::kVBytes + j * 16) = make_uint4(0u, 0u, 0u, 0u);
              }
              fence_proxy_async();
              __syncwarp();
              if (lane == 0) mbar_arrive_release_pair(B.v_ready(vr.slot) + to_first);
            } else if (lane == 0) {
              mbar_arrive_pair(B.v_ready(vr.slot) + to_first);
            }
          }
        }
      }
      // The MMAs report to the barriers of both CTAs, also where nobody waits for it: all reports of the last uses have to be in before
      // the CTA may leave its shared memory to another.
#pragma unroll 1
      for (uint32_t g = steps > kKSlots ? steps - kKSlots : 0u; g < steps && ok; ++g) {
        ok = mbar_wait_warp(B.k_empty(g % kKSlots), (g / kKSlots) & 1u, s_abort);
        if (ok && g + kVSlots >= steps) ok = mbar_wait_warp(B.v_empty(g % kVSlots), (g / kVSlots) & 1u, s_abort);
        if (ok && g + kSBufs >= steps) ok = mbar_wait_warp(B.o_done(g % kSBufs), (g / kSBufs) & 1u, s_abort);
      }
#pragma unroll 1
      for (uint32_t i = items > 2 ? items - 2 : 0u; i < items && ok; ++i) ok = mbar_wait_warp(B.q_empty(i & 1u), (i >> 1) & 1u, s_abort);
    } else if (warp == R::kQK) {
      // =========================================================================== S = Q K^T, up to three steps ahead of the softmax
      if (lane == 0 && (CODES || rank == 0)) {
        constexpr uint32_t idesc = CODES ? instr_desc_half(256, kChunkTile, false) : instr_desc(256, kChunkTile, false);
        const uint32_t q_lo = desc_lo(sbase + S::kQ), k_lo = desc_lo(sbase + S::kK);
        const uint32_t to_first = map_to_rank(sbase, 0) - sbase;
        Ring<kKSlots> kr;
        Ring<kSBufs> sr;
        uint32_t steps = 0, items = 0;
        bool ok = true;
        for (int i = 0; i < n_items && ok; ++i) {
          const Item it = item(i);
          if (it.t1 <= it.t0) continue;
          const uint32_t qb = items & 1u;
          if constexpr (CODES) {
            if (rank != 0) {
              ok = mbar_wait(B.q_done(qb), (items >> 1) & 1u, s_abort);
              if (ok) mbar_arrive_release_pair(B.q_ready(qb) + to_first);
            } else {
              ok = mbar_wait_cluster(B.q_ready(qb), (items >> 1) & 1u, s_abort);
            }
          } else {
            ok = mbar_wait(B.q_ready(qb), (items >> 1) & 1u, s_abort);
          }
          for (int t = it.t0; t < it.t1 && ok; ++t, ++steps) {
            if constexpr (CODES) {
              if (rank != 0) {
                ok = mbar_wait(B.k_done(kr.slot), kr.par, s_abort);
                if (ok) mbar_arrive_release_pair(B.k_ready(kr.slot) + to_first);
                kr.step();
                continue;
              }
              ok = mbar_wait_cluster(B.k_ready(kr.slot), kr.par, s_abort);
            } else {
              ok = mbar_wait(B.k_ready(kr.slot), kr.par, s_abort);
            }
            if (ok && steps >= kSBufs) ok = mbar_wait(B.o_done(sr.slot), sr.par ^ 1u, s_abort);   // the buffer's last P has been used
            if (!ok) break;
            fence_after();
            issue_qk_pair<D>(tmem + sr.slot * 128, q_lo + qb * (S::kQBytes >> 4), k_lo + kr.slot * (S::kKBytes >> 4), idesc);
            commit_pair(B.s_full(sr.slot));
            commit_pair(B.k_empty(kr.slot));
            if (t == it.t1 - 1) commit_pair(B.q_empty(qb));
            kr.step();
            sr.step();
          }
          ++items;
        }
      }
    } else if (warp == R::kPV) {
      // =========================================================================== O += P V
      if (lane == 0 && (CODES || rank == 0)) {
        constexpr uint32_t idesc = CODES ? instr_desc_half(256, D, true) : instr_desc(256, D, true);
        const uint32_t v_lo = desc_lo(sbase + S::kV);
        const uint32_t to_first = map_to_rank(sbase, 0) - sbase;
        Ring<kVSlots> vr;
        Ring<kSBufs> sr;
        uint32_t items = 0;
        bool ok = true;
        for (int i = 0; i < n_items && ok; ++i) {
          const Item it = item(i);
          if (it.t1 <= it.t0) continue;
          for (int t = it.t0; t < it.t1 && ok; ++t) {
            if constexpr (CODES) {
              if (rank != 0) {
                ok = mbar_wait(B.v_full(vr.slot), vr.par, s_abort);
                if (ok) mbar_arrive_release_pair(B.v_ready(vr.slot) + to_first);
                vr.step();
                continue;
              }
              ok = mbar_wait_cluster(B.v_ready(vr.slot), vr.par, s_abort);
            } else {
              ok = mbar_wait(B.v_ready(vr.slot), vr.par, s_abort);
            }
            if (ok && t == it.t0 && items > 0) ok = mbar_wait(B.o_free(), (items - 1) & 1u, s_abort);   // the last item's output has been read
            ok = ok && mbar_wait(B.p_full(sr.slot), sr.par, s_abort);
            if (!ok) break;
            fence_after();
            issue_pv_pair<D>(tmem + kColO, tmem + sr.slot * 128, v_lo + vr.slot * (S::kVBytes >> 4), idesc, t == it.t0 ? 0u : 1u);
            commit_pair(B.o_done(sr.slot));
            commit_pair(B.v_empty(vr.slot));
            vr.step();
            sr.step();
          }
          ++items;
        }
      }
    } else {
      // =========================================================================== widening (codes)
      // Two warps take the K tiles in turn, two the V tiles: what a tile costs is mostly waiting (for the codes, for the slot, for shared memory), so
      // four tiles are under way at a time.  The K warps turn an item's queries, too, half the rows each.  The eight lanes of a 16-byte access
      // meet no bank twice: K's lanes of the upper columns store their odd piece first.
      if constexpr (CODES) {
        const uint32_t w = static_cast<uint32_t>(warp - R::kConv) & 1u;
        const bool is_v = warp >= R::kConv + 2;
        bool ok = true;
        uint32_t g = 0, items = 0;
        for (int i = 0; i < n_items && ok; ++i) {
          const Item it = item(i);
          if (it.t1 <= it.t0) continue;
          const ChunkSpan span = span_of(it);
          if (!is_v) {
            // ---- the item's queries, in place: a lane per row
            const uint32_t qb = items & 1u;
            ok = mbar_wait_warp(B.q_full(qb), (items >> 1) & 1u, s_abort);
            if (!ok) break;
#pragma unroll 1
            for (int half = 0; half < 2; ++half) {
              const int row = static_cast<int>(w) * 64 + half * 32 + lane;
              const uint32_t at = sbase + S::kQ + qb * S::kQBytes + row * 128, swz = row & 7;
              uint32_t top = 0;
#pragma unroll 1
              for (int e = 0; e < 16; ++e) {
                const uint4 v = load_shared(at + (e >> 3) * S::kQSlab + (((e & 7) ^ swz) << 4));
                top = max(max(top, max(magnitude_bits(v.x), magnitude_bits(v.y))), max(magnitude_bits(v.z), magnitude_bits(v.w)));
              }
              const RowFactor f = row_factor(top);
#pragma unroll 1
              for (int e = 0; e < 16; ++e) {
                const uint32_t to = at + (e >> 3) * S::kQSlab + (((e & 7) ^ swz) << 4);
                const uint4 v = load_shared(to);
                store_shared(to, make_uint4(half_of_bf16(v.x, f.down), half_of_bf16(v.y, f.down), half_of_bf16(v.z, f.down), half_of_bf16(v.w, f.down)));
              }
              reinterpret_cast<volatile unsigned long long*>(smem + S::kFactor)[(items % S::kFactors) * 128 + row] = tagged(items, f.up);
            }
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) mbar_arrive(rank == 0 ? B.q_ready(qb) : B.q_done(qb));
          }
          ++items;
          for (int t = it.t0 + static_cast<int>((g ^ w) & 1u); t < it.t1 && ok; t += 2) {
            const uint32_t gs = g + (t - it.t0);
            if (!is_v) {
              const uint32_t st = gs % S::kKStages, sl = gs % kKSlots;
              ok = mbar_wait_warp(B.kc_full(st), (gs / S::kKStages) & 1u, s_abort) && mbar_wait_warp(B.k_empty(sl), ((gs / kKSlots) & 1u) ^ 1u, s_abort);
              if (!ok) break;
              const uint32_t piece = lane & 7, flip = piece >> 2, row0 = lane >> 3;
              const uint32_t from = sbase + S::kKC + st * S::kKCodes + lane * 16, to = sbase + S::kK + sl * S::kKBytes + flip * S::kKSlab;
              const uint32_t one = 2 * (piece & 3) + flip, two = 2 * (piece & 3) + 1 - flip;
#pragma unroll 1
              for (uint32_t u = 0; u < 16; ++u) {
                const uint32_t row = u * 4 + row0;
                uint4 lo, hi;
                widen_codes(load_shared(from + u * 512), lo, hi);
                store_shared(to + row * 128 + ((one ^ (row & 7)) << 4), flip ? hi : lo);
                store_shared(to + row * 128 + ((two ^ (row & 7)) << 4), flip ? lo : hi);
              }
              fence_proxy_async();
              __syncwarp();
              if (lane == 0) {
                mbar_arrive(rank == 0 ? B.k_ready(sl) : B.k_done(sl));
                mbar_arrive(B.kc_empty(st));
              }
            } else {
              const uint32_t st = gs % S::kVStages, sl = gs % kVSlots;
              // The tile's turn first: V's stages change owners from use to use, and a wait by parity does not tell the use before last from this one.
              // With as many tiles as stages, the tile being free says that the stage's last use is over.
              ok = mbar_wait_warp(B.v_empty(sl), ((gs / kVSlots) & 1u) ^ 1u, s_abort) && mbar_wait_warp(B.vc_full(st), (gs / S::kVStages) & 1u, s_abort);
              if (!ok) break;
              // values of slots that the unit does not see may be anything, and 0 * garbage must not reach O
              const int key0 = span.tile(t) * kChunkTile, in_use = it.L + it.n;
              const bool clean = key0 + kChunkTile <= in_use && span.sees_all(key0, kChunkTile);
              const uint32_t piece = lane & 3, row0 = lane >> 2;
              const uint32_t from = sbase + S::kVC + st * S::kVCodes + lane * 16, to = sbase + S::kV + sl * S::kVBytes + row0 * 128;
              const uint32_t one = ((2 * piece) ^ row0) << 4, two = ((2 * piece + 1) ^ row0) << 4;
#pragma unroll 1
              for (uint32_t u = 0; u < 16; ++u) {
                const int key = key0 + static_cast<int>(u * 8 + row0);
                uint4 c = load_shared(from + u * 512), lo, hi;
                if (!clean && (key >= in_use || !span.sees(key))) c = make_uint4(0u, 0u, 0u, 0u);
                widen_codes(c, lo, hi);
                store_shared(to + u * 1024 + one, lo);
                store_shared(to + u * 1024 + two, hi);
              }
              fence_proxy_async();
              __syncwarp();
              if (lane == 0) {
                mbar_arrive(rank == 0 ? B.v_ready(sl) : B.v_full(sl));
                mbar_arrive(B.vc_empty(st));
              }
            }
          }
          g += static_cast<uint32_t>(it.t1 - it.t0);
        }
      }
    }
  } else {
    // =========================================================================== softmax and output
    // As in chunk.cu: two groups of four warps take alternate steps; thread r of a group owns query row r (tensor-memory lane r), all 128
    // score columns.  The two threads of a row share one reference maximum: the one that handled step g publishes it, tagged with g, before it
    // takes its exponentials, and the other picks it up at step g + 1; each keeps its own part of the row sum.  fp32 throughout, in the log2
    // domain; the probabilities are rounded to bf16 (relative 2^-8 each) or, over codes and times vs, to fp16 (2^-11) for the tensor cores, the sum that divides
    // them is kept from the unrounded ones.
    const uint32_t grp = static_cast<uint32_t>(warp >> 2);
    const int r = tid & 127;
    const uint32_t lane_addr = static_cast<uint32_t>((warp & 3) * 32) << 16;
    volatile unsigned long long* tag = reinterpret_cast<volatile unsigned long long*>(smem + S::kTag) + r;
    volatile unsigned long long* lfin = reinterpret_cast<volatile unsigned long long*>(smem + S::kLfin) + r;
    const uint32_t o_addr = tmem + lane_addr + kColO;
    const uint32_t p_to = map_to_rank(B.p_full(0), 0), o_free_to = map_to_rank(B.o_free(), 0);
    const int tok_r = r / p.G, head_r = r - tok_r * p.G;   // token and head within the tile
    const float scale_log2 = p.scale_log2;
    uint32_t sg = 0, items = 0;                            // steps and items before the current item
    bool ok = true;
    for (int i = 0; i < n_items && ok; ++i) {
      const Item it = item(i);
      const int steps = it.t1 - it.t0;
      if (steps <= 0) continue;
      const ChunkSpan span = span_of(it);
      const int first = (2 * it.part + static_cast<int>(rank)) * p.tpt, token = first + tok_r;    // place in the chunk
      const bool row_valid = tok_r < p.tpt && token < it.n;
      const bool warp_rests = !__any_sync(0xffffffffu, row_valid);
      // What a row sees: slots up to `limit`; of a tree, those of the prefix and the bits of `path` from slot L on.  With a window, from `low` on and
      // below the sinks.
      const int place = token < it.n ? token : it.n - 1;
      unsigned long long path = 0;
      int limit = it.L + place, low = 0;
      if (p.tree > 0) {
        limit = it.L - 1;
        const int32_t* parent = p.tree_parent + (p.shared_tree ? 0 : static_cast<size_t>(it.b) * p.tree);
        int depth = 0;
        for (int m = place; m >= 0; m = __ldg(parent + m), ++depth) path |= 1ull << m;      // (the planner has checked that parents come first)
        low = it.L + depth - p.window;
      } else {
        low = limit - p.window + 1;
      }
      if (p.window <= 0) low = 0;
      // tiles that every row of this query tile sees whole: up to `upto`, and from `from` on or below the sinks
      const int upto = p.tree > 0 ? it.L : it.L + first + 1;
      const int from = p.window > 0 ? (p.tree > 0 ? it.L + kMaxTree : it.L + first + p.tpt) - p.window : 0;
      float up = 1.f;                                      // what the row's scores are multiplied by again (codes)
      if constexpr (CODES) {
        if (!warp_rests && (steps > 1 || ((sg ^ grp) & 1u) == 0)) {
          // (a group without a step of the item has no use for it; one with a step holds its place in the ring until it has read it)
          const unsigned long long t = tag_wait(reinterpret_cast<volatile unsigned long long*>(smem + S::kFactor) + (items % S::kFactors) * 128 + r, items, s_abort);
          ok = __all_sync(0xffffffffu, has_tag(t, items));
          if (!ok) break;
          up = value_of(t);
        }
      }
      float m_ref = -INFINITY;   // reference this thread's row sum is relative to
      float m_in = -INFINITY;    // reference the other group left behind at the step before this group's latest one
      float l_sum = 0.f;
      for (int s = static_cast<int>((sg ^ grp) & 1u); s < steps; s += 2) {
        const uint32_t gs = sg + s, sb = gs % kSBufs, sph = (gs / kSBufs) & 1u;
        const uint32_t s_addr = tmem + lane_addr + sb * 128;
        ok = mbar_wait_warp(B.s_full(sb), sph, s_abort);
        if (!ok) break;
        if (!warp_rests) {
          fence_after();
          const int key0 = span.tile(it.t0 + s) * kChunkTile;
          if (key0 + kChunkTile > upto || (key0 < from && key0 + kChunkTile > p.sinks)) {
            // a tile that some row of this query tile does not see whole: -inf over the invisible scores, in place
#pragma unroll 1
            for (int c = 0; c < 4; ++c) {
              const int k0 = key0 + c * 32;
              auto below = [](int n) { return n >= 32 ? 0xffffffffu : (n <= 0 ? 0u : (1u << n) - 1u); };      // the first n bits
              uint32_t see = below(limit - k0 + 1);
              if (p.window > 0) see &= ~below(low - k0) | below(p.sinks - k0);
              if (p.tree > 0) {
                const int sh = k0 - it.L;
                if (sh >= 0) see |= sh < 64 ? static_cast<uint32_t>(path >> sh) : 0u;
                else if (sh > -32) see |= static_cast<uint32_t>(path << -sh);
              }
              if (__all_sync(0xffffffffu, see == 0xffffffffu)) continue;
              uint32_t t[32];
              if (__any_sync(0xffffffffu, see != 0u)) {
                ld32(s_addr + c * 32, t);
                wait_ld();
#pragma unroll
                for (int e = 0; e < 32; ++e) t[e] = (see >> e) & 1u ? t[e] : 0xff800000u;
              } else {
#pragma unroll
                for (int e = 0; e < 32; ++e) t[e] = 0xff800000u;
              }
              st32(s_addr + c * 32, t);
            }
            wait_st();
          }
          // ---- row maximum.  bf16: chunks 0 and 1 stay in registers, chunks 2 and 3 are fetched again for the exponentials.  Codes: all are fetched
          // twice, in short loops.  The code that a step runs through in all sixteen warps is more than the instruction caches hold, so that straight
          // lines cost more than what they do: with the loops unrolled and a third of the exponentials on the FMA pipe a step took half as
          // long again.
          const uint32_t scale_at = sbase + S::kScale + sb * kGroups * 16;
          uint32_t ra[32], rb[32];
          float tmax = -INFINITY;
          bool odd = false;                                // a visible score that is NaN or +inf
          if constexpr (CODES) {
            auto top_of = [&](const uint32_t* raw, const uint4& c) {      // of 16 scores, with their scales
              float x = -INFINITY, y = -INFINITY;
#pragma unroll
              for (int e = 0; e < 16; e += 4) {
                x = max3_nan(x, __uint_as_float(raw[e]), __uint_as_float(raw[e + 1]));
                y = max3_nan(y, __uint_as_float(raw[e + 2]), __uint_as_float(raw[e + 3]));
              }
              tmax = max3_nan(tmax, fmaf(max3_nan(x, y, -INFINITY), score_factor(__uint_as_float(c.x), up), __uint_as_float(c.y)), -INFINITY);
            };
            ld32(s_addr, ra);
#pragma unroll 1
            for (int h = 0; h < 2; ++h) {
              const uint4 c0 = load_shared(scale_at + h * 64), c1 = load_shared(scale_at + h * 64 + 16);
              const uint4 c2 = load_shared(scale_at + h * 64 + 32), c3 = load_shared(scale_at + h * 64 + 48);
              wait_ld();
              ld32(s_addr + h * 64 + 32, rb);
              top_of(ra, c0);
              top_of(ra + 16, c1);
              wait_ld();
              if (h == 0) ld32(s_addr + 64, ra);
              top_of(rb, c2);
              top_of(rb + 16, c3);
            }
            ld16(s_addr, ra);                              // (the first scores again)
            odd = !(tmax < INFINITY);
          } else {
            uint32_t rc[32], rd[32];
            ld32(s_addr + 64, rc);
            ld32(s_addr + 96, rd);
            ld32(s_addr, ra);
            ld32(s_addr + 32, rb);
            wait_ld();
            float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int e = 0; e < 32; e += 2) {
              mx[0] = max3_nan(mx[0], __uint_as_float(rc[e]), __uint_as_float(rc[e + 1]));
              mx[1] = max3_nan(mx[1], __uint_as_float(rd[e]), __uint_as_float(rd[e + 1]));
              mx[2] = max3_nan(mx[2], __uint_as_float(ra[e]), __uint_as_float(ra[e + 1]));
              mx[3] = max3_nan(mx[3], __uint_as_float(rb[e]), __uint_as_float(rb[e + 1]));
            }
            tmax = max3_nan(max3_nan(mx[0], mx[1], mx[2]), mx[3], -INFINITY) * scale_log2;   // scale > 0
            odd = !(tmax < INFINITY);
          }
          // such a score makes the row NaN (through its sum: not every exponential below passes one on)
          if (odd) l_sum = __uint_as_float(0x7fffffffu);

          // the reference the other group settled on at the previous step (waited for at an item's first step too, where its value
          // is not used: the other group must have read the tag of step gs - 2 before it is replaced)
          float m_prev = -INFINITY;
          if (gs > 0) {
            const unsigned long long t = tag_wait(tag, gs - 1u, s_abort);
            ok = __all_sync(0xffffffffu, has_tag(t, gs - 1u));
            if (!ok) break;
            if (s > 0) m_prev = value_of(t);
          }
          if (m_prev != m_ref) {
            l_sum *= fast_exp2(m_ref - m_prev);     // m_ref = -inf: nothing summed yet, the factor is 0
            m_ref = m_prev;
          }
          m_in = m_prev;
          const bool grow = tmax > m_ref + kRescaleThreshold || (m_ref == -INFINITY && tmax > -INFINITY);
          float factor = 1.f;
          if (grow) {
            factor = fast_exp2(m_ref - tmax);      // 0 when there was no reference yet
            m_ref = tmax;
            l_sum *= factor;
          }
          *tag = tagged(gs, m_ref);
          if (s > 0 && __any_sync(0xffffffffu, grow)) {
            // the previous step accumulated into O and may still be running
            ok = mbar_wait_warp(B.o_done((gs - 1) % kSBufs), ((gs - 1) / kSBufs) & 1u, s_abort);
            if (!ok) break;
            fence_after();
            uint32_t o[32];
#pragma unroll 1
            for (int c = 0; c < D / 32; ++c) {
              ld32(o_addr + c * 32, o);
              wait_ld();
#pragma unroll
              for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * factor);
              st32(o_addr + c * 32, o);
            }
            wait_st();
          }
          // ---- exponentials and packed P over score columns that have been read
          const float neg_base = m_ref == -INFINITY ? 0.f : -m_ref;
          if constexpr (CODES) {
            auto exp_group = [&](const uint32_t* raw, int group, const uint4& c) {   // 16 scores with their scales
              const float a = score_factor(__uint_as_float(c.x), up), base = __uint_as_float(c.y) + neg_base + kHalfShift;
              const uint64_t scale2 = pack2(a, a), base2 = pack2(base, base);
              uint64_t ls2[2] = {0ull, 0ull};
              uint32_t pk[8];
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                float x, y;
                unpack2(fma2(pack2(__uint_as_float(raw[2 * e]), __uint_as_float(raw[2 * e + 1])), scale2, base2), x, y);
                float p0, p1;
                if (e == 7) {                              // (one pair in eight on the FMA pipe: 3 % faster than none, one in four 1 %)
                  poly_exp2_pair(pack2(x, y), p0, p1);
                } else {
                  p0 = fast_exp2(x);
                  p1 = fast_exp2(y);
                }
                ls2[e & 1] = add2(ls2[e & 1], pack2(p0, p1));
                pk[e] = pack_half(p0, p1);
              }
              st8(s_addr + group * 8, pk);
              float x, y;
              unpack2(add2(ls2[0], ls2[1]), x, y);
              l_sum = fmaf(x + y, __uint_as_float(c.z), l_sum);
            };
#pragma unroll 1
            for (int h = 0; h < 4; ++h) {
              const uint4 c0 = load_shared(scale_at + h * 32), c1 = load_shared(scale_at + h * 32 + 16);
              wait_ld();
              ld16(s_addr + h * 32 + 16, rb);
              exp_group(ra, 2 * h, c0);
              wait_ld();
              if (h < 3) ld16(s_addr + h * 32 + 32, ra);
              exp_group(rb, 2 * h + 1, c1);
            }
          } else {
            uint64_t ls2[2] = {0ull, 0ull};
            const uint64_t scale2 = pack2(scale_log2, scale_log2), base2 = pack2(neg_base, neg_base);
            uint32_t pk[16];
            auto exp_chunk = [&](const uint32_t* raw, int c) {
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                const uint64_t x2 = fma2(pack2(__uint_as_float(raw[2 * e]), __uint_as_float(raw[2 * e + 1])), scale2, base2);
                float p0, p1;
                if (e % kPolyStride == kPolyStride - 1) {
                  poly_exp2_pair(x2, p0, p1);
                } else {
                  float a, b;
                  unpack2(x2, a, b);
                  p0 = fast_exp2(a);
                  p1 = fast_exp2(b);
                }
                ls2[e & 1] = add2(ls2[e & 1], pack2(p0, p1));
                pk[e] = pack_bf16(p0, p1);
              }
              st16(s_addr + c * 16, pk);
            };
            exp_chunk(ra, 0);
            ld32(s_addr + 64, ra);
            exp_chunk(rb, 1);
            ld32(s_addr + 96, rb);
            wait_ld();
            exp_chunk(ra, 2);
            exp_chunk(rb, 3);
            float a, b, c, d;
            unpack2(ls2[0], a, b);
            unpack2(ls2[1], c, d);
            l_sum += (a + b) + (c + d);
          }
          if (s == steps - 2) {
            // This group's last step of the item, but not the item's: hand the row sum to the group that writes the output, with the
            // item's number (in the second CTA the barriers on the way between the two lie in the first one and order nothing here).
            // (That group reads it before it publishes a tag of the next item, and this place is written again two items on.)
            lfin[(items & 1u) * 128] = tagged(items, l_sum);
          }
          wait_st();
          fence_before();
        } else {
          // (the chain of tags goes on: the next item's rows may be in use)
          if (gs > 0) {
            ok = __all_sync(0xffffffffu, has_tag(tag_wait(tag, gs - 1u, s_abort), gs - 1u));
            if (!ok) break;
          }
          *tag = tagged(gs, -INFINITY);
        }
        __syncwarp();
        if (lane == 0) mbar_arrive_pair(p_to + 8u * sb);

        if (s == steps - 1) {
          // ---- this group took the item's last step: it writes the item's output
          unsigned long long other = tagged(items, 0.f);
          if (!warp_rests && steps > 1) other = tag_wait(lfin + (items & 1u) * 128, items, s_abort);
          ok = mbar_wait_warp(B.o_done(sb), sph, s_abort) && __all_sync(0xffffffffu, has_tag(other, items));      // PVs complete in order
          if (!ok) break;
          if (!warp_rests) {
            fence_after();
            const float l_row = fmaf(value_of(other), m_in == m_ref ? 1.f : fast_exp2(m_in - m_ref), l_sum);   // the other's sum is relative to the reference it last saw
            const float inv = l_row > 0.f ? 1.f / l_row : (l_row == 0.f ? 0.f : l_row);                 // a NaN sum stays one
            const int slot = it.slot < 0 ? -1 : it.slot + static_cast<int>(rank);
            __nv_bfloat16* out_row = p.out + (static_cast<size_t>(it.start + token) * p.Hq + it.g * p.G + head_r) * D;
            // an fp32 partial is laid out [4 columns][row], so that the lanes of a store write consecutive 16-byte pieces
            float* part = p.work.part_o + static_cast<size_t>(slot < 0 ? 0 : slot) * (D / 4) * (128 * 4) + r * 4;
            auto write = [&](const uint32_t* o, int c) {     // 32 columns of the accumulator
              if (row_valid && slot < 0) {
#pragma unroll
                for (int e = 0; e < 32; e += 16) {
                  uint32_t v[8];
#pragma unroll
                  for (int k = 0; k < 8; ++k) v[k] = pack_bf16(__uint_as_float(o[e + 2 * k]) * inv, __uint_as_float(o[e + 2 * k + 1]) * inv);
                  st_global_v8(out_row + c * 32 + e, v);
                }
              } else if (row_valid) {
#pragma unroll
                for (int e = 0; e < 32; e += 4)
                  *reinterpret_cast<uint4*>(part + (c * 8 + e / 4) * (128 * 4)) = make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]);
              }
            };
            if constexpr (CODES) {
              uint32_t o[32];
#pragma unroll 1
              for (int c = 0; c < D / 32; ++c) {
                ld32(o_addr + c * 32, o);
                wait_ld();
                if (c == D / 32 - 1) {
                  fence_before();
                  __syncwarp();
                  if (lane == 0) mbar_arrive_pair(o_free_to);
                }
                write(o, c);
              }
            } else {
              // The accumulator is given back as soon as it is in registers: the next item's first PV waits for that.
              uint32_t o[D];
#pragma unroll
              for (int c = 0; c < D / 32; ++c) ld32(o_addr + c * 32, o + c * 32);
              wait_ld();
              fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive_pair(o_free_to);
#pragma unroll
              for (int c = 0; c < D / 32; ++c) write(o + c * 32, c);
            }
            if (row_valid && slot >= 0) p.work.part_ml[static_cast<size_t>(slot) * 128 + r] = make_float2(m_ref, l_row);
          } else if (lane == 0) {
            mbar_arrive_pair(o_free_to);
          }
        }
      }
      sg += steps;
      ++items;
    }
  }

  // ---- teardown: everyone arrives here, normally or after an abort; neither CTA leaves while the other may still reach into it
  fence_before();
  __syncthreads();
  if (*s_abort) {
    if (tid == 0) report_status(p.status, EAGLE_ERR_TIMEOUT);
    let_work_land();
  }
  cluster_sync();
  if (warp == R::kQK) {
    __syncwarp();
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
  }
}

template <int D, bool CODES>
cudaError_t launch_tiles(const ChunkParams& p, cudaStream_t stream) {
  using S = Smem<D, CODES>;
  CUtensorMap mk, mv, mq;
  const bool paged = p.block_table != nullptr;
  const int k_rows = paged && p.page_size < 64 ? p.page_size : 64, v_rows = paged && p.page_size < 128 ? p.page_size : 128;
  const long long n1 = paged ? p.page_size : (p.capacity > 0 ? p.capacity : 1);
  const long long n2 = paged ? static_cast<long long>(p.num_pages) * p.Hkv : static_cast<long long>(p.B) * p.Hkv;
  if constexpr (CODES) {
    if (!map_codes_3d(&mk, p.k, n1, n2, 128, k_rows, false) || !map_codes_3d(&mv, p.v, n1, n2, 64, v_rows, false)) return cudaErrorInvalidValue;
  } else {
    if (!map_bf16_3d(&mk, p.k, D, n1, n2, 64, k_rows, 1) || !map_bf16_3d(&mv, p.v, D, n1, n2, D / 2, v_rows, 1)) return cudaErrorInvalidValue;
  }
  if (!map_bf16_3d(&mq, p.q, D, p.Hq, p.N, 64, p.G, p.tpt)) return cudaErrorInvalidValue;
  BehindLaunch at(2 * p.num_workers, Roles<D, CODES>::kThreads, S::kBytes, stream);
  auto kernel = p.stall_after_tiles >= 0 ? (paged ? window_attn_kernel<D, true, CODES, true> : window_attn_kernel<D, false, CODES, true>)
                                         : (paged ? window_attn_kernel<D, true, CODES, false> : window_attn_kernel<D, false, CODES, false>);
  return cudaLaunchKernelEx(&at.config, kernel, p, mk, mv, mq);
}

template <int D, bool CODES>
cudaError_t prepare() {
  for (auto kernel : {window_attn_kernel<D, false, CODES, false>, window_attn_kernel<D, true, CODES, false>, window_attn_kernel<D, false, CODES, true>,
                      window_attn_kernel<D, true, CODES, true>}) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Smem<D, CODES>::kBytes);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace

cudaError_t window_prepare(int head_dim) {
  if (head_dim == 64) return prepare<64, false>();
  const cudaError_t e = prepare<128, false>();
  return e == cudaSuccess ? prepare<128, true>() : e;
}

cudaError_t launch_window(const ChunkParams& p, cudaStream_t stream) {
  cudaError_t e = launch_chunk_plan(p, stream);
  if (e != cudaSuccess) return e;
  if (p.few) e = p.k_scale ? launch_window_codes(p, stream) : launch_window_rows(p, stream);
  else if (p.k_scale) e = launch_tiles<128, true>(p, stream);
  else e = p.D == 128 ? launch_tiles<128, false>(p, stream) : launch_tiles<64, false>(p, stream);
  if (e != cudaSuccess) return e;
  count_launch();
  return launch_chunk_merge(p, stream);
}

}  // namespace eagle
