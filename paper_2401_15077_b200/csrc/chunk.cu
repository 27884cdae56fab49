// Causal attention of packed chunks of new tokens over the cache they have just been written to (contiguous or paged).
//
//   out[t] = sum_j softmax_j(scale * q[t].k[j]) v[j],  j <= L_b + i, for token t = token_start[b] + i of sequence b.
//
// Three launches: a planner (one CTA), an attention kernel (persistent) and the merge of what was cut.  The attention kernel of
// this file is one cluster of two CTAs on every two SMs; calls of single tokens take the one of chunk_rows.cu.
//
// A query tile is 128 rows of one (sequence, KV head): TPT = 128 / G tokens (rounded down) times the G heads of the group.  The two
// CTAs of a pair take neighbouring query tiles over the same K/V tiles, and the tensor cores of both work on one MMA of 256
// rows (cta_group::2): each CTA holds half of every K tile (64 keys) and half of every V tile (D / 2 columns), so a tile is
// loaded once for both, and each SM reads half of the operand from its shared memory.
//
// What bounds it is the way of one score buffer around the loop (score MMA, softmax, PV MMA, and a wait between each two): about 4700
// cycles, with three buffers on it 1550 per 128 keys, of which the tensor cores need 1036.  Replayed from a graph, a prompt of 4096
// tokens, 32 heads, D = 128 (137 GFLOP, causal) takes 154 us, 890 TFLOP/s (180 us as a single call on cold inputs: 765); two chunks of
// 2048 tokens behind 16384 (1.17 TFLOP) 1.05 to 1.13 ms, by the clock that the power limit leaves (a call: 1.17 ms, 1.0 PFLOP/s), where a
// large matrix product reaches 1.65 PFLOP/s, 1.40 sustained.
#include "chunk.cuh"
#include "tc.cuh"

namespace eagle {

namespace {

using namespace tc;

// ================================================================================================================ planner
constexpr int kPlanThreads = 512;
constexpr int kNearSeqs = 256, kNearUnits = 4096;      // tables of calls this small stay in shared memory as well

__device__ __forceinline__ int ceil_div(int a, int b) { return (a + b - 1) / b; }

// Inclusive prefix sums of (a, b) over the block; every thread gets its own, `tot` the block's.
struct Sum2 {
  int a;
  long long b;
};
__device__ Sum2 block_scan(Sum2 v, Sum2* warp_tot, Sum2* tot) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int a = __shfl_up_sync(0xffffffffu, v.a, o);
    const long long b = __shfl_up_sync(0xffffffffu, v.b, o);
    if (lane >= o) { v.a += a; v.b += b; }
  }
  __syncthreads();
  if (lane == 31) warp_tot[w] = v;
  __syncthreads();
  if (w == 0) {
    Sum2 t = lane < kPlanThreads / 32 ? warp_tot[lane] : Sum2{0, 0};
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int a = __shfl_up_sync(0xffffffffu, t.a, o);
      const long long b = __shfl_up_sync(0xffffffffu, t.b, o);
      if (lane >= o) { t.a += a; t.b += b; }
    }
    if (lane < kPlanThreads / 32) warp_tot[lane] = t;
  }
  __syncthreads();
  if (w > 0) { v.a += warp_tot[w - 1].a; v.b += warp_tot[w - 1].b; }
  *tot = warp_tot[kPlanThreads / 32 - 1];
  return v;
}

// largest i in [0, n) with a[i] <= v (a ascending, a[0] <= v)
template <typename T>
__device__ __forceinline__ int last_le(const T* a, int n, T v) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int m = (lo + hi) >> 1;
    if (a[m] <= v) lo = m; else hi = m;
  }
  return lo;
}

// K/V tile at which position `pos` of the work line cuts a unit of `tiles` tiles that starts at `x`.
__device__ __forceinline__ int cut_tile(long long pos, long long x, int tiles) {
  const long long t = (pos - x - kChunkItemKeys + kChunkTile / 2) >> 7;
  if (t < kChunkSnap) return 0;
  return t > tiles - kChunkSnap ? tiles : static_cast<int>(t);
}

// Work is counted in keys: a unit costs the keys that its last token sees plus a constant for starting it.  All units lie end
// to end on one line.  Whole units are dealt to the workers in rounds (worker c gets units c, c + P, ...) while every worker's sum
// stays within its equal share W / P: they then start neighbouring units at the same time, walk the same keys at the same
// pace and share them through L2.  The units that are left are cut in contiguous shares that fill each worker up to W / P exactly,
// so the split needs at most P - 1 cuts whatever the lengths are.
__global__ void __launch_bounds__(kPlanThreads) chunk_plan_kernel(ChunkParams p) {
  __shared__ Sum2 s_warp[kPlanThreads / 32];
  __shared__ long long s_pos[kMaxPlanCtas + 1], s_cost[kNearSeqs], s_x[kNearUnits + 1];
  __shared__ int s_base[kNearSeqs], s_first[kMaxPlanCtas], s_last[kMaxPlanCtas];
  __shared__ ChunkSeq s_seq[kNearSeqs];
  const int tid = threadIdx.x, P = p.num_workers, B = p.B, Hkv = p.Hkv, ut = p.ut;
  ChunkWork& w = p.work;
  ChunkSeq* seqs = B <= kNearSeqs ? s_seq : w.seq;
  int* base_of = B <= kNearSeqs ? s_base : w.unit_base;
  long long* cost_of = B <= kNearSeqs ? s_cost : w.cost_base;

  launch_dependents();
  // the packed layout has to be an ascending list of starts inside the tensor: everything below relies on it
  int bad = 0;
  for (int b = tid; b < B; b += kPlanThreads) {
    const int s = p.token_start[b], e = p.token_start[b + 1];
    if (s < 0 || e < s || e > p.N) bad = 1;
    if (b < kNearSeqs) s_seq[b] = ChunkSeq{s, e - s, p.seq_lens[b], 0};
  }
  bad = __syncthreads_or(bad);
  if (bad && tid == 0) report_status(p.status, EAGLE_ERR_SEQ);

  // ---- sequences: validity, units and cost, and where both start
  Sum2 carry = {0, 0};
  for (int base = 0; base < B; base += kPlanThreads) {
    const int b = base + tid;
    ChunkSeq q = {0, 0, 0, 0};
    Sum2 v = {0, 0};
    if (b < B) {
      int n;
      if (B <= kNearSeqs) {
        q = s_seq[b];
        n = q.n;
      } else {
        q.start = p.token_start[b];
        q.L = p.seq_lens[b];
        n = p.token_start[b + 1] - q.start;
      }
      q.n = 0;
      if (!bad && n > 0) {
        if (q.L < 0 || static_cast<long long>(q.L) + n > p.capacity) report_status(p.status, EAGLE_ERR_SEQ);
        else q.n = n;
      }
      if (q.n > 0) {
        q.parts = ceil_div(q.n, ut);
        const long long np = q.parts;
        v.a = static_cast<int>(np) * Hkv;
        // sum over the parts of L + (p + 1) UT, but the last one ends at n
        v.b = (np * (static_cast<long long>(q.L) + kChunkItemKeys) + ut * (np * (np + 1) / 2) - (np * ut - q.n)) * Hkv;
      }
    }
    Sum2 tot;
    const Sum2 inc = block_scan(v, s_warp, &tot);
    if (b < B) {
      seqs[b] = q;
      if (seqs != w.seq) w.seq[b] = q;
      w.bad_page[b] = 0;
      base_of[b] = carry.a + inc.a - v.a;
      cost_of[b] = carry.b + inc.b - v.b;
    }
    carry.a += tot.a;
    carry.b += tot.b;
    __syncthreads();
  }
  const int U = carry.a;
  const long long W = carry.b;
  if (tid < P) w.cut[tid].unit = -1;
  if (U == 0) {
    if (tid < P) w.cta[tid] = make_int4(0, 0, 0, 0);
    return;
  }
  long long* x_of = U <= kNearUnits ? s_x : w.x;
  __syncthreads();

  // ---- units: a sequence's parts from the longest to the shortest, KV heads innermost
  auto unit_of = [&](int u, long long* x) {
    const int b = last_le(base_of, B, u);
    const ChunkSeq q = seqs[b];
    const int i = u - base_of[b], r = i / Hkv, pr = q.parts - 1 - r;      // r longer parts come before
    ChunkUnit un;
    un.b = b;
    un.g = i - r * Hkv;
    un.part = pr;
    const long long over = static_cast<long long>(q.parts) * ut - q.n;     // the last part is that much shorter
    const long long keys = q.L + (pr + 1ll) * ut - (r == 0 ? over : 0);
    un.tiles = static_cast<int>((keys + kChunkTile - 1) / kChunkTile);
    if (x) {
      const long long before = r * (static_cast<long long>(q.L) + kChunkItemKeys) +
                               ut * ((static_cast<long long>(q.parts) * (q.parts + 1) - static_cast<long long>(pr + 1) * (pr + 2)) / 2) - (r > 0 ? over : 0);
      *x = cost_of[b] + before * Hkv + un.g * (keys + kChunkItemKeys);
    }
    return un;
  };
  ChunkUnit own = {};                                                      // this thread's first unit, looked up once
  long long own_x = 0;
  if (tid < U) own = unit_of(tid, &own_x);
  for (int u = tid; u < U; u += kPlanThreads) {
    ChunkUnit un = own;
    long long x = own_x;
    if (u != tid) un = unit_of(u, &x);
    w.unit[u] = un;
    x_of[u] = x;
  }
  if (tid == 0) x_of[U] = W;
  __syncthreads();

  // ---- whole units while they fit every worker's share
  const long long T = (W + P - 1) / P;
  long long S = 0;
  int k = 0;
  for (; (k + 1) * P <= U; ++k) {
    long long cost = 0;
    if (tid < P) cost = x_of[k * P + tid + 1] - x_of[k * P + tid];
    if (__syncthreads_or(S + cost > T)) break;
    S += cost;
  }
  const int F = k * P;
  // ---- what is left is shared out so that every worker comes to T
  {
    Sum2 v = {0, tid < P ? T - S : 0}, tot;
    const Sum2 inc = block_scan(v, s_warp, &tot);
    if (tid <= P) {
      const long long at = x_of[F] + inc.b - v.b;
      s_pos[tid] = tid == P || at > W ? W : at;
    }
  }
  __syncthreads();

  const int tiles = p.few ? 1 : 2;                                         // query tiles of a unit, a partial slot each
  auto emit = [&](int at, const ChunkUnit& un, int t0, int t1, int slot) {
    const ChunkSeq q = seqs[un.b];
    int4* it = reinterpret_cast<int4*>(w.items + at);
    it[0] = make_int4(un.b, un.g, un.part, q.start);
    it[1] = make_int4(q.n, q.L, t0, t1);
    it[2] = make_int4(slot, 0, 0, 0);
  };
  // Whole units are items c * k + round.  Of the shares, piece (u, c) of unit u in worker c's share is item u + c; the units in
  // which a share begins and ends are noted for the worker.
  for (int u = tid; u < U; u += kPlanThreads) {
    const ChunkUnit un = u == tid ? own : unit_of(u, nullptr);
    if (u < F) {
      emit((u % P) * k + u / P, un, 0, un.tiles, -1);
      continue;
    }
    const long long x0 = x_of[u], x1 = x_of[u + 1];
    const int c_lo = last_le(s_pos, P, x0);
    int c = c_lo, t0 = 0;
    if (s_pos[c] == x0) s_first[c] = u;
    for (;; ++c) {
      const bool ends = x1 <= s_pos[c + 1];
      const int cut = ends ? un.tiles : cut_tile(s_pos[c + 1], x0, un.tiles), t1 = cut > t0 ? cut : t0;
      emit(u + c, un, t0, t1, t0 == 0 && t1 == un.tiles ? -1 : (2 * c + (t0 > 0 ? 0 : 1)) * tiles);
      if (x1 >= s_pos[c + 1]) s_last[c] = u;
      if (ends) break;
      s_first[c + 1] = u;
      t0 = t1;
    }
    if (c > c_lo) w.cut[c_lo] = ChunkCut{u, c_lo, c, 0};
  }
  __syncthreads();
  if (tid < P) {
    const bool some = s_pos[tid + 1] > s_pos[tid];
    w.cta[tid] = make_int4(tid * k, k, some ? s_first[tid] + tid : 0, some ? s_last[tid] - s_first[tid] + 1 : 0);
  }
}

// ============================================================================================================== attention
constexpr int kThreads = 384;            // two softmax groups of four warps, K/V producer, relay, two MMA issuers (idle in the second CTA)
constexpr int kWarpProducer = 8, kWarpRelay = 9, kWarpQK = 10, kWarpPV = 11;
constexpr int kSBufs = 3;                // score buffers in tensor memory; step g uses buffer g % 3
constexpr int kKSlots = 5, kVSlots = 4;  // rings of half tiles; step g's tiles lie in slots g % 5 and g % 4
constexpr uint32_t kTmemCols = 512;      // S0 S1 S2 | O; P (packed bf16, 64 columns) overwrites the front of its S
constexpr uint32_t kColO = 384;
constexpr float kRescaleThreshold = 8.0f;   // log2 units: the accumulator is rescaled when the row maximum outgrows its reference by more
// One pair of exponentials in so many is a polynomial on the FMA pipe, beside the special-function unit (a prompt of 4096 tokens x 32
// heads: 172 us with none, 160 us with one in 3 or two in 3, 154 us with one in 2, 206 us with all; where the power limit sets the clock,
// one in 2 and one in 3 are within 0.5 %).
constexpr int kPolyStride = 2;

template <int D>
struct Smem {
  static constexpr int kSlabs = D / 64;                      // 64 bf16 = one 128-byte swizzled row
  static constexpr int kQSlab = 128 * 128, kQBytes = kSlabs * kQSlab;
  static constexpr int kKSlab = 64 * 128, kKBytes = kSlabs * kKSlab;     // half a K tile: 64 keys
  static constexpr int kVBytes = 128 * D;                    // half a V tile: 128 keys x D / 2 columns
  static constexpr int kQ = 0;                               // two query tiles: the current item's and the next one's
  static constexpr int kK = 2 * kQBytes;
  static constexpr int kV = kK + kKSlots * kKBytes;
  static constexpr int kTag = kV + kVSlots * kVBytes;        // uint64 [128 rows]: step number | reference maximum
  static constexpr int kLfin = kTag + 128 * 8;               // uint64 [2][128 rows]: item number | row sum on its way to the output, by items in turn
  static constexpr int kBar = kLfin + 2 * 128 * 8;
  static constexpr int kNumBars = 2 * (kKSlots + 2) + 3 * kVSlots + 3 * kSBufs + 1;
  static constexpr int kMisc = kBar + 8 * kNumBars;          // tensor-memory base, abort flag, wait limit (8 bytes)
  static constexpr int kBytes = kMisc + 16;
};

// The same places in both CTAs.  ready: a tile has landed in both (first CTA only); full: this CTA's half of a V tile has
// landed; empty: the MMAs have finished with the slot (both CTAs).
struct Bars {
  uint32_t base;
  static constexpr uint32_t kVAt = 2 * kKSlots, kQAt = kVAt + 3 * kVSlots, kSAt = kQAt + 4;
  __device__ __forceinline__ uint32_t at(uint32_t i) const { return base + 8u * i; }
  __device__ __forceinline__ uint32_t k_ready(uint32_t i) const { return at(i); }
  __device__ __forceinline__ uint32_t k_empty(uint32_t i) const { return at(kKSlots + i); }
  __device__ __forceinline__ uint32_t v_full(uint32_t i) const { return at(kVAt + i); }
  __device__ __forceinline__ uint32_t v_ready(uint32_t i) const { return at(kVAt + kVSlots + i); }
  __device__ __forceinline__ uint32_t v_empty(uint32_t i) const { return at(kVAt + 2 * kVSlots + i); }
  __device__ __forceinline__ uint32_t q_ready(uint32_t i) const { return at(kQAt + i); }
  __device__ __forceinline__ uint32_t q_empty(uint32_t i) const { return at(kQAt + 2 + i); }
  __device__ __forceinline__ uint32_t s_full(uint32_t i) const { return at(kSAt + i); }                  // scores of a step (both CTAs)
  __device__ __forceinline__ uint32_t p_full(uint32_t i) const { return at(kSAt + kSBufs + i); }         // its probabilities (first CTA only)
  __device__ __forceinline__ uint32_t o_done(uint32_t i) const { return at(kSAt + 2 * kSBufs + i); }     // its PV has finished (both CTAs)
  __device__ __forceinline__ uint32_t o_free() const { return at(kSAt + 3 * kSBufs); }                   // an item's accumulators have been read (first CTA only)
};

// A float with a number, written and read in one piece.
__device__ __forceinline__ unsigned long long tagged(uint32_t number, float x) { return static_cast<unsigned long long>(number) << 32 | __float_as_uint(x); }
__device__ __forceinline__ float value_of(unsigned long long t) { return __uint_as_float(static_cast<uint32_t>(t)); }
__device__ __forceinline__ bool has_tag(unsigned long long t, uint32_t want) { return static_cast<uint32_t>(t >> 32) == want; }
// Bounded wait for the word with number `want` in shared memory; one with another number when the CTA was aborted or the time
// limit passed.
__device__ __noinline__ unsigned long long tag_wait_slow(volatile unsigned long long* slot, uint32_t want, volatile int* abort_flag) {
  const unsigned long long t0 = global_timer(), limit = *reinterpret_cast<volatile unsigned long long*>(abort_flag + 1);
  for (uint32_t spins = 1;; ++spins) {
    const unsigned long long t = *slot;
    if (has_tag(t, want)) return t;
    if ((spins & 63u) == 0) {
      if (*abort_flag) return tagged(~want, 0.f);
      if (global_timer() - t0 > limit) {
        *abort_flag = 1;
        return tagged(~want, 0.f);
      }
    }
    __nanosleep(20);
  }
}
__device__ __forceinline__ unsigned long long tag_wait(volatile unsigned long long* slot, uint32_t want, volatile int* abort_flag) {
  const unsigned long long t = *slot;
  if (has_tag(t, want)) return t;
  return tag_wait_slow(slot, want, abort_flag);
}

// (STALL: of the test hook that lets the waits run out, an instantiation of its own because the comparison would cost every other
// call 2 to 3 %.)
template <int D, bool PAGED, bool STALL>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
chunk_attn_kernel(ChunkParams p, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                  const __grid_constant__ CUtensorMap map_q) {
  using S = Smem<D>;
  extern __shared__ __align__(1024) unsigned char smem[];
  const uint32_t sbase = smem_u32(smem);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = cluster_rank();
  if (sbase & 1023u) {   // the swizzled tiles need a 1024-byte aligned base; uniform over the launch
    if (tid == 0) report_status(p.status, EAGLE_ERR_DEVICE);
    return;
  }
  Bars B;
  B.base = sbase + S::kBar;
  volatile uint32_t* s_tmem = reinterpret_cast<volatile uint32_t*>(smem + S::kMisc);
  volatile int* s_abort = reinterpret_cast<volatile int*>(smem + S::kMisc + 4);

  if (tid == 0) {
    prefetch_map(&map_k);
    prefetch_map(&map_v);
    prefetch_map(&map_q);
    for (int i = 0; i < kKSlots; ++i) { mbar_init(B.k_ready(i), 1); mbar_init(B.k_empty(i), 1); }
    for (int i = 0; i < kVSlots; ++i) { mbar_init(B.v_full(i), 1); mbar_init(B.v_ready(i), 2); mbar_init(B.v_empty(i), 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(B.q_ready(i), 1); mbar_init(B.q_empty(i), 1); }
    for (int i = 0; i < kSBufs; ++i) {
      mbar_init(B.s_full(i), 1);
      mbar_init(B.p_full(i), 8);           // a group's four warps, in both CTAs
      mbar_init(B.o_done(i), 1);
    }
    mbar_init(B.o_free(), 8);
    *s_abort = 0;
    *reinterpret_cast<volatile unsigned long long*>(smem + S::kMisc + 8) = p.wait_limit_ns;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (tid < 3 * 128) reinterpret_cast<volatile unsigned long long*>(smem + S::kTag)[tid] = ~0ull;   // (kLfin too) no step and no item has this number
  if (warp == kWarpQK) {
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

  if (warp == kWarpProducer) {
    // =========================================================================== copies
    // Order: K(0), K(1), K(2), then V(g), K(g + 3), g counting this pair's steps over all items (the score MMA runs up to three
    // steps ahead of the PV MMA); an item's query tile goes with its first K tile.  Each CTA's producer fetches its own halves; K
    // and query tiles report to the first CTA's barrier, V tiles to the relay of their own CTA.  A lane per box (a page, or a
    // 64-column half); the page of a lane's next box is looked up while the box before it is on its way.
    struct Cursor {
      Item it;
      int i, tile, end;
      int y, page;                         // this lane's next box: row in its page (or in the sequence), page (or sequence)
      bool valid, fresh;
      bool wrong;                          // some entry of the item was outside the pool
    };
    const int k_rows = PAGED ? min(p.page_size, 64) : 64, v_rows = PAGED ? min(p.page_size, kChunkTile) : kChunkTile;
    const int k_r0 = (lane / S::kSlabs) * k_rows, v_r0 = lane * v_rows, half = static_cast<int>(rank);
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
        c.tile = c.it.t0;
        c.end = c.it.t1;
        c.fresh = true;
      }
      const int r0 = is_v ? v_r0 : k_r0, key = c.tile * kChunkTile + (is_v ? 0 : half * 64) + r0;
      c.y = key;
      c.page = c.it.b;
      if (PAGED && r0 < (is_v ? kChunkTile : 64)) {
        // a box past the sequence's last page fetches that page again (its rows are masked), so that a tile's byte count never changes
        const int last = (c.it.L + c.it.n - 1) >> p.page_shift, pi = key >> p.page_shift;
        c.page = __ldg(p.block_table + static_cast<size_t>(c.it.b) * p.max_pages + (pi < last ? pi : last));
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
    Ring<kKSlots> kr;
    Ring<kVSlots> vr;
    uint32_t q_items = 0;
    Cursor ck, cv;
    ck.i = cv.i = -1;
    ck.tile = ck.end = cv.tile = cv.end = 0;
    ck.valid = cv.valid = true;
    ck.wrong = cv.wrong = false;
    advance(ck, false);
    advance(cv, true);
    [[maybe_unused]] int keys = 0, values = 0;                     // tiles issued
    auto next_key = [&]() {
      if (!ck.valid || !ok) return;
      if constexpr (STALL) {
        if (keys++ >= p.stall_after_tiles) return;
      }
      if (ck.fresh) {
        // box of TPT tokens x G heads x 64 columns: rows land in (token, head) order; rows of the next sequence (or zeros past
        // the tensor) that come along are computed and never written
        const uint32_t qb = q_items & 1u;
        ok = mbar_wait_warp(B.q_empty(qb), ((q_items >> 1) & 1u) ^ 1u, s_abort);
        if (!ok) return;
        if (lane == 0) {
          if (rank == 0) mbar_expect_tx(B.q_ready(qb), 2 * S::kSlabs * p.tpt * p.G * 128);
#pragma unroll
          for (int sl = 0; sl < S::kSlabs; ++sl)
            tma_load_3d_pair(sbase + S::kQ + qb * S::kQBytes + sl * S::kQSlab, &map_q, sl * 64, ck.it.g * p.G,
                             ck.it.start + (2 * ck.it.part + half) * p.tpt, B.q_ready(qb) + to_first);
        }
        ++q_items;
      }
      ok = mbar_wait_warp(B.k_empty(kr.slot), kr.par ^ 1u, s_abort);
      if (!ok) return;
      if (lane == 0 && rank == 0) mbar_expect_tx(B.k_ready(kr.slot), 2 * S::kKBytes);
      const int sl = lane % S::kSlabs;
      if (k_r0 < 64)
        tma_load_3d_pair(sbase + S::kK + kr.slot * S::kKBytes + sl * S::kKSlab + k_r0 * 128, &map_k, sl * 64, ck.y, place(ck),
                         B.k_ready(kr.slot) + to_first);
      kr.step();
      advance(ck, false);
    };
    for (int i = 0; i < 3; ++i) next_key();
    while (cv.valid && ok) {
      if constexpr (STALL) {
        if (values++ >= p.stall_after_tiles) break;
      }
      ok = mbar_wait_warp(B.v_empty(vr.slot), vr.par ^ 1u, s_abort);
      if (!ok) break;
      if (lane == 0) mbar_expect_tx(B.v_full(vr.slot), S::kVBytes);
      __syncwarp();
      if (v_r0 < kChunkTile)
        tma_load_3d(sbase + S::kV + vr.slot * S::kVBytes + v_r0 * D, &map_v, half * (D / 2), cv.y, place(cv), B.v_full(vr.slot));
      vr.step();
      advance(cv, true);
      next_key();
    }
  } else if (warp == kWarpRelay) {
    // =========================================================================== V tiles that have landed
    // The rows of V past the sequence may hold anything, and 0 * garbage must not reach O: they are zeroed here before the first
    // CTA's issuer hears of the tile.
    bool ok = true;
    Ring<kVSlots> vr;
    uint32_t steps = 0, items = 0;
    const uint32_t to_first = map_to_rank(sbase, 0) - sbase;
    for (int i = 0; i < n_items && ok; ++i) {
      const Item it = item(i);
      items += it.t1 > it.t0 ? 1u : 0u;
      for (int t = it.t0; t < it.t1; ++t, ++steps, vr.step()) {
        ok = mbar_wait_warp(B.v_full(vr.slot), vr.par, s_abort);
        if (!ok) break;
        const int valid = it.L + it.n - t * kChunkTile;            // keys of the tile that belong to the sequence
        if (valid < kChunkTile) {
          for (int j = valid * (D / 16) + lane; j < kChunkTile * (D / 16); j += 32)        // whole rows of D bytes, so the swizzle does not matter
            *reinterpret_cast<uint4*>(smem + S::kV + vr.slot * S::kVBytes + j * 16) = make_uint4(0u, 0u, 0u, 0u);
          fence_proxy_async();
          __syncwarp();
          if (lane == 0) mbar_arrive_release_pair(B.v_ready(vr.slot) + to_first);
        } else if (lane == 0) {
          mbar_arrive_pair(B.v_ready(vr.slot) + to_first);
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
  } else if (warp == kWarpQK) {
    // =========================================================================== S = Q K^T, up to three steps ahead of the softmax
    if (lane == 0 && rank == 0) {
      constexpr uint32_t idesc = instr_desc(256, kChunkTile, false);
      const uint32_t q_lo = desc_lo(sbase + S::kQ), k_lo = desc_lo(sbase + S::kK);
      Ring<kKSlots> kr;
      Ring<kSBufs> sr;
      uint32_t steps = 0, items = 0;
      bool ok = true;
      for (int i = 0; i < n_items && ok; ++i) {
        const Item it = item(i);
        if (it.t1 <= it.t0) continue;
        const uint32_t qb = items & 1u;
        ok = mbar_wait(B.q_ready(qb), (items >> 1) & 1u, s_abort);
        for (int t = it.t0; t < it.t1 && ok; ++t, ++steps) {
          ok = mbar_wait(B.k_ready(kr.slot), kr.par, s_abort);
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
  } else if (warp == kWarpPV) {
    // =========================================================================== O += P V
    if (lane == 0 && rank == 0) {
      constexpr uint32_t idesc = instr_desc(256, D, true);
      const uint32_t v_lo = desc_lo(sbase + S::kV);
      Ring<kVSlots> vr;
      Ring<kSBufs> sr;
      uint32_t items = 0;
      bool ok = true;
      for (int i = 0; i < n_items && ok; ++i) {
        const Item it = item(i);
        if (it.t1 <= it.t0) continue;
        for (int t = it.t0; t < it.t1 && ok; ++t) {
          ok = mbar_wait(B.v_ready(vr.slot), vr.par, s_abort);
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
    // =========================================================================== softmax and output
    // Two groups of four warps take alternate steps, so that one computes while the other waits.  Thread r of a group owns query
    // row r (tensor-memory lane r), all 128 score columns.  The two threads of a row share one reference maximum: the one
    // that handled step g publishes it, tagged with g, before it takes its exponentials, and the other picks it up at step g + 1;
    // each keeps its own part of the row sum.  The reference is a whole fp32 number: what is left between it and the product that it
    // stands for is within half a step for all of a row's exponentials alike, so it cancels, however large the scores are.  fp32 throughout, in the log2 domain; the probabilities are rounded to bf16 for
    // the tensor cores (relative 2^-8 each, half of the inputs' own spacing), the sum that divides them is kept from the
    // unrounded ones.  A warp without a row that belongs to the sequence only passes its turns on.
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
      const int first = (2 * it.part + static_cast<int>(rank)) * p.tpt, token = first + tok_r;    // place in the chunk
      const bool row_valid = tok_r < p.tpt && token < it.n;
      const bool warp_rests = !__any_sync(0xffffffffu, row_valid);
      const int limit = it.L + (token < it.n ? token : it.n - 1);                 // the last key this row sees
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
          const int key0 = (it.t0 + s) * kChunkTile;
          if (key0 + kChunkTile - 1 > it.L + first) {
            // a tile that some row of this query tile does not see whole: -inf over the invisible scores, in place
            const int lim = limit - key0;                  // last visible column of this row
            const int lim_lo = __reduce_min_sync(0xffffffffu, lim), lim_hi = __reduce_max_sync(0xffffffffu, lim);
#pragma unroll 1
            for (int c = 0; c < 4; ++c) {
              if (lim_lo >= c * 32 + 31) continue;         // uniform: every row of the warp sees the whole chunk
              const int v = lim - c * 32;
              const uint32_t see = v >= 31 ? 0xffffffffu : (v < 0 ? 0u : (2u << v) - 1u);
              uint32_t t[32];
              if (lim_hi >= c * 32) {                      // (uniform too: some row sees some of it)
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
          // ---- row maximum.  Chunks 0 and 1 stay in registers, chunks 2 and 3 are fetched again for the exponentials.
          uint32_t ra[32], rb[32];
          float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
          {
            uint32_t rc[32], rd[32];
            ld32(s_addr + 64, rc);
            ld32(s_addr + 96, rd);
            ld32(s_addr, ra);
            ld32(s_addr + 32, rb);
            wait_ld();
#pragma unroll
            for (int e = 0; e < 32; e += 2) {
              mx[0] = max3_nan(mx[0], __uint_as_float(rc[e]), __uint_as_float(rc[e + 1]));
              mx[1] = max3_nan(mx[1], __uint_as_float(rd[e]), __uint_as_float(rd[e + 1]));
              mx[2] = max3_nan(mx[2], __uint_as_float(ra[e]), __uint_as_float(ra[e + 1]));
              mx[3] = max3_nan(mx[3], __uint_as_float(rb[e]), __uint_as_float(rb[e + 1]));
            }
          }
          const float tmax = max3_nan(max3_nan(mx[0], mx[1], mx[2]), mx[3], -INFINITY) * scale_log2;   // scale > 0
          // a visible score that is NaN or +inf makes the row NaN (through its sum: not every exponential below passes one on)
          if (!(tmax < INFINITY)) l_sum = __uint_as_float(0x7fffffffu);

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
          const uint64_t scale2 = pack2(scale_log2, scale_log2), base2 = pack2(neg_base, neg_base);
          uint64_t ls2[2] = {0ull, 0ull};
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
          {
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
            // The accumulator is given back as soon as it is in registers: the next item's first PV waits for that.
            uint32_t o[D];
#pragma unroll
            for (int c = 0; c < D / 32; ++c) ld32(o_addr + c * 32, o + c * 32);
            wait_ld();
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_pair(o_free_to);
            if (row_valid && slot < 0) {
              __nv_bfloat16* out_row = p.out + (static_cast<size_t>(it.start + token) * p.Hq + it.g * p.G + head_r) * D;
#pragma unroll
              for (int e = 0; e < D; e += 16) {
                uint32_t v[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = pack_bf16(__uint_as_float(o[e + 2 * k]) * inv, __uint_as_float(o[e + 2 * k + 1]) * inv);
                st_global_v8(out_row + e, v);
              }
            } else if (row_valid) {
              // an fp32 partial is laid out [4 columns][row], so that the lanes of a store write consecutive 16-byte pieces
              float* part = p.work.part_o + static_cast<size_t>(slot) * (D / 4) * (128 * 4) + r * 4;
#pragma unroll
              for (int e = 0; e < D; e += 4)
                *reinterpret_cast<uint4*>(part + (e / 4) * (128 * 4)) = make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]);
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
  if (warp == kWarpQK) {
    __syncwarp();
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
  }
}

// ================================================================================================================== merge
// Cut query tiles: m* = max m_i, l* = sum l_i 2^(m_i - m*), out = sum o_i 2^(m_i - m*) / l*.  A block takes 8 rows of one query
// tile of one record (a warp: 8 rows x 4 groups of 4 columns, so that its loads are runs of 128 bytes); the slots of the
// pieces are looked up together, and four pieces' loads are in flight at a time.  The blocks behind them look at one sequence
// each: rows of a sequence that does not fit its cache, or whose block table names a page outside the pool, become zeros.  Nothing
// orders the two kinds of blocks, so those of a cut unit leave the rows of such a sequence alone; every page in use has been copied
// from by some worker, so the attention kernel has looked at all of them.
constexpr int kMergeThreads = 256;

template <int D>
__global__ void __launch_bounds__(kMergeThreads) chunk_merge_kernel(ChunkParams p, int row_blocks) {
  wait_for_prerequisites();                              // partials and outputs of the attention kernel are there
  const ChunkWork& w = p.work;
  const int tid = threadIdx.x, records = p.num_workers, halves = p.few ? 1 : 2;
  if (static_cast<int>(blockIdx.x) >= records * halves * row_blocks) {
    const int b = blockIdx.x - records * halves * row_blocks;
    const ChunkSeq q = w.seq[b];
    const int s = p.token_start[b], e = p.token_start[b + 1];
    if (s < 0 || e <= s || e > p.N) return;
    const bool wrong = w.bad_page[b] != 0;
    if (wrong && tid == 0) report_status(p.status, EAGLE_ERR_PAGE);
    if (q.n > 0 && !wrong) return;                       // (n = 0: the planner refused it, and reported it)
    uint4* out = reinterpret_cast<uint4*>(p.out + static_cast<size_t>(s) * p.Hq * D);
    const size_t vecs = static_cast<size_t>(e - s) * p.Hq * (D / 8);
    for (size_t i = tid; i < vecs; i += kMergeThreads) out[i] = make_uint4(0u, 0u, 0u, 0u);
    return;
  }
  __shared__ int s_slot[kMaxPlanCtas];                      // slots of the pieces that are not empty, in order
  __shared__ int s_count;
  const int rec = blockIdx.x / (halves * row_blocks), rest = blockIdx.x - rec * halves * row_blocks, half = rest / row_blocks, rb = rest - half * row_blocks;
  const ChunkCut cut = w.cut[rec];
  if (cut.unit < 0) return;
  const ChunkUnit un = w.unit[cut.unit];
  const ChunkSeq q = w.seq[un.b];
  const int first = un.part * p.ut + half * p.tpt;
  if (first + rb * 8 / p.G >= q.n || rb * 8 / p.G >= p.tpt) return;      // no row of this block belongs to the sequence
  if (w.bad_page[un.b]) return;
  if (tid < 32) {
    int count = 0;
    for (int i = cut.c_lo; i <= cut.c_hi; i += 32) {
      const int c = i + tid;
      int slot = -1;
      if (c <= cut.c_hi) {
        const ChunkItem* it = w.items + cut.unit + c;
        if (it->t1 > it->t0) slot = it->slot;
      }
      const unsigned has = __ballot_sync(0xffffffffu, slot >= 0);
      if (slot >= 0) s_slot[count + __popc(has & ((1u << tid) - 1u))] = slot + half;
      count += __popc(has);
    }
    if (tid == 0) s_count = count;
  }
  __syncthreads();
  const int pieces = s_count;                            // 0: the cuts snapped to the unit's edges, its output is there already
  const int row = rb * 8 + ((tid >> 2) & 7), cols = (tid >> 5) * 4 + (tid & 3);      // row of the tile, group of 4 columns
  const int tok = row / p.G, head = row - tok * p.G, token = first + tok;
  if (pieces == 0 || tok >= p.tpt || token >= q.n || cols >= D / 4) return;
  float m = -INFINITY, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int i = 0; i < pieces; i += 4) {
    float2 ml[4];
    float4 v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      ml[k] = make_float2(-INFINITY, 0.f);
      v[k] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (i + k < pieces) {
        const size_t slot = s_slot[i + k];
        ml[k] = w.part_ml[slot * p.rows + row];
        v[k] = *reinterpret_cast<const float4*>(w.part_o + (slot * (D / 4) + cols) * (p.rows * 4) + row * 4);
      }
    }
    const float top = fmaxf(fmaxf(fmaxf(ml[0].x, ml[1].x), fmaxf(ml[2].x, ml[3].x)), m);
    const float base = top == -INFINITY ? 0.f : top;     // (nothing visible so far: every weight is 2^-inf)
    const float a = exp2f(m - base);
    l *= a;
    o = make_float4(o.x * a, o.y * a, o.z * a, o.w * a);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      // a piece in which the row sees nothing has m = -inf and l = 0, and an accumulator that the weight 0 keeps out
      const float c = exp2f(ml[k].x - base);
      l = fmaf(ml[k].y, c, l);
      o = make_float4(fmaf(v[k].x, c, o.x), fmaf(v[k].y, c, o.y), fmaf(v[k].z, c, o.z), fmaf(v[k].w, c, o.w));
    }
    m = top;
  }
  const float inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);
  uint2 out;
  out.x = pack_bf16(o.x * inv, o.y * inv);
  out.y = pack_bf16(o.z * inv, o.w * inv);
  *reinterpret_cast<uint2*>(p.out + (static_cast<size_t>(q.start + token) * p.Hq + un.g * p.G + head) * D + cols * 4) = out;
}

template <int D>
cudaError_t launch_tiles(const ChunkParams& p, cudaStream_t stream) {
  CUtensorMap mk, mv, mq;
  const bool paged = p.block_table != nullptr;
  const int k_rows = paged && p.page_size < 64 ? p.page_size : 64, v_rows = paged && p.page_size < 128 ? p.page_size : 128;
  const long long n1 = paged ? p.page_size : (p.capacity > 0 ? p.capacity : 1);
  const long long n2 = paged ? static_cast<long long>(p.num_pages) * p.Hkv : static_cast<long long>(p.B) * p.Hkv;
  if (!map_bf16_3d(&mk, p.k, D, n1, n2, 64, k_rows, 1) || !map_bf16_3d(&mv, p.v, D, n1, n2, D / 2, v_rows, 1) ||
      !map_bf16_3d(&mq, p.q, D, p.Hq, p.N, 64, p.G, p.tpt))
    return cudaErrorInvalidValue;
  BehindLaunch at(2 * p.num_workers, kThreads, Smem<D>::kBytes, stream);
  auto kernel = p.stall_after_tiles >= 0 ? (paged ? chunk_attn_kernel<D, true, true> : chunk_attn_kernel<D, false, true>)
                                         : (paged ? chunk_attn_kernel<D, true, false> : chunk_attn_kernel<D, false, false>);
  return cudaLaunchKernelEx(&at.config, kernel, p, mk, mv, mq);
}

template <int D>
cudaError_t launch_all(const ChunkParams& p, cudaStream_t stream) {
  // Both kernels after the planner are launched programmatically: their prologues (and the launches themselves) overlap the
  // kernel before, whose results they wait for.
  chunk_plan_kernel<<<1, kPlanThreads, 0, stream>>>(p);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  count_launch();
  e = p.few ? launch_chunk_rows(p, stream) : launch_tiles<D>(p, stream);
  if (e != cudaSuccess) return e;
  count_launch();
  const int rows = p.max_rows < p.rows ? p.max_rows : p.rows, row_blocks = (rows + 7) / 8;
  BehindLaunch at(p.num_workers * (p.few ? 1 : 2) * row_blocks + p.B, kMergeThreads, 0, stream);
  e = cudaLaunchKernelEx(&at.config, chunk_merge_kernel<D>, p, row_blocks);
  if (e != cudaSuccess) return e;
  count_launch();
  return cudaSuccess;
}

template <int D>
cudaError_t prepare() {
  for (auto kernel : {chunk_attn_kernel<D, false, false>, chunk_attn_kernel<D, true, false>, chunk_attn_kernel<D, false, true>, chunk_attn_kernel<D, true, true>}) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Smem<D>::kBytes);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace

cudaError_t chunk_prepare(int head_dim) { return head_dim == 128 ? prepare<128>() : prepare<64>(); }

cudaError_t launch_chunk(const ChunkParams& p, cudaStream_t stream) { return p.D == 128 ? launch_all<128>(p, stream) : launch_all<64>(p, stream); }

}  // namespace eagle
