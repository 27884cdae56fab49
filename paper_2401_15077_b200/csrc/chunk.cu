// Causal attention of packed chunks of new tokens over the cache they have just been written to (contiguous or paged).
//
//   out[t] = sum_j softmax_j(scale * q[t].k[j]) v[j],  j <= L_b + i, for token t = token_start[b] + i of sequence b.
//
// Three launches: a planner (one CTA), the attention kernel (one persistent CTA per SM) and the merge of what was cut.
//
// A query tile is 128 rows of one (sequence, KV head): TPT = 128 / G tokens (rounded down) times the G heads of the group.
// A CTA runs two *streams* side by side, each with its own query tile, score buffer, accumulator and softmax warps:
//   - a pair: query tiles 2p and 2p + 1 of one (sequence, KV head) over the same K/V tiles, which are loaded once;
//   - a twin: the odd last query tile of two neighbouring KV heads, each with its own K/V tiles;
//   - a lone tile (odd number of KV heads): one query tile, the streams take the two halves of its keys.
// While one stream's softmax works on its scores the tensor pipe runs the other stream's products, so neither waits for the
// other as long as a softmax step is shorter than two products of 128 x 128 x D.
#include "chunk.cuh"
#include "tc.cuh"

namespace eagle {

namespace {

using namespace tc;

// ================================================================================================================ planner
constexpr int kPlanThreads = 1024;

__device__ __forceinline__ int ceil_div(int a, int b) { return (a + b - 1) / b; }

// Keys that query tile `qt` of a sequence sees at the most: the prefix and the tile's last token.
__device__ __forceinline__ long long tile_keys(int L, int n, int qt, int tpt) {
  const long long last = static_cast<long long>(qt + 1) * tpt;
  return L + (last < n ? last : n);
}

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
    Sum2 t = warp_tot[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int a = __shfl_up_sync(0xffffffffu, t.a, o);
      const long long b = __shfl_up_sync(0xffffffffu, t.b, o);
      if (lane >= o) { t.a += a; t.b += b; }
    }
    warp_tot[lane] = t;
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

// K/V tile (of the unit's rounds) at which position `pos` of the work line cuts a unit that starts at `x`.
__device__ __forceinline__ int cut_round(long long pos, long long x, int rounds) {
  const long long t = (pos - x - kChunkItemKeys + kChunkTile / 2) >> 7;
  if (t < kChunkSnap) return 0;
  return t > rounds - kChunkSnap ? rounds : static_cast<int>(t);
}

// Work is counted in keys: a unit (pair, twin, lone) costs the keys of its longer stream plus a constant for starting it.
// All units lie end to end on one line.  Whole units are dealt to the CTAs in rounds (CTA c gets units c, c + P, ...) while
// every CTA's sum stays within its equal share W / P: CTAs then start neighbouring units at the same time, walk the same
// keys at the same pace and share them through L2.  The units that are left are cut in contiguous shares that fill each
// CTA up to W / P exactly, so the split needs at most P - 1 cuts whatever the lengths are.
__global__ void __launch_bounds__(kPlanThreads) chunk_plan_kernel(ChunkParams p) {
  __shared__ Sum2 s_warp[kPlanThreads / 32];
  __shared__ long long s_pos[kMaxPlanCtas + 1];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, P = p.num_ctas, B = p.B, Hkv = p.Hkv;
  ChunkWork& w = p.work;

  // the packed layout has to be an ascending list of starts inside the tensor: everything below relies on it
  int bad = 0;
  for (int b = tid; b <= B; b += kPlanThreads) {
    const int s = p.token_start[b];
    if (s < 0 || s > p.N || (b < B && p.token_start[b + 1] < s)) bad = 1;
  }
  bad = __syncthreads_or(bad);
  if (bad && tid == 0) report_status(p.status, EAGLE_ERR_SEQ);

  // ---- sequences: validity, units and cost, and where both start
  const int singles = (Hkv + 1) / 2;                 // units of an odd last query tile: twins and, if Hkv is odd, a lone one
  Sum2 carry = {0, 0};
  for (int base = 0; base < B; base += kPlanThreads) {
    const int b = base + tid;
    ChunkSeq q = {0, 0, 0, 0};
    Sum2 v = {0, 0};
    if (b < B) {
      const int s = p.token_start[b], e = p.token_start[b + 1];
      q.L = p.seq_lens[b];
      q.start = s;
      if (!bad && e > s) {
        if (q.L < 0 || static_cast<long long>(q.L) + (e - s) > p.capacity) report_status(p.status, EAGLE_ERR_SEQ);
        else q.n = e - s;
      }
      if (q.n > 0) {
        q.qtiles = ceil_div(q.n, p.tpt);
        const long long np = q.qtiles / 2, keys = static_cast<long long>(q.L) + q.n;
        v.a = static_cast<int>(np) * Hkv;
        // sum over the pairs of L + (2p + 2) TPT, the last one's end being n
        long long pairs = np * (q.L + kChunkItemKeys) + p.tpt * np * (np + 1);
        if (np > 0 && !(q.qtiles & 1)) pairs -= static_cast<long long>(q.qtiles) * p.tpt - q.n;
        v.b = pairs * Hkv;
        if (q.qtiles & 1) {
          v.a += singles;
          v.b += (Hkv / 2) * (keys + kChunkItemKeys);
          if (Hkv & 1) v.b += (keys + 1) / 2 + kChunkItemKeys;
        }
      }
    }
    Sum2 tot;
    const Sum2 inc = block_scan(v, s_warp, &tot);
    if (b < B) {
      w.seq[b] = q;
      w.unit_base[b] = carry.a + inc.a - v.a;
      w.cost_base[b] = carry.b + inc.b - v.b;
      w.cut[P + b].unit = -1;
    }
    carry.a += tot.a;
    carry.b += tot.b;
    __syncthreads();
  }
  const int U = carry.a;
  const long long W = carry.b;
  for (int c = tid; c < P; c += kPlanThreads) w.cut[c].unit = -1;
  if (U == 0) {
    for (int c = tid; c < P; c += kPlanThreads) w.cta[c] = make_int4(0, 0, 0, 0);
    return;
  }
  __syncthreads();

  // ---- units: the odd last query tile first, then the pairs from the longest to the shortest, KV heads innermost
  for (int u = tid; u < U; u += kPlanThreads) {
    const int b = last_le(w.unit_base, B, u);
    const ChunkSeq q = w.seq[b];
    int i = u - w.unit_base[b];
    long long x = w.cost_base[b];
    const long long keys = static_cast<long long>(q.L) + q.n;
    ChunkUnit un;
    un.b = b;
    un.pad = 0;
    const int first = q.qtiles & 1 ? singles : 0;
    if (i < first) {
      un.g = 2 * i;
      un.qt = q.qtiles - 1;
      un.kind = 2 * i + 1 < Hkv ? kChunkTwin : kChunkLone;
      x += i * (keys + kChunkItemKeys);
    } else {
      i -= first;
      const int np = q.qtiles / 2, r = i / Hkv, pr = np - 1 - r;     // pairs pr + 1 .. np - 1 come before
      un.g = i - r * Hkv;
      un.qt = 2 * pr;
      un.kind = kChunkPair;
      if (first) x += (Hkv / 2) * (keys + kChunkItemKeys) + (Hkv & 1 ? (keys + 1) / 2 + kChunkItemKeys : 0);
      long long before = static_cast<long long>(r) * (q.L + kChunkItemKeys) +
                         p.tpt * (static_cast<long long>(np) * (np + 1) - static_cast<long long>(pr + 1) * (pr + 2));
      const long long over = q.qtiles & 1 ? 0 : static_cast<long long>(q.qtiles) * p.tpt - q.n;   // the last pair is that much shorter
      if (r > 0) before -= over;
      long long one = q.L + kChunkItemKeys + static_cast<long long>(2 * pr + 2) * p.tpt;
      if (r == 0) one -= over;
      x += before * Hkv + un.g * one;
    }
    un.nt[0] = static_cast<int>((tile_keys(q.L, q.n, un.qt, p.tpt) + kChunkTile - 1) / kChunkTile);
    un.nt[1] = un.kind == kChunkPair ? static_cast<int>((tile_keys(q.L, q.n, un.qt + 1, p.tpt) + kChunkTile - 1) / kChunkTile) : un.nt[0];
    w.unit[u] = un;
    w.x[u] = x;
  }
  if (tid == 0) w.x[U] = W;
  __syncthreads();

  // ---- whole units while they fit every CTA's share
  const long long T = (W + P - 1) / P;
  long long S = 0;
  int k = 0;
  for (; (k + 1) * P <= U; ++k) {
    long long cost = 0;
    if (tid < P) cost = w.x[k * P + tid + 1] - w.x[k * P + tid];
    if (__syncthreads_or(S + cost > T)) break;
    S += cost;
  }
  const int F = k * P;
  // ---- what is left is shared out so that every CTA comes to T
  {
    Sum2 v = {0, tid < P ? T - S : 0}, tot;
    const Sum2 inc = block_scan(v, s_warp, &tot);
    if (tid <= P) {
      const long long at = w.x[F] + inc.b - v.b;
      s_pos[tid] = tid == P || at > W ? W : at;
    }
  }
  __syncthreads();

  auto emit = [&](int slot_index, int u, int r0, int r1, int part) {   // rounds [r0, r1) of unit u; part < 0: all of it
    const ChunkUnit un = w.unit[u];
    const ChunkSeq q = w.seq[un.b];
    ChunkItem it;
    it.b = un.b;
    it.kind = un.kind;
    it.start = q.start;
    it.n = q.n;
    it.L = q.L;
    it.pad = 0;
    it.g[0] = un.g;
    it.g[1] = un.kind == kChunkTwin ? un.g + 1 : un.g;
    it.qt[0] = un.qt;
    it.qt[1] = un.kind == kChunkPair ? un.qt + 1 : un.qt;
    const int half = un.kind == kChunkLone ? (un.nt[0] + 1) / 2 : 0;
    const int end0 = un.kind == kChunkLone ? half : un.nt[0], end1 = un.nt[1];
    it.t0[0] = r0;
    it.t1[0] = r1 < end0 ? r1 : end0;
    it.t0[1] = half + r0;
    it.t1[1] = half + r1 < end1 ? half + r1 : end1;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      if (it.t1[s] < it.t0[s]) it.t1[s] = it.t0[s];
      it.slot[s] = part < 0 ? -1 : 2 * part + s;
    }
    w.items[slot_index] = it;
  };
  auto rounds_of = [&](const ChunkUnit& un) { return un.kind == kChunkLone ? (un.nt[0] + 1) / 2 : un.nt[1]; };
  // a lone tile that is not cut is merged from its two halves all the same (unless there is only one K/V tile)
  auto whole_part = [&](int u, const ChunkUnit& un) {
    if (un.kind != kChunkLone || un.nt[0] < 2) return -1;
    w.cut[P + un.b] = ChunkCut{u, -1, 2 * P + un.b, 0};
    return 2 * P + un.b;
  };

  for (int u = tid; u < F; u += kPlanThreads) {
    const ChunkUnit un = w.unit[u];
    emit((u % P) * k + u / P, u, 0, rounds_of(un), whole_part(u, un));
  }
  // the shares: piece (u, c) of unit u in CTA c's share is item u + c
  for (int u = F + warp; u < U; u += kPlanThreads / 32) {
    const ChunkUnit un = w.unit[u];
    const long long x0 = w.x[u], x1 = w.x[u + 1];
    const int c_lo = last_le(s_pos, P, x0), c_hi = last_le(s_pos, P, x1 - 1), rounds = rounds_of(un);
    for (int c = c_lo + lane; c <= c_hi; c += 32) {
      const int r0 = c == c_lo ? 0 : cut_round(s_pos[c], x0, rounds), r1 = c == c_hi ? rounds : cut_round(s_pos[c + 1], x0, rounds);
      if (r0 == 0 && r1 == rounds) emit(u + c, u, r0, r1, whole_part(u, un));
      else emit(u + c, u, r0, r1 > r0 ? r1 : r0, 2 * c + (r0 > 0 ? 0 : 1));
    }
    if (lane == 0 && c_hi > c_lo) w.cut[c_lo] = ChunkCut{u, c_lo, c_hi, 0};
  }
  if (tid < P) {
    int first = 0, count = 0;
    if (s_pos[tid + 1] > s_pos[tid] && F < U) {
      const int u0 = last_le(w.x, U, s_pos[tid]), u1 = last_le(w.x, U, s_pos[tid + 1] - 1);
      first = u0 + tid;
      count = u1 - u0 + 1;
    }
    w.cta[tid] = make_int4(tid * k, k, first, count);
  }
}

// ============================================================================================================== attention
constexpr int kThreads = 384;            // two softmax groups of four warps, producer, two MMA issuers, query loader
constexpr int kGroupThreads = 128;
constexpr int kWarpProducer = 8, kWarpMma = 9, kWarpQuery = 11;
constexpr int kSlots = 4;                // K/V ring: a pair uses slots 0, 1 for K and 2, 3 for V; a twin's stream s slots s and 2 + s
constexpr uint32_t kTmemCols = 512;      // S0 S1 | O0 O1; P (packed bf16, 64 columns) overwrites the front of its S
constexpr float kRescaleThreshold = 8.0f;   // log2 units: the accumulator is rescaled when the row maximum outgrows its reference by more
#ifndef EAGLE_CHUNK_POLY
#define EAGLE_CHUNK_POLY 3
#endif
constexpr int kPolyStride = EAGLE_CHUNK_POLY;   // one pair of exponentials in so many is a polynomial on the FMA pipe (0: none)

template <int D>
struct Smem {
  static constexpr int kSlabs = D / 64;                      // 64 bf16 = one 128-byte swizzled row
  static constexpr int kSlabBytes = kChunkTile * 128;
  static constexpr int kTileBytes = kSlabs * kSlabBytes;
  static constexpr int kQ = 0;                               // one query tile per stream
  static constexpr int kRing = 2 * kTileBytes;
  static constexpr int kBar = kRing + kSlots * kTileBytes;
  static constexpr int kNumBars = 3 * kSlots + 12;
  static constexpr int kMisc = kBar + 8 * kNumBars;          // tensor-memory base, abort flag, wait limit (8 bytes)
  static constexpr int kBytes = kMisc + 16;
};

// A slot has one "empty" barrier and two "full" ones, for its uses in pairs and in twins.  A waiter tells the phases of a
// barrier apart by parity only, so it has to see every one of them: both issuers see every load of a pair (the stream with
// fewer tiles walks past those it does not need), and the loads of a twin are seen by the one stream that owns the slot.
struct Bars {
  uint32_t base;
  __device__ __forceinline__ uint32_t full(bool shared, uint32_t i) const { return base + 8u * ((shared ? 0 : kSlots) + i); }
  __device__ __forceinline__ uint32_t empty(uint32_t i) const { return base + 8u * (2 * kSlots + i); }
  __device__ __forceinline__ uint32_t q_full(uint32_t s) const { return base + 8u * (3 * kSlots + s); }
  __device__ __forceinline__ uint32_t q_empty(uint32_t s) const { return base + 8u * (3 * kSlots + 2 + s); }
  __device__ __forceinline__ uint32_t s_full(uint32_t s) const { return base + 8u * (3 * kSlots + 4 + s); }   // scores are there
  __device__ __forceinline__ uint32_t p_full(uint32_t s) const { return base + 8u * (3 * kSlots + 6 + s); }   // probabilities are there
  __device__ __forceinline__ uint32_t o_full(uint32_t s) const { return base + 8u * (3 * kSlots + 8 + s); }   // an item's last PV has finished
  __device__ __forceinline__ uint32_t o_free(uint32_t s) const { return base + 8u * (3 * kSlots + 10 + s); }  // its accumulator has been read
};

// How often the items so far have used slots 0 and 1 (slots 2 and 3: the same), in pairs and in twins; and where round j of
// stream s finds its K tile (the V tile is two slots further): the slot and the number of that use among those of its kind.
struct Place {
  uint32_t slot, use;
};
struct Uses {
  uint32_t pair[2] = {0, 0}, twin[2] = {0, 0};
  __device__ __forceinline__ Place place(bool shared, int s, int j) const {
    if (shared) return {static_cast<uint32_t>(j & 1), ((j & 1) ? pair[1] : pair[0]) + static_cast<uint32_t>(j >> 1)};
    return {static_cast<uint32_t>(s), (s ? twin[1] : twin[0]) + static_cast<uint32_t>(j)};
  }
  // parity to wait for before the slot is filled again: uses of either kind count
  __device__ __forceinline__ uint32_t free_parity(bool shared, const Place& pl) const {
    const uint32_t before = pl.use + (shared ? (pl.slot ? twin[1] : twin[0]) : (pl.slot ? pair[1] : pair[0]));
    return (before & 1u) ^ 1u;
  }
  __device__ __forceinline__ void add(bool shared, int len0, int len1) {
    if (shared) {
      const uint32_t len = static_cast<uint32_t>(len0 > len1 ? len0 : len1);
      pair[0] += (len + 1) >> 1;
      pair[1] += len >> 1;
    } else {
      twin[0] += static_cast<uint32_t>(len0);
      twin[1] += static_cast<uint32_t>(len1);
    }
  }
};

// (a runtime index into the item's arrays would put it into local memory)
__device__ __forceinline__ int of_stream(const int32_t (&a)[2], int s) { return s ? a[1] : a[0]; }

template <int D, bool PAGED>
__global__ void __launch_bounds__(kThreads, 1)
chunk_attn_kernel(ChunkParams p, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                  const __grid_constant__ CUtensorMap map_q) {
  using S = Smem<D>;
  extern __shared__ __align__(1024) unsigned char smem[];
  const uint32_t sbase = smem_u32(smem);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (sbase & 1023u) {   // the swizzled tiles need a 1024-byte aligned base; uniform over the CTA
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
    for (int i = 0; i < kSlots; ++i) {
      mbar_init(B.full(false, i), 1);
      mbar_init(B.full(true, i), 1);
      mbar_init(B.empty(i), 2);          // both streams of a pair, or twice the one that uses it
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(B.q_full(s), 1);
      mbar_init(B.q_empty(s), 1);
      mbar_init(B.s_full(s), 1);
      mbar_init(B.p_full(s), kGroupThreads);
      mbar_init(B.o_full(s), 1);
      mbar_init(B.o_free(s), kGroupThreads);
    }
    *s_abort = 0;
    *reinterpret_cast<volatile unsigned long long*>(smem + S::kMisc + 8) = p.wait_limit_ns;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kWarpMma) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(sbase + S::kMisc), "r"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = *s_tmem;

  const int4 mine = p.work.cta[blockIdx.x];              // whole units first, then this CTA's share of the rest
  const int n_items = mine.y + mine.w;
  auto item = [&](int i) { return p.work.items[i < mine.y ? mine.x + i : mine.z + (i - mine.y)]; };

  if (warp == kWarpMma || warp == kWarpMma + 1) {
    // =========================================================================== MMA issuer of one stream
    // The tensor pipe runs one thread's MMAs in the order they were issued: S(j + 1) may overwrite P(j) without a wait, and
    // the arrival that reports S(j + 1) reports PV(j) too.
    if (lane == 0) {
      const int s = warp - kWarpMma;
      constexpr uint32_t idesc_qk = instr_desc(128, kChunkTile, false), idesc_pv = instr_desc(128, D, true);
      const uint32_t q_lo = desc_lo(sbase + S::kQ + s * S::kTileBytes, 16);
      const uint32_t k_lo = desc_lo(sbase + S::kRing, 16), v_lo = desc_lo(sbase + S::kRing, S::kSlabBytes);
      constexpr uint32_t kTileStep = S::kTileBytes >> 4, kSlabStep = S::kSlabBytes >> 4;
      const uint32_t t_s = tmem + s * 128, t_o = tmem + 256 + s * 128;
      Uses uses;
      uint32_t steps = 0, items = 0;
      bool ok = true;
      for (int i = 0; i < n_items && ok; ++i) {
        const ChunkItem it = item(i);
        const bool shared = it.kind == kChunkPair;
        const int len0 = it.t1[0] - it.t0[0], len1 = it.t1[1] - it.t0[1], len = s ? len1 : len0;
        auto release = [&](uint32_t bar) {
          commit(bar);
          if (!shared) commit(bar);          // nobody else uses the slot
        };
        auto score = [&](int j) {
          const Place pl = uses.place(shared, s, j);
          ok = mbar_wait(B.full(shared, pl.slot), pl.use & 1u, s_abort);
          if (!ok) return;
          fence_after();
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk) {
            const uint32_t step = (kk >> 2) * kSlabStep + (kk & 3) * 2;
            mma_ss(t_s, desc(q_lo + step), desc(k_lo + pl.slot * kTileStep + step), idesc_qk, kk != 0);
          }
          commit(B.s_full(s));
          release(B.empty(pl.slot));
          if (j == len - 1) commit(B.q_empty(s));
        };
        if (len > 0) {
          ok = mbar_wait(B.q_full(s), items & 1u, s_abort);
          if (!ok) break;
          score(0);
          for (int j = 0; j < len && ok; ++j, ++steps) {
            const Place pl = uses.place(shared, s, j);
            ok = mbar_wait(B.full(shared, 2 + pl.slot), pl.use & 1u, s_abort);
            if (!ok) break;
            if (j == 0 && items > 0) {
              ok = mbar_wait(B.o_free(s), (items - 1) & 1u, s_abort);
              if (!ok) break;
            }
            ok = mbar_wait(B.p_full(s), steps & 1u, s_abort);
            if (!ok) break;
            fence_after();
#pragma unroll
            for (int kk = 0; kk < kChunkTile / 16; ++kk)
              mma_ts(t_o, t_s + kk * 8, desc(v_lo + (2 + pl.slot) * kTileStep + kk * 128), idesc_pv, (j | kk) != 0);
            release(B.empty(2 + pl.slot));
            if (j == len - 1) commit(B.o_full(s));
            else score(j + 1);
          }
          ++items;
        }
        if (shared) {
          for (int j = len; j < len1 && ok; ++j) {   // the first stream of a pair may have fewer tiles: it lets the others pass
            const Place pl = uses.place(true, 0, j);
            ok = mbar_wait(B.full(true, pl.slot), pl.use & 1u, s_abort);
            if (!ok) break;
            mbar_arrive(B.empty(pl.slot));
            ok = mbar_wait(B.full(true, 2 + pl.slot), pl.use & 1u, s_abort);
            if (!ok) break;
            mbar_arrive(B.empty(2 + pl.slot));
          }
        }
        uses.add(shared, len0, len1);
      }
    }
  } else if (warp == kWarpQuery) {
    // =========================================================================== query tiles
    // Box of TPT tokens x G heads x 64 columns: rows land in (token, head) order.  A tile that reaches past the sequence's
    // last token brings rows of the next sequence (or zeros past the tensor) along; they are computed and never written.
    if (lane == 0) {
      uint32_t items[2] = {0, 0};
      bool ok = true;
      for (int i = 0; i < n_items && ok; ++i) {
        const ChunkItem it = item(i);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          if (it.t1[s] <= it.t0[s] || !ok) continue;
          ok = mbar_wait(B.q_empty(s), (items[s] & 1u) ^ 1u, s_abort);
          if (!ok) break;
          mbar_expect_tx(B.q_full(s), S::kSlabs * p.tpt * p.G * 128);
#pragma unroll
          for (int sl = 0; sl < S::kSlabs; ++sl)
            tma_load_3d(sbase + S::kQ + s * S::kTileBytes + sl * S::kSlabBytes, &map_q, sl * 64, it.g[s] * p.G, it.start + it.qt[s] * p.tpt,
                        B.q_full(s));
          ++items[s];
        }
      }
    }
  } else if (warp == kWarpProducer) {
    // =========================================================================== K/V tiles
    // Paged cache: the whole warp walks the list in step and each lane fetches one box (a page, or a page's 64-column half).
    if (lane == 0 || PAGED) {
      Uses uses;
      bool ok = true;
      for (int i = 0; i < n_items && ok; ++i) {
        const ChunkItem it = item(i);
        const bool shared = it.kind == kChunkPair;
        const int len0 = it.t1[0] - it.t0[0], len1 = it.t1[1] - it.t0[1], len = len0 > len1 ? len0 : len1;
        const int32_t* pages = PAGED ? p.block_table + static_cast<size_t>(it.b) * p.max_pages : nullptr;
        const int last_page = PAGED ? (it.L + it.n - 1) >> p.page_shift : 0;
        auto load = [&](uint32_t slot, uint32_t parity, const CUtensorMap* map, int g, int tile) {
          const uint32_t dst = sbase + S::kRing + slot * S::kTileBytes;
          if constexpr (PAGED) {
            // The box past the sequence's last page fetches that page again (its rows are masked), so that a tile's byte
            // count never changes; an entry outside the pool reads page 0 (the merge kernel reports and zeroes the sequence).
            const int rows = p.page_size < kChunkTile ? p.page_size : kChunkTile;
            const int sl = lane % S::kSlabs, r0 = (lane / S::kSlabs) * rows;
            const int key = tile * kChunkTile + r0;
            int page = 0;
            if (r0 < kChunkTile) {
              const int pi = key >> p.page_shift;
              page = __ldg(pages + (pi < last_page ? pi : last_page));
              if (page < 0 || page >= p.num_pages) page = 0;
            }
            ok = mbar_wait_warp(B.empty(slot), parity, s_abort);
            if (!ok) return;
            if (lane == 0) mbar_expect_tx(B.full(shared, slot), S::kTileBytes);
            __syncwarp();
            if (r0 < kChunkTile)
              tma_load_3d(dst + sl * S::kSlabBytes + r0 * 128, map, sl * 64, key & (p.page_size - 1), page * p.Hkv + g, B.full(shared, slot));
          } else {
            ok = mbar_wait(B.empty(slot), parity, s_abort);
            if (!ok) return;
            mbar_expect_tx(B.full(shared, slot), S::kTileBytes);
#pragma unroll
            for (int sl = 0; sl < S::kSlabs; ++sl)
              tma_load_3d(dst + sl * S::kSlabBytes, map, sl * 64, tile * kChunkTile, it.b * p.Hkv + g, B.full(shared, slot));
          }
        };
        for (int j = 0; j < len && ok; ++j) {
          if (shared) {
            const Place pl = uses.place(true, 0, j);
            const int tile = it.t0[1] + j;               // (the second stream of a pair is never the shorter one)
            const uint32_t parity = uses.free_parity(true, pl);
            load(pl.slot, parity, &map_k, it.g[0], tile);
            if (ok) load(2 + pl.slot, parity, &map_v, it.g[0], tile);
          } else {
#pragma unroll
            for (int kv = 0; kv < 2; ++kv)
#pragma unroll
              for (int s = 0; s < 2; ++s) {
                if (!ok || j >= (s ? len1 : len0)) continue;
                const Place pl = uses.place(false, s, j);
                load(2 * kv + pl.slot, uses.free_parity(false, pl), kv ? &map_v : &map_k, it.g[s], it.t0[s] + j);
              }
          }
        }
        uses.add(shared, len0, len1);
      }
    }
  } else {
    // =========================================================================== softmax and output of one stream
    // Thread r owns query row r (tensor-memory lane r), all 128 score columns.  fp32 throughout, in the log2 domain; the
    // probabilities are rounded to bf16 for the tensor cores (relative 2^-8 each, half of the inputs' own spacing), the sum
    // that divides them is kept from the unrounded ones.
    const int s = warp >> 2;
    const int r = tid & (kGroupThreads - 1);
    const uint32_t lane_addr = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t s_addr = tmem + lane_addr + s * 128, o_addr = tmem + lane_addr + 256 + s * 128;
    const int tok_r = r / p.G, head_r = r - tok_r * p.G;   // token and head within the tile
    const bool row_used = tok_r < p.tpt;
    const float scale_log2 = p.scale_log2;
    Uses uses;
    uint32_t steps = 0, items = 0;
    bool ok = true;
    for (int i = 0; i < n_items && ok; ++i) {
      const ChunkItem it = item(i);
      const bool shared = it.kind == kChunkPair;
      const int len0 = it.t1[0] - it.t0[0], len1 = it.t1[1] - it.t0[1], len = s ? len1 : len0;
      if (len > 0) {
        const int tile0 = of_stream(it.t0, s), kv_end = it.L + it.n;
        const int first = of_stream(it.qt, s) * p.tpt, token = first + tok_r;                  // place in the chunk
        const bool row_valid = row_used && token < it.n;
        const int limit = it.L + (token < it.n ? token : it.n - 1);                 // the last key this row sees
        float m_ref = -INFINITY, l_sum = 0.f;
        for (int j = 0; j < len; ++j, ++steps) {
          const int key0 = (tile0 + j) * kChunkTile;
          ok = mbar_wait_warp(B.s_full(s), steps & 1u, s_abort);
          if (!ok) break;
          fence_after();
          if (key0 + kChunkTile - 1 > it.L + first) {
            // a tile that some row of this query tile does not see whole: -inf over the invisible scores, in place
            const int lim = limit - key0;                  // last visible column of this row
            const int lim_lo = __reduce_min_sync(0xffffffffu, lim);
#pragma unroll 1
            for (int c = 0; c < 4; ++c) {
              if (lim_lo >= c * 32 + 31) continue;         // uniform: every row of the warp sees the whole chunk
              const int v = lim - c * 32;
              const uint32_t see = v >= 31 ? 0xffffffffu : (v < 0 ? 0u : (2u << v) - 1u);
              uint32_t t[32];
              ld32(s_addr + c * 32, t);
              wait_ld();
#pragma unroll
              for (int e = 0; e < 32; ++e) t[e] = (see >> e) & 1u ? t[e] : 0xff800000u;
              st32(s_addr + c * 32, t);
            }
            wait_st();
          }
          if (key0 + kChunkTile > kv_end) {
            // slots past the sequence may hold anything: their V rows are zeroed so that 0 * garbage cannot reach O.  Both
            // streams of a pair do it, each before it hands over its own probabilities.
            const Place pl = uses.place(shared, s, j);
            ok = mbar_wait_warp(B.full(shared, 2 + pl.slot), pl.use & 1u, s_abort);
            if (!ok) break;
            if (key0 + r >= kv_end) {
#pragma unroll
              for (int c = 0; c < 8 * S::kSlabs; ++c)
                *reinterpret_cast<uint4*>(smem + S::kRing + (2 + pl.slot) * S::kTileBytes + (c >> 3) * S::kSlabBytes + r * 128 + (c & 7) * 16) =
                    make_uint4(0u, 0u, 0u, 0u);
            }
            fence_proxy_async();
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
              mx[0] = max3(mx[0], __uint_as_float(rc[e]), __uint_as_float(rc[e + 1]));
              mx[1] = max3(mx[1], __uint_as_float(rd[e]), __uint_as_float(rd[e + 1]));
              mx[2] = max3(mx[2], __uint_as_float(ra[e]), __uint_as_float(ra[e + 1]));
              mx[3] = max3(mx[3], __uint_as_float(rb[e]), __uint_as_float(rb[e + 1]));
            }
          }
          const float tmax = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * scale_log2;   // scale > 0
          const bool grow = tmax > m_ref + kRescaleThreshold || (m_ref == -INFINITY && tmax > -INFINITY);
          float factor = 1.f;
          if (grow) {
            factor = fast_exp2(m_ref - tmax);            // 0 when there was no reference yet
            m_ref = tmax;
            l_sum *= factor;
          }
          if (j > 0 && __any_sync(0xffffffffu, grow)) {
            // the PV of the step before has finished (it was issued before the scores that have just arrived)
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
              if (kPolyStride > 0 && e % (kPolyStride > 0 ? kPolyStride : 1) == (kPolyStride > 0 ? kPolyStride : 1) - 1) {
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
          wait_st();
          fence_before();
          mbar_arrive(B.p_full(s));
        }
        if (!ok) break;
        // ---- output: a bf16 row, or the unnormalised fp32 partial of a cut tile, laid out [4 columns][row] so that the
        // lanes of a store write consecutive 16-byte pieces
        ok = mbar_wait_warp(B.o_full(s), items & 1u, s_abort);
        if (!ok) break;
        fence_after();
        const float inv = l_sum > 0.f ? 1.f / l_sum : (l_sum == 0.f ? 0.f : l_sum);    // a NaN sum stays one
        const int slot = of_stream(it.slot, s), g = of_stream(it.g, s);
        uint32_t oa[32], ob[32];
        auto store_chunk = [&](uint32_t (&o)[32], int c) {
          if (!row_valid) return;
          if (slot < 0) {
            __nv_bfloat16* out_row = p.out + (static_cast<size_t>(it.start + token) * p.Hq + g * p.G + head_r) * D;
#pragma unroll
            for (int e = 0; e < 32; e += 16) {
              uint32_t v[8];
#pragma unroll
              for (int k = 0; k < 8; ++k) v[k] = pack_bf16(__uint_as_float(o[e + 2 * k]) * inv, __uint_as_float(o[e + 2 * k + 1]) * inv);
              st_global_v8(out_row + c * 32 + e, v);
            }
          } else {
            float* part = p.work.part_o + (static_cast<size_t>(slot) * (D / 4) + c * 8) * (128 * 4) + r * 4;
#pragma unroll
            for (int e = 0; e < 32; e += 4)
              *reinterpret_cast<uint4*>(part + (e / 4) * (128 * 4)) = make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]);
          }
        };
        ld32(o_addr, oa);
#pragma unroll
        for (int c = 0; c < D / 32; c += 2) {
          wait_ld();
          ld32(o_addr + (c + 1) * 32, ob);
          store_chunk(oa, c);
          wait_ld();
          if (c + 2 < D / 32) ld32(o_addr + (c + 2) * 32, oa);
          store_chunk(ob, c + 1);
        }
        if (row_valid && slot >= 0) p.work.part_ml[static_cast<size_t>(slot) * 128 + r] = make_float2(m_ref, l_sum);
        fence_before();
        mbar_arrive(B.o_free(s));
        ++items;
      }
      uses.add(shared, len0, len1);
    }
  }

  // ---- teardown: everyone arrives here, normally or after an abort
  fence_before();
  __syncthreads();
  if (tid == 0 && *s_abort) report_status(p.status, EAGLE_ERR_TIMEOUT);
  if (warp == kWarpMma) {
    __syncwarp();
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
  }
}

// ================================================================================================================== merge
// Cut query tiles: m* = max m_i, l* = sum l_i 2^(m_i - m*), out = sum o_i 2^(m_i - m*) / l*.  A block takes 8 rows of one
// stream of one record (a warp: 8 rows x 4 groups of 4 columns, so that its loads are runs of 128 bytes).  The blocks behind
// them look at one sequence each: rows of a sequence that does not fit its cache, or whose block table names a page outside
// the pool, become zeros.
constexpr int kMergeThreads = 256;

template <int D>
__global__ void __launch_bounds__(kMergeThreads) chunk_merge_kernel(ChunkParams p, int records, int row_blocks) {
  const ChunkWork& w = p.work;
  const int tid = threadIdx.x;
  if (static_cast<int>(blockIdx.x) >= records * 2 * row_blocks) {
    const int b = blockIdx.x - records * 2 * row_blocks;
    const ChunkSeq q = w.seq[b];
    const int s = p.token_start[b], e = p.token_start[b + 1];
    if (s < 0 || e <= s || e > p.N) return;
    bool bad = q.n == 0;                                 // the planner refused it (and reported it)
    if (p.block_table && q.n > 0) {
      int wrong = 0;
      const int pages = ((q.L + q.n - 1) >> p.page_shift) + 1;
      for (int i = tid; i < pages; i += kMergeThreads) {
        const int pg = p.block_table[static_cast<size_t>(b) * p.max_pages + i];
        if (pg < 0 || pg >= p.num_pages) wrong = 1;
      }
      wrong = __syncthreads_or(wrong);
      if (wrong && tid == 0) report_status(p.status, EAGLE_ERR_PAGE);
      bad = bad || wrong;
    }
    if (!bad) return;
    uint4* out = reinterpret_cast<uint4*>(p.out + static_cast<size_t>(s) * p.Hq * D);
    const size_t vecs = static_cast<size_t>(e - s) * p.Hq * (D / 8);
    for (size_t i = tid; i < vecs; i += kMergeThreads) out[i] = make_uint4(0u, 0u, 0u, 0u);
    return;
  }
  const int rec = blockIdx.x / (2 * row_blocks), rest = blockIdx.x - rec * 2 * row_blocks, s = rest / row_blocks, rb = rest - s * row_blocks;
  const ChunkCut cut = w.cut[rec];
  if (cut.unit < 0) return;
  const ChunkUnit un = w.unit[cut.unit];
  const bool lone = un.kind == kChunkLone;
  if (lone && s) return;                                 // its two streams are halves of one tile
  const ChunkSeq q = w.seq[un.b];
  const int qt = un.kind == kChunkPair ? un.qt + s : un.qt, g = un.kind == kChunkTwin ? un.g + s : un.g;
  const int row = rb * 8 + ((tid >> 2) & 7), cols = (tid >> 5) * 4 + (tid & 3);      // row of the tile, group of 4 columns
  const int tok = row / p.G, head = row - tok * p.G, token = qt * p.tpt + tok;
  if (tok >= p.tpt || token >= q.n || cols >= D / 4) return;
  const int pieces = cut.c_lo < 0 ? 1 : cut.c_hi - cut.c_lo + 1, streams = lone ? 2 : 1;
  float m = -INFINITY, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int i = 0; i < pieces; ++i) {
    for (int t = 0; t < streams; ++t) {
      const int st = lone ? t : s;
      int slot;
      if (cut.c_lo < 0) {
        slot = 2 * cut.c_hi + st;                        // both halves of a lone tile that was not cut
      } else {
        const ChunkItem* it = w.items + cut.unit + cut.c_lo + i;
        if (it->t1[st] <= it->t0[st]) continue;
        slot = it->slot[st];
        if (slot < 0) return;                            // its cuts snapped to the edges: the output is there already
        if (lone && it->slot[st] >= 4 * p.num_ctas) return;   // the same, merged from the halves by the record of its sequence
      }
      const float2 ml = w.part_ml[static_cast<size_t>(slot) * 128 + row];
      const float4 v = *reinterpret_cast<const float4*>(w.part_o + (static_cast<size_t>(slot) * (D / 4) + cols) * (128 * 4) + row * 4);
      if (ml.x == -INFINITY && ml.y == 0.f) continue;    // nothing visible in this piece
      const float top = fmaxf(m, ml.x);
      const float a = m == -INFINITY ? 0.f : exp2f(m - top), c = exp2f(ml.x - top);
      m = top;
      l = l * a + ml.y * c;
      o = make_float4(o.x * a + v.x * c, o.y * a + v.y * c, o.z * a + v.z * c, o.w * a + v.w * c);
    }
  }
  const float inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);
  uint2 out;
  out.x = pack_bf16(o.x * inv, o.y * inv);
  out.y = pack_bf16(o.z * inv, o.w * inv);
  *reinterpret_cast<uint2*>(p.out + (static_cast<size_t>(q.start + token) * p.Hq + g * p.G + head) * D + cols * 4) = out;
}

template <int D>
cudaError_t launch_all(const ChunkParams& p, cudaStream_t stream) {
  CUtensorMap mk, mv, mq;
  const bool paged = p.block_table != nullptr;
  if (paged) {
    const int rows = p.page_size < kChunkTile ? p.page_size : kChunkTile;
    const long long ph = static_cast<long long>(p.num_pages) * p.Hkv;
    if (!map_bf16_3d(&mk, p.k, D, p.page_size, ph, rows, 1) || !map_bf16_3d(&mv, p.v, D, p.page_size, ph, rows, 1)) return cudaErrorInvalidValue;
  } else {
    const long long bh = static_cast<long long>(p.B) * p.Hkv, cap = p.capacity > 0 ? p.capacity : 1;
    if (!map_bf16_3d(&mk, p.k, D, cap, bh, kChunkTile, 1) || !map_bf16_3d(&mv, p.v, D, cap, bh, kChunkTile, 1)) return cudaErrorInvalidValue;
  }
  if (!map_bf16_3d(&mq, p.q, D, p.Hq, p.N, p.G, p.tpt)) return cudaErrorInvalidValue;
  chunk_plan_kernel<<<1, kPlanThreads, 0, stream>>>(p);
  count_launch();
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  if (paged) chunk_attn_kernel<D, true><<<p.num_ctas, kThreads, Smem<D>::kBytes, stream>>>(p, mk, mv, mq);
  else chunk_attn_kernel<D, false><<<p.num_ctas, kThreads, Smem<D>::kBytes, stream>>>(p, mk, mv, mq);
  count_launch();
  e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  const int records = p.num_ctas + ((p.Hkv & 1) ? p.B : 0);
  const int rows = p.max_rows < 128 ? p.max_rows : 128, row_blocks = (rows + 7) / 8;
  chunk_merge_kernel<D><<<records * 2 * row_blocks + p.B, kMergeThreads, 0, stream>>>(p, records, row_blocks);
  count_launch();
  return cudaGetLastError();
}

}  // namespace

cudaError_t chunk_prepare(int head_dim) {
  cudaError_t e;
  if (head_dim == 128) {
    e = cudaFuncSetAttribute(chunk_attn_kernel<128, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, Smem<128>::kBytes);
    return e != cudaSuccess ? e : cudaFuncSetAttribute(chunk_attn_kernel<128, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, Smem<128>::kBytes);
  }
  e = cudaFuncSetAttribute(chunk_attn_kernel<64, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, Smem<64>::kBytes);
  return e != cudaSuccess ? e : cudaFuncSetAttribute(chunk_attn_kernel<64, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, Smem<64>::kBytes);
}

cudaError_t launch_chunk(const ChunkParams& p, cudaStream_t stream) { return p.D == 128 ? launch_all<128>(p, stream) : launch_all<64>(p, stream); }

}  // namespace eagle
