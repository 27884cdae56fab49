// Attention of single tokens with a window, over bf16 or block-scaled codes: 16 query rows of one (sequence, KV head) against the slots that
// they see, streamed through a ring in shared memory.
//
// Bound by the reading of the cache, like the kernel without a window (chunk_rows.cu): one warp issues copies of 32 keys with their
// values as far ahead as shared memory allows, the other warps take the tiles in turn, each with its own maximum, sum and
// accumulator.  K/V tiles between the sinks and the window are not in the plan.
//
// Codes have half the bytes, so twice the tiles pass per time: eight warps take them instead of four.  They are widened to fp16 in
// registers, on their way from shared memory to the matrix instructions.  The order of the contraction is free, so a lane reads 16 codes of a
// key at once (the keys of a group of eight permuted so that the eight lanes of a 16-byte access meet no bank twice) and queries are
// arranged to match; values come through the transposing matrix load as pairs of codes, neighbours in the head, whose bytes are
// sorted into even and odd columns.  With the blocks' scales, z = (q.c) ks scale, and the maximum is taken over z + log2 vs: then
// 2^(z + log2 vs - m) is the weight of the code itself, never too large for fp16, and the row sum is divided by vs again, once per 16 keys.
#include "window.cuh"

namespace eagle {

namespace {

using namespace tc;

constexpr int kRowKeys = 32;             // keys of a tile: a quarter of a K/V tile of the plan

template <int D, bool CODES>
struct RowSmem {
  static constexpr int kWarps = CODES ? 8 : 4, kThreads = 32 * (kWarps + 1);
  static constexpr int kSlabs = CODES ? 1 : D / 64;          // 128-byte swizzled rows: 64 bf16, or 128 codes
  static constexpr int kSlab = kRowKeys * 128, kTile = kSlabs * kSlab, kStage = 2 * kTile;    // K, then V
  static constexpr int kStages = CODES ? 16 : 12 * 128 / D;
  // A warp takes all uses of a slot: copies land in any order, and a warp that came to a slot's next use before another had seen
  // the last one would find its parity there already.
  static_assert(kStages % kWarps == 0, "a slot belongs to one warp");
  static constexpr int kAccRow = CODES ? D + 16 : D + 8;     // (rows 16 or 8 floats apart in the banks: stores of neighbouring rows do not meet)
  static constexpr int kAcc = kStages * kStage;              // float [warps][16][kAccRow]
  static constexpr int kMl = kAcc + kWarps * kFewRows * kAccRow * 4;         // float2 [warps][16]: maximum and sum
  static constexpr int kScale = kMl + kWarps * kFewRows * 8; // float [kStages][4]: ks of 16 keys each, vs of 16 keys each
  static constexpr int kBar = kScale + (CODES ? kStages * 16 : 0);           // full [kStages], empty [kStages]
  static constexpr int kMisc = kBar + 16 * kStages;          // abort flag (at + 4), wait limit (8 bytes)
  static constexpr int kBytes = kMisc + 16;
  static_assert(kBytes <= 227 * 1024, "shared memory of an SM");
};

__device__ __forceinline__ void load_matrices(uint32_t* r, uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void load_matrices_t(uint32_t* r, uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint4 load_shared(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}
// c[16 x 8] += a[16 x 16] b[16 x 8], operands bf16 or fp16
template <bool HALF>
__device__ __forceinline__ void mma_16x8x16(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  if constexpr (HALF)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float quad_max(float x) {
  x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
  return fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
}
__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
  x = max(x, __shfl_xor_sync(0xffffffffu, x, 1));
  return max(x, __shfl_xor_sync(0xffffffffu, x, 2));
}
__device__ __forceinline__ float quad_sum(float x) {
  x += __shfl_xor_sync(0xffffffffu, x, 1);
  return x + __shfl_xor_sync(0xffffffffu, x, 2);
}
// One 4-byte copy that reports to no one by itself, and the arrival of all of this lane's copies at a barrier.
__device__ __forceinline__ void copy_word(uint32_t dst, const float* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void arrive_with_copies(uint32_t bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}

template <int D, bool PAGED, bool CODES, bool STALL>         // (STALL: of the test hook, as in chunk.cu)
__global__ void __launch_bounds__(RowSmem<D, CODES>::kThreads, 1)
window_rows_kernel(ChunkParams p, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v) {
  using S = RowSmem<D, CODES>;
  extern __shared__ __align__(1024) unsigned char smem[];
  const uint32_t sbase = smem_u32(smem);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (sbase & 1023u) {   // the swizzled tiles need a 1024-byte aligned base; uniform over the launch
    if (tid == 0) report_status(p.status, EAGLE_ERR_DEVICE);
    return;
  }
  volatile int* s_abort = reinterpret_cast<volatile int*>(smem + S::kMisc + 4);
  auto full = [&](uint32_t i) { return sbase + S::kBar + 8u * i; };
  auto empty = [&](uint32_t i) { return sbase + S::kBar + 8u * (S::kStages + i); };
  if (tid == 0) {
    prefetch_map(&map_k);
    prefetch_map(&map_v);
    for (int i = 0; i < S::kStages; ++i) { mbar_init(full(i), CODES ? 5 : 1); mbar_init(empty(i), 1); }      // (codes: four lanes with scales)
    *s_abort = 0;
    *reinterpret_cast<volatile unsigned long long*>(smem + S::kMisc + 8) = p.wait_limit_ns;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  launch_dependents();
  wait_for_prerequisites();                // the plan is there
  const int4 mine = p.work.cta[blockIdx.x];              // whole units first, then this CTA's share of the rest
  const int n_items = mine.y + mine.w;
  // first: token of the chunk in row 0; `steps` tiles from place0 on, counted in keys of the plan (without the gap)
  struct Item {
    int b, g, first, start, n, L, place0, steps, slot;
    ChunkSpan span;
    __device__ int key(int step) const { return place0 + step * kRowKeys + (place0 + step * kRowKeys >= span.before * kChunkTile ? span.skip * kChunkTile : 0); }
  };
  auto item = [&](int i) {
    const int4* at = reinterpret_cast<const int4*>(p.work.items + (i < mine.y ? mine.x + i : mine.z + (i - mine.y)));
    const int4 a = at[0], b = at[1];
    Item it;
    it.b = a.x;
    it.g = a.y;
    it.first = a.z * p.tpt;
    it.start = a.w;
    it.n = b.x;
    it.L = b.y;
    it.span = chunk_span(p, it.L, it.first);
    it.place0 = b.z * kChunkTile;
    const int keys = it.L + min(it.first + p.tpt, it.n) - it.span.skip * kChunkTile;      // where what the last row sees ends
    const long long end = static_cast<long long>(b.w) * kChunkTile < keys ? static_cast<long long>(b.w) * kChunkTile : keys;
    it.steps = b.w > b.z ? static_cast<int>((end - it.place0 + kRowKeys - 1) / kRowKeys) : 0;
    it.slot = at[2].x;
    return it;
  };

  if (warp == S::kWarps) {
    // =========================================================================== copies
    // A lane per box (a page's rows x 64 columns or 128 codes, of K or of V); the page of a lane's next box is looked up while the box
    // before it is on its way.  A box past the sequence's last page fetches that page again, and one of a page that holds nothing the unit
    // sees fetches the first that does (their rows are masked), so that a tile's byte count never changes; an entry outside the pool reads
    // page 0, and marks its sequence when the item ends (the merge kernel reports it and zeroes the rows).  Of codes, four lanes fetch the
    // scales of each half of the tile, which the barrier counts as well.
    const int box_rows = PAGED ? min(p.page_size, kRowKeys) : kRowKeys, per = S::kSlabs * (kRowKeys / box_rows);
    const bool is_v = lane >= per, active = lane < 2 * per;
    const int r0 = ((lane - (is_v ? per : 0)) / S::kSlabs) * box_rows, sl = lane % S::kSlabs;      // (per is a multiple of kSlabs)
    const uint32_t dst = sbase + (is_v ? S::kTile : 0) + sl * S::kSlab + r0 * 128;
    const float* scales = lane < 2 ? p.k_scale : p.v_scale;
    Item it = {};
    int i = -1, step = 0, y = 0, z = 0, ys = 0, zs = 0;
    bool more = true, wrong = false;                       // wrong: some entry of the item was outside the pool
    auto page_of = [&](int key) {
      const int last = (it.L + it.n - 1) >> p.page_shift, pi = key >> p.page_shift;
      return __ldg(p.block_table + static_cast<size_t>(it.b) * p.max_pages + it.span.page(pi < last ? pi : last, p.page_shift));
    };
    auto advance = [&]() {
      if (++step >= it.steps) {
        if (PAGED && wrong) p.work.bad_page[it.b] = 1;
        wrong = false;
        for (++i; i < n_items; ++i) {
          it = item(i);
          if (it.steps > 0) break;
        }
        if (i >= n_items) {
          more = false;
          return;
        }
        step = 0;
      }
      const int key0 = it.key(step);
      y = key0 + r0;
      z = it.b;
      if (PAGED && active) {
        z = page_of(y);
        y &= p.page_size - 1;
      }
      if (CODES && lane < 4) {
        ys = min(key0 + (lane & 1) * 16, static_cast<int>(p.capacity) - 1);
        zs = it.b;
        if (PAGED) {
          zs = page_of(ys);
          ys &= p.page_size - 1;
        }
      }
    };
    advance();
    Ring<S::kStages> ring;
    [[maybe_unused]] int tiles = 0;                        // issued
    while (more) {
      if constexpr (STALL) {
        if (tiles++ >= p.stall_after_tiles) break;
      }
      if (!mbar_wait_warp(empty(ring.slot), ring.par ^ 1u, s_abort)) break;
      if (lane == 0) mbar_expect_tx(full(ring.slot), S::kStage);
      __syncwarp();
      const bool out_of_pool = PAGED && active && static_cast<uint32_t>(z) >= static_cast<uint32_t>(p.num_pages);
      const int page = out_of_pool ? 0 : z;
      wrong |= out_of_pool;
      if (active) tma_load_3d(dst + ring.slot * S::kStage, is_v ? &map_v : &map_k, sl * 64, y, page * p.Hkv + it.g, full(ring.slot));
      if (CODES && lane < 4) {
        const int ps = PAGED && static_cast<uint32_t>(zs) >= static_cast<uint32_t>(p.num_pages) ? 0 : zs;
        copy_word(sbase + S::kScale + ring.slot * 16 + lane * 4, scales + (static_cast<long long>(ps) * p.Hkv + it.g) * p.head_blocks + (ys >> p.block_shift));
        arrive_with_copies(full(ring.slot));
      }
      ring.step();
      advance();
    }
  } else {
    // =========================================================================== scores, softmax, output
    // Scores: a lane holds two columns of rows l / 4 and l / 4 + 8 of every 8 keys: 2 (l % 4), + 1 of bf16, l % 4 and l % 4 + 4 of codes
    // (whose keys are permuted).  fp32 throughout, in the log2 domain; the probabilities are rounded for the second product, to bf16
    // (relative 2^-8 each) or, over codes and times vs, to fp16 (2^-11); the sum that divides them is kept from the unrounded ones.
    const int row = lane >> 2, quad = lane & 3, G = p.G;
    constexpr int kPair = CODES ? 4 : 1;                   // from a lane's first column to its second
    const int col = CODES ? quad : 2 * quad;
    const int tok0 = row / G, tok1 = (row + 8) / G;        // tokens of this lane's rows within the tile
    const int head0 = row - tok0 * G, head1 = row + 8 - tok1 * G;
    const float scale_log2 = p.scale_log2;
    float* acc = reinterpret_cast<float*>(smem + S::kAcc);
    float2* ml = reinterpret_cast<float2*>(smem + S::kMl);
    // rows of the matrix loads of this lane: K by (key, 16-byte piece), V by (key, 16-byte piece) too, transposed on the way
    const uint32_t swz = lane & 7;
    const uint32_t k_row = (lane & 7) * 128, k_piece = lane >> 3, v_row = (lane & 15) * 128, v_piece = lane >> 4;      // bf16
    const uint32_t spread = ((row & 1) << 2) | (row >> 1);                                    // codes: key of a group that a lane reads
    const uint32_t v_key = ((lane & 1) << 2) | ((lane & 7) >> 1);                             // and that it addresses for the transposing load
    const uint32_t vc_row = (((lane >> 3) & 1) * 8 + v_key) * 128, vc_piece = lane >> 4;
    uint32_t before = 0;                                   // tiles of the items before
    bool ok = true;
    for (int i = 0; i < n_items; ++i) {
      const Item it = item(i);
      if (it.steps <= 0) continue;                         // (uniform over the CTA)
      const bool valid0 = tok0 < p.tpt && it.first + tok0 < it.n, valid1 = tok1 < p.tpt && it.first + tok1 < it.n;
      uint32_t qa[D / 16][4];
      float s0 = scale_log2, s1 = scale_log2;              // times what the rows were multiplied by
      {
        const __nv_bfloat16* q0 = p.q + (static_cast<size_t>(it.start + it.first + tok0) * p.Hq + it.g * G + head0) * D;
        const __nv_bfloat16* q1 = p.q + (static_cast<size_t>(it.start + it.first + tok1) * p.Hq + it.g * G + head1) * D;
        if constexpr (CODES) {
          // four neighbours per 16 of the contraction: those of the codes of a word
          uint32_t top0 = 0, top1 = 0;
#pragma unroll
          for (int k = 0; k < D / 16; ++k) {
            const int d = (k >> 2) * 64 + quad * 16 + (k & 3) * 4;
            const uint2 a = valid0 ? __ldg(reinterpret_cast<const uint2*>(q0 + d)) : make_uint2(0u, 0u);
            const uint2 b = valid1 ? __ldg(reinterpret_cast<const uint2*>(q1 + d)) : make_uint2(0u, 0u);
            qa[k][0] = a.x;
            qa[k][1] = b.x;
            qa[k][2] = a.y;
            qa[k][3] = b.y;
            top0 = max(top0, max(magnitude_bits(a.x), magnitude_bits(a.y)));
            top1 = max(top1, max(magnitude_bits(b.x), magnitude_bits(b.y)));
          }
          const RowFactor f0 = row_factor(quad_max(top0)), f1 = row_factor(quad_max(top1));
#pragma unroll
          for (int k = 0; k < D / 16; ++k) {
            qa[k][0] = half_of_bf16(qa[k][0], f0.down);
            qa[k][1] = half_of_bf16(qa[k][1], f1.down);
            qa[k][2] = half_of_bf16(qa[k][2], f0.down);
            qa[k][3] = half_of_bf16(qa[k][3], f1.down);
          }
          s0 *= f0.up;
          s1 *= f1.up;
        } else {
#pragma unroll
          for (int k = 0; k < D / 16; ++k) {
            const uint32_t* w0 = reinterpret_cast<const uint32_t*>(q0 + col + k * 16);
            const uint32_t* w1 = reinterpret_cast<const uint32_t*>(q1 + col + k * 16);
            qa[k][0] = valid0 ? __ldg(w0) : 0u;
            qa[k][1] = valid1 ? __ldg(w1) : 0u;
            qa[k][2] = valid0 ? __ldg(w0 + 4) : 0u;
            qa[k][3] = valid1 ? __ldg(w1 + 4) : 0u;
          }
        }
      }
      // accumulators: of 8 columns of the head each; over codes the even ones of 16, then the odd ones
      float o[D / 8][4];
#pragma unroll
      for (int d = 0; d < D / 8; ++d) o[d][0] = o[d][1] = o[d][2] = o[d][3] = 0.f;
      float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;
      const int limit0 = it.L + it.first + tok0, limit1 = it.L + it.first + tok1;       // the last key a row sees
      const int low0 = p.window > 0 ? limit0 - p.window + 1 : 0, low1 = p.window > 0 ? limit1 - p.window + 1 : 0;      // and the first behind the sinks
      for (int s = static_cast<int>((warp - before) & (S::kWarps - 1)); s < it.steps && ok; s += S::kWarps) {
        const uint32_t gs = before + s, slot = gs % S::kStages, par = (gs / S::kStages) & 1u;
        const uint32_t k_at = sbase + slot * S::kStage, v_at = k_at + S::kTile;
        const int key0 = it.key(s);
        ok = mbar_wait_warp(full(slot), par, s_abort);
        if (!ok) break;
        float sc[kRowKeys / 8][4];
#pragma unroll
        for (int j = 0; j < kRowKeys / 8; ++j) {
          sc[j][0] = sc[j][1] = sc[j][2] = sc[j][3] = 0.f;
          if constexpr (CODES) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint4 c = load_shared(k_at + (j * 8 + spread) * 128 + (((h * 4 + quad) ^ spread) << 4));
              const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                uint32_t b0, b1;
                half_of_codes(w[k], b0, b1);
                mma_16x8x16<true>(sc[j], qa[h * 4 + k], b0, b1);
              }
            }
          } else {
#pragma unroll
            for (int k = 0; k < D / 32; ++k) {             // 32 columns of 8 keys: two steps of 16
              uint32_t kb[4];
              load_matrices(kb, k_at + (k >> 1) * S::kSlab + j * 1024 + k_row + ((((k & 1) * 4 + k_piece) ^ swz) << 4));
              mma_16x8x16<false>(sc[j], qa[2 * k], kb[0], kb[1]);
              mma_16x8x16<false>(sc[j], qa[2 * k + 1], kb[2], kb[3]);
            }
          }
        }
        // scales of the tile's halves; those of a half that the unit sees nothing of may be anything
        float ks[2] = {1.f, 1.f}, vs[2] = {1.f, 1.f}, lv[2] = {0.f, 0.f}, iv[2] = {1.f, 1.f};
        const int in_use = it.L + it.n;                    // slots of the sequence
        if constexpr (CODES) {
          const uint4 raw = load_shared(sbase + S::kScale + slot * 16);
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            const int a = key0 + t * 16;
            if (a < in_use && it.span.sees_some(a, 16)) {
              ks[t] = __uint_as_float(t ? raw.y : raw.x);
              vs[t] = __uint_as_float(t ? raw.w : raw.z);
              lv[t] = fast_log2(vs[t]);
              iv[t] = fast_rcp(vs[t]);
            }
          }
        }
        const bool whole = key0 + kRowKeys - 1 <= it.L + it.first && (key0 >= low1 || key0 + kRowKeys <= p.sinks || p.window <= 0);
        if (!whole) {                                      // a tile that some row does not see whole
          auto mask = [&](float& x, int key, int limit, int low) {
            if (key > limit || (key < low && key >= p.sinks)) x = -INFINITY;
          };
#pragma unroll
          for (int j = 0; j < kRowKeys / 8; ++j) {
            const int key = key0 + j * 8 + col;
            mask(sc[j][0], key, limit0, low0);
            mask(sc[j][1], key + kPair, limit0, low0);
            mask(sc[j][2], key, limit1, low1);
            mask(sc[j][3], key + kPair, limit1, low1);
          }
        }
        // row maxima, of 16 keys at a time, in the log2 domain
        float t0 = -INFINITY, t1 = -INFINITY;
        float bad0 = 0.f, bad1 = 0.f;                      // NaN where a score is NaN or +inf
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const float x0 = max3_nan(max3_nan(sc[2 * t][0], sc[2 * t][1], sc[2 * t + 1][0]), sc[2 * t + 1][1], -INFINITY);
          const float x1 = max3_nan(max3_nan(sc[2 * t][2], sc[2 * t][3], sc[2 * t + 1][2]), sc[2 * t + 1][3], -INFINITY);
          const float z0 = fmaf(x0, ks[t] * s0, lv[t]), z1 = fmaf(x1, ks[t] * s1, lv[t]);
          if (!(z0 < INFINITY)) bad0 = __uint_as_float(0x7fffffffu);
          if (!(z1 < INFINITY)) bad1 = __uint_as_float(0x7fffffffu);
          t0 = fmaxf(t0, z0);
          t1 = fmaxf(t1, z1);
        }
        l0 += bad0;
        l1 += bad1;
        const float n0 = fmaxf(m0, quad_max(t0)), n1 = fmaxf(m1, quad_max(t1));
        const float b0 = n0 == -INFINITY ? 0.f : -n0, b1 = n1 == -INFINITY ? 0.f : -n1;
        if (__any_sync(0xffffffffu, n0 != m0 || n1 != m1)) {
          const float f0 = fast_exp2(m0 + b0), f1 = fast_exp2(m1 + b1);      // m = -inf: nothing summed yet, the factor is 0
          l0 *= f0;
          l1 *= f1;
#pragma unroll
          for (int d = 0; d < D / 8; ++d) {
            o[d][0] *= f0;
            o[d][1] *= f0;
            o[d][2] *= f1;
            o[d][3] *= f1;
          }
          m0 = n0;
          m1 = n1;
        }
        uint32_t pa[kRowKeys / 16][4];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const float a0 = ks[t] * s0, a1 = ks[t] * s1;
          const float c0 = b0 + lv[t] + (CODES ? kHalfShift : 0.f), c1 = b1 + lv[t] + (CODES ? kHalfShift : 0.f);
          float u0 = 0.f, u1 = 0.f;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int j = 2 * t + h;
            const float p0 = fast_exp2(fmaf(sc[j][0], a0, c0)), p1 = fast_exp2(fmaf(sc[j][1], a0, c0));
            const float p2 = fast_exp2(fmaf(sc[j][2], a1, c1)), p3 = fast_exp2(fmaf(sc[j][3], a1, c1));
            u0 += p0 + p1;
            u1 += p2 + p3;
            pa[t][h * 2] = CODES ? pack_half(p0, p1) : pack_bf16(p0, p1);
            pa[t][h * 2 + 1] = CODES ? pack_half(p2, p3) : pack_bf16(p2, p3);
          }
          l0 = fmaf(u0, iv[t], l0);
          l1 = fmaf(u1, iv[t], l1);
        }
        if (key0 + kRowKeys > in_use || !it.span.sees_all(key0, kRowKeys)) {
          // values of slots that the unit does not see may be anything, and 0 * garbage must not reach O
          for (int sl = 0; sl < S::kSlabs; ++sl)
            for (int j = lane; j < kRowKeys * 8; j += 32) {
              const int key = key0 + (j >> 3);
              if (key >= in_use || !it.span.sees(key))
                *reinterpret_cast<uint4*>(smem + slot * S::kStage + S::kTile + sl * S::kSlab + j * 16) = make_uint4(0u, 0u, 0u, 0u);
            }
          fence_proxy_async();                             // (the slot's next copy is ordered behind these stores)
          __syncwarp();
        }
        if constexpr (CODES) {
#pragma unroll
          for (int d = 0; d < D / 32; ++d) {               // 32 columns: two pieces of 16 codes
#pragma unroll
            for (int k = 0; k < kRowKeys / 16; ++k) {
              uint32_t vb[4];                              // keys 0 .. 7 and 8 .. 15 of the first piece, then of the second
              load_matrices_t(vb, v_at + k * 2048 + vc_row + (((d * 2 + vc_piece) ^ v_key) << 4));
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const uint32_t even = __byte_perm(vb[2 * h], vb[2 * h + 1], 0x6420), odd = __byte_perm(vb[2 * h], vb[2 * h + 1], 0x7531);
                uint32_t b0, b1;
                half_of_codes(even, b0, b1);
                mma_16x8x16<true>(o[(2 * d + h) * 2], pa[k], b0, b1);
                half_of_codes(odd, b0, b1);
                mma_16x8x16<true>(o[(2 * d + h) * 2 + 1], pa[k], b0, b1);
              }
            }
          }
        } else {
#pragma unroll
          for (int d = 0; d < D / 16; ++d) {
#pragma unroll
            for (int k = 0; k < kRowKeys / 16; ++k) {      // 16 keys of 16 columns
              uint32_t vb[4];
              load_matrices_t(vb, v_at + (d >> 2) * S::kSlab + k * 2048 + v_row + ((((d & 3) * 2 + v_piece) ^ swz) << 4));
              mma_16x8x16<false>(o[2 * d], pa[k], vb[0], vb[1]);
              mma_16x8x16<false>(o[2 * d + 1], pa[k], vb[2], vb[3]);
            }
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(empty(slot));
      }
      before += it.steps;

      // ---- the warps' parts are joined: m* = max m_w, l* = sum l_w 2^(m_w - m*), out = sum o_w 2^(m_w - m*) / l*.  (After an abort
      // every warp still comes to the barriers.)
      l0 = quad_sum(l0);
      l1 = quad_sum(l1);
      if (quad == 0) {
        ml[warp * kFewRows + row] = make_float2(m0, l0);
        ml[warp * kFewRows + row + 8] = make_float2(m1, l1);
      }
      float* part0 = acc + (warp * kFewRows + row) * S::kAccRow;
      float* part1 = part0 + 8 * S::kAccRow;
      if constexpr (CODES) {
#pragma unroll
        for (int d = 0; d < D / 16; ++d) {
          const float *e = o[2 * d], *f = o[2 * d + 1];
          *reinterpret_cast<float4*>(part0 + d * 16 + quad * 4) = make_float4(e[0], f[0], e[1], f[1]);
          *reinterpret_cast<float4*>(part1 + d * 16 + quad * 4) = make_float4(e[2], f[2], e[3], f[3]);
        }
      } else {
#pragma unroll
        for (int d = 0; d < D / 8; ++d) {
          *reinterpret_cast<float2*>(part0 + d * 8 + col) = make_float2(o[d][0], o[d][1]);
          *reinterpret_cast<float2*>(part1 + d * 8 + col) = make_float2(o[d][2], o[d][3]);
        }
      }
      asm volatile("bar.sync 1, %0;" ::"n"(32 * S::kWarps) : "memory");
      {
        constexpr int kLanes = 2 * S::kWarps;              // threads to a row
        const int r = tid / kLanes, c = (tid % kLanes) * 4, tok = r / G, head = r - tok * G, token = it.first + tok;
        if (tok < p.tpt && token < it.n) {
          float2 part[S::kWarps];
          float m = -INFINITY, l = 0.f;
#pragma unroll
          for (int w = 0; w < S::kWarps; ++w) {
            part[w] = ml[w * kFewRows + r];
            m = fmaxf(m, part[w].x);
          }
          const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
          for (int w = 0; w < S::kWarps; ++w) {
            part[w].x = fast_exp2(part[w].x - base);
            l = fmaf(part[w].y, part[w].x, l);
          }
          const float inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);                   // a NaN sum stays one
#pragma unroll
          for (int e = 0; e < D; e += 4 * kLanes) {
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < S::kWarps; ++w) {
              const float4 a = *reinterpret_cast<const float4*>(acc + (w * kFewRows + r) * S::kAccRow + e + c);
              v = make_float4(fmaf(a.x, part[w].x, v.x), fmaf(a.y, part[w].x, v.y), fmaf(a.z, part[w].x, v.z), fmaf(a.w, part[w].x, v.w));
            }
            if (it.slot < 0)
              *reinterpret_cast<uint2*>(p.out + (static_cast<size_t>(it.start + token) * p.Hq + it.g * G + head) * D + e + c) =
                  make_uint2(pack_bf16(v.x * inv, v.y * inv), pack_bf16(v.z * inv, v.w * inv));
            else
              *reinterpret_cast<float4*>(p.work.part_o + (static_cast<size_t>(it.slot) * (D / 4) + (e + c) / 4) * (kFewRows * 4) + r * 4) = v;
          }
          if (it.slot >= 0 && c == 0) p.work.part_ml[static_cast<size_t>(it.slot) * kFewRows + r] = make_float2(m, l);
        }
      }
      asm volatile("bar.sync 1, %0;" ::"n"(32 * S::kWarps) : "memory");
    }
  }
  __syncthreads();
  if (*s_abort) {
    if (tid == 0) report_status(p.status, EAGLE_ERR_TIMEOUT);
    let_work_land();
  }
}

template <int D, bool CODES>
cudaError_t launch(const ChunkParams& p, cudaStream_t stream) {
  using S = RowSmem<D, CODES>;
  CUtensorMap mk, mv;
  const bool paged = p.block_table != nullptr;
  const int box_rows = paged && p.page_size < kRowKeys ? p.page_size : kRowKeys;
  const long long n1 = paged ? p.page_size : (p.capacity > 0 ? p.capacity : 1);
  const long long n2 = paged ? static_cast<long long>(p.num_pages) * p.Hkv : static_cast<long long>(p.B) * p.Hkv;
  if constexpr (CODES) {
    if (!map_codes_3d(&mk, p.k, n1, n2, 128, box_rows, true) || !map_codes_3d(&mv, p.v, n1, n2, 128, box_rows, true)) return cudaErrorInvalidValue;
  } else {
    if (!map_bf16_3d(&mk, p.k, D, n1, n2, 64, box_rows, 1) || !map_bf16_3d(&mv, p.v, D, n1, n2, 64, box_rows, 1)) return cudaErrorInvalidValue;
  }
  BehindLaunch at(p.num_workers, S::kThreads, S::kBytes, stream);
  auto kernel = p.stall_after_tiles >= 0 ? (paged ? window_rows_kernel<D, true, CODES, true> : window_rows_kernel<D, false, CODES, true>)
                                         : (paged ? window_rows_kernel<D, true, CODES, false> : window_rows_kernel<D, false, CODES, false>);
  return cudaLaunchKernelEx(&at.config, kernel, p, mk, mv);
}

template <int D, bool CODES>
cudaError_t prepare() {
  for (auto kernel : {window_rows_kernel<D, false, CODES, false>, window_rows_kernel<D, true, CODES, false>, window_rows_kernel<D, false, CODES, true>,
                      window_rows_kernel<D, true, CODES, true>}) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, RowSmem<D, CODES>::kBytes);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace

cudaError_t window_rows_prepare(int head_dim) {
  if (head_dim == 64) return prepare<64, false>();
  const cudaError_t e = prepare<128, false>();
  return e == cudaSuccess ? prepare<128, true>() : e;
}
cudaError_t launch_window_rows(const ChunkParams& p, cudaStream_t stream) {
  if (p.k_scale) return launch<128, true>(p, stream);
  return p.D == 128 ? launch<128, false>(p, stream) : launch<64, false>(p, stream);
}

}  // namespace eagle
