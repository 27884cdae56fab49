// Attention of single tokens with a window over block-scaled codes: 8 or 16 query rows of one (sequence, KV head) against the slots that they see,
// streamed through a ring in shared memory.
//
// Bound by the reading of the cache, which is half of what the bf16 kernel (window_rows.cu) reads, so that everything that is done per key has
// to take half as long.  What differs from it:
//
// The products are turned around, S' = K Q' and O' = V' P': keys, then columns of the head, are the 16 rows of a matrix instruction and query rows its
// 8 columns, so a group of up to 8 heads takes half of the instructions that 16 query rows would.  The codes are the left operand, widened to
// fp16 (exactly) in registers.  The order of the contraction over the head is free: a lane reads 16 codes of a key at once (the keys of a group of eight
// permuted so that the eight lanes of a 16-byte access meet no bank twice) and queries are arranged to match.  Values come through the
// transposing matrix load as pairs of codes, neighbours in the head, whose bytes are sorted into even and odd columns: eight rows of an instruction
// each.  Probabilities change sides by an 8 x 8 transposition within the warp.
//
// With the blocks' scales, z = (q.c) ks scale, and the maximum is taken over z + log2 vs: then 2^(z + log2 vs - m) is the weight of the code itself,
// never too large for fp16, and the row sum is divided by vs again, once per 16 keys.  Query rows are scaled by a power of two (row_factor).
//
// Copies are 64 keys with their values, eight of them in flight; one warp looks up pages and issues them, another one brings the scales (a
// single warp for both was what the kernel waited for).
//
// From a graph, with planner and merge: 64 single tokens over 512 to 8192 slots, 32 heads over 8 (608 MB): 125 us, 4.9 TB/s (278 us as 16 query rows by
// 8 keys, four warps' worth of copies at a time and one warp for pages and scales); one token over 65536 slots, 64 heads over 8 (134 MB): 42 us (planner,
// merge and their launches are about 12 us of it).
#include "window.cuh"

namespace eagle {

namespace {

using namespace tc;

constexpr int D = 128;
constexpr int kKeys = 64, kTiles16 = kKeys / 16;           // keys of a step, in matrix instructions' rows
constexpr int kWarps = 8, kThreads = 32 * (kWarps + 2);

template <int NT>                                          // query rows: 8 NT
struct CodeSmem {
  static constexpr int kRows = 8 * NT;
  static constexpr int kTile = kKeys * D, kStage = 2 * kTile;      // K, then V: 128-byte swizzled rows
  static constexpr int kStages = 8;
  // A warp takes all uses of a slot: copies land in any order, and a warp that came to a slot's next use before another had seen
  // the last one would find its parity there already.
  static_assert(kStages % kWarps == 0, "a slot belongs to one warp");
  static constexpr int kAccRow = D + 4;                      // (8-byte stores of 16 lanes, four rows two apart and four columns, meet no bank twice)
  static constexpr int kAcc = kStages * kStage;              // float [warps][rows][kAccRow]
  static constexpr int kMl = kAcc + kWarps * kRows * kAccRow * 4;          // float2 [warps][rows]: maximum and sum
  static constexpr int kScale = kMl + kWarps * kRows * 8;    // float [kStages][8]: ks, then vs, of 16 keys each
  static constexpr int kBar = kScale + kStages * 32;         // full [kStages], empty [kStages]
  static constexpr int kMisc = kBar + 16 * kStages;          // abort flag (at + 4), wait limit (8 bytes)
  static constexpr int kBytes = kMisc + 16;
  static_assert(kBytes <= 227 * 1024, "shared memory of an SM");
};

__device__ __forceinline__ void load_matrices_t(uint32_t* r, uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint4 load_shared(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}
// c[16 x 8] += a[16 x 16] b[16 x 8], fp16 operands
__device__ __forceinline__ void mma_16x8x16(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, const uint32_t* b) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b[0]), "r"(b[1]));
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {      // of an 8 x 8 matrix of 16-bit elements
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// Over the lanes with the same l % 4: those of a column.
__device__ __forceinline__ float column_max(float x) {
  x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
  x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
  return fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
}
__device__ __forceinline__ float column_sum(float x) {
  x += __shfl_xor_sync(0xffffffffu, x, 4);
  x += __shfl_xor_sync(0xffffffffu, x, 8);
  return x + __shfl_xor_sync(0xffffffffu, x, 16);
}
// One 4-byte copy that reports to no one by itself, and the arrival of all of this lane's copies at a barrier.
__device__ __forceinline__ void copy_word(uint32_t dst, const float* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void arrive_with_copies(uint32_t bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}

__device__ const float kNoScale = 1.f;                       // what stands for the scales of a page outside the pool

template <int NT, bool PAGED, bool STALL>                    // (STALL: of the test hook, as in chunk.cu)
__global__ void __launch_bounds__(kThreads, 1)
window_codes_kernel(ChunkParams p, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v) {
  using S = CodeSmem<NT>;
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
    for (int i = 0; i < S::kStages; ++i) { mbar_init(full(i), 9); mbar_init(empty(i), 1); }      // (eight lanes bring scales)
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
    __device__ int key(int step) const { return place0 + step * kKeys + (place0 + step * kKeys >= span.before * kChunkTile ? span.skip * kChunkTile : 0); }
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
    it.steps = b.w > b.z ? static_cast<int>((end - it.place0 + kKeys - 1) / kKeys) : 0;
    it.slot = at[2].x;
    return it;
  };
  // The helpers walk the work list a step at a time.
  struct Walk {
    Item it;
    int i, step;
  };
  auto next_step = [&](Walk& w) {          // false: the list is at its end
    if (++w.step < w.it.steps) return true;
    for (++w.i; w.i < n_items; ++w.i) {
      w.it = item(w.i);
      if (w.it.steps > 0) break;
    }
    w.step = 0;
    return w.i < n_items;
  };
  // A key past the sequence's last page stands for that page, one of a page that holds nothing the unit sees for the first that does.
  auto page_of = [&](const Item& it, int key) {
    const int last = (it.L + it.n - 1) >> p.page_shift, pi = key >> p.page_shift;
    return __ldg(p.block_table + static_cast<size_t>(it.b) * p.max_pages + it.span.page(pi < last ? pi : last, p.page_shift));
  };

  if (warp == kWarps) {
    // =========================================================================== copies
    // A lane per box (a page's rows x 128 codes, of K or of V); the page of a lane's next box is looked up while the box before it is on its
    // way.  Boxes that nothing is seen of fetch a page that is (their rows are masked), so that a tile's byte count never changes; an
    // entry outside the pool reads page 0, and marks its sequence when the item ends (the merge kernel reports it and zeroes the rows).
    const int box_rows = PAGED ? min(p.page_size, kKeys) : kKeys, per = kKeys / box_rows;
    const bool is_v = lane >= per, active = lane < 2 * per;
    const int r0 = (lane - (is_v ? per : 0)) * box_rows;
    const uint32_t dst = sbase + (is_v ? S::kTile : 0) + r0 * 128;
    Walk w;
    w.it.steps = 0;
    w.i = w.step = -1;
    int y = 0, z = 0;
    bool wrong = false;                                    // some entry of the item was outside the pool
    auto look_up = [&]() {
      y = w.it.key(w.step) + r0;
      z = w.it.b;
      if (PAGED && active) {
        z = page_of(w.it, y);
        y &= p.page_size - 1;
      }
    };
    bool more = next_step(w);
    if (more) look_up();
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
      if (active) tma_load_3d(dst + ring.slot * S::kStage, is_v ? &map_v : &map_k, 0, y, page * p.Hkv + w.it.g, full(ring.slot));
      ring.step();
      if (w.step + 1 >= w.it.steps) {
        if (PAGED && wrong) p.work.bad_page[w.it.b] = 1;
        wrong = false;
      }
      more = next_step(w);
      if (more) look_up();
    }
  } else if (warp == kWarps + 1) {
    // =========================================================================== scales: four groups of 16 keys, ks and vs
    Walk w;
    w.it.steps = 0;
    w.i = w.step = -1;
    const float* scales = lane < 4 ? p.k_scale : p.v_scale;
    long long row = 0;                                     // page (or sequence) of this lane's group
    int y = 0;
    auto look_up = [&]() {
      y = min(w.it.key(w.step) + (lane & 3) * 16, static_cast<int>(p.capacity) - 1);
      row = w.it.b;
      if (PAGED && lane < 8) {
        row = page_of(w.it, y);
        y &= p.page_size - 1;
      }
    };
    bool more = next_step(w);
    if (more) look_up();
    Ring<S::kStages> ring;
    while (more) {
      if (!mbar_wait_warp(empty(ring.slot), ring.par ^ 1u, s_abort)) break;
      if (lane < 8) {
        const bool out_of_pool = PAGED && static_cast<unsigned long long>(row) >= static_cast<unsigned long long>(p.num_pages);
        copy_word(sbase + S::kScale + ring.slot * 32 + lane * 4, out_of_pool ? &kNoScale : scales + (row * p.Hkv + w.it.g) * p.head_blocks + (y >> p.block_shift));
        arrive_with_copies(full(ring.slot));
      }
      ring.step();
      more = next_step(w);
      if (more) look_up();
    }
  } else {
    // =========================================================================== scores, softmax, output
    // A lane holds, of every 16 keys, two (8 apart) in two columns: query rows 2 (l % 4), + 1.  fp32 throughout, in the log2 domain; the
    // probabilities times vs are rounded to fp16 for the second product (relative 2^-11 each), the sum that divides them is kept from the
    // unrounded ones.
    const int sub = lane >> 2, quad = lane & 3, G = p.G;
    float* acc = reinterpret_cast<float*>(smem + S::kAcc);
    float2* ml = reinterpret_cast<float2*>(smem + S::kMl);
    const uint32_t spread = ((sub & 1) << 2) | (sub >> 1);                         // key of a group of eight that this lane's rows are of
    const uint32_t v_key = ((lane & 1) << 2) | ((lane & 7) >> 1);                  // and that it addresses for the transposing load
    const uint32_t v_row = (((lane >> 3) & 1) * 8 + v_key) * 128, v_piece = lane >> 4;
    uint32_t before = 0;                                   // tiles of the items before
    bool ok = true;
    for (int i = 0; i < n_items; ++i) {
      const Item it = item(i);
      if (it.steps <= 0) continue;                         // (uniform over the CTA)
      // queries: the right operand, four neighbours per 16 of the contraction (those of the codes of a word)
      uint32_t q[NT][D / 16][2];
      float scale[NT][2];                                  // of this lane's columns, with what their rows were multiplied by
      int limit[NT][2], low[NT][2];                        // the last key a column's row sees, and the first behind the sinks
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const int row = t * 8 + sub, tok = row / G;
        const bool valid = tok < p.tpt && it.first + tok < it.n;
        const __nv_bfloat16* src = p.q + (static_cast<size_t>(it.start + it.first + tok) * p.Hq + it.g * G + (row - tok * G)) * D;
        uint32_t top = 0;
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const uint2 a = valid ? __ldg(reinterpret_cast<const uint2*>(src + (k >> 2) * 64 + quad * 16 + (k & 3) * 4)) : make_uint2(0u, 0u);
          q[t][k][0] = a.x;
          q[t][k][1] = a.y;
          top = max(top, max(magnitude_bits(a.x), magnitude_bits(a.y)));
        }
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const RowFactor f = row_factor(top);
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          q[t][k][0] = half_of_bf16(q[t][k][0], f.down);
          q[t][k][1] = half_of_bf16(q[t][k][1], f.down);
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          scale[t][j] = p.scale_log2 * __shfl_sync(0xffffffffu, f.up, (2 * quad + j) * 4);
          limit[t][j] = it.L + it.first + (t * 8 + 2 * quad + j) / G;
          low[t][j] = p.window > 0 ? limit[t][j] - p.window + 1 : 0;
        }
      }
      const int low_last = p.window > 0 ? it.L + it.first + p.tpt - p.window : 0;        // from here on every row sees all behind the sinks
      // accumulators: even and odd columns of 16, by query rows
      float o[NT][D / 16][4];
      float m[NT][2], l[NT][2];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int d = 0; d < D / 16; ++d) o[t][d][0] = o[t][d][1] = o[t][d][2] = o[t][d][3] = 0.f;
        m[t][0] = m[t][1] = -INFINITY;
        l[t][0] = l[t][1] = 0.f;
      }
      for (int s = static_cast<int>((warp - before) & (kWarps - 1)); s < it.steps && ok; s += kWarps) {
        const uint32_t gs = before + s, slot = gs % S::kStages, par = (gs / S::kStages) & 1u;
        const uint32_t k_at = sbase + slot * S::kStage, v_at = k_at + S::kTile;
        const int key0 = it.key(s), in_use = it.L + it.n;  // in_use: slots of the sequence
        ok = mbar_wait_warp(full(slot), par, s_abort);
        if (!ok) break;
        float sc[NT][kTiles16][4];
#pragma unroll
        for (int u = 0; u < kTiles16; ++u) {
#pragma unroll
          for (int t = 0; t < NT; ++t) sc[t][u][0] = sc[t][u][1] = sc[t][u][2] = sc[t][u][3] = 0.f;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t at = k_at + (u * 16 + spread) * 128 + (((h * 4 + quad) ^ spread) << 4);
            const uint4 lo = load_shared(at), hi = load_shared(at + 1024);
            const uint32_t wl[4] = {lo.x, lo.y, lo.z, lo.w}, wh[4] = {hi.x, hi.y, hi.z, hi.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              uint32_t a0, a1, a2, a3;
              half_of_codes(wl[k], a0, a2);
              half_of_codes(wh[k], a1, a3);
#pragma unroll
              for (int t = 0; t < NT; ++t) mma_16x8x16(sc[t][u], a0, a1, a2, a3, q[t][h * 4 + k]);
            }
          }
        }
        // scales of the 16 keys; those that the unit sees nothing of may be anything
        float ks[kTiles16], vs[kTiles16];
        {
          const uint4 a = load_shared(sbase + S::kScale + slot * 32), b = load_shared(sbase + S::kScale + slot * 32 + 16);
          const uint32_t wa[4] = {a.x, a.y, a.z, a.w}, wb[4] = {b.x, b.y, b.z, b.w};
          uint32_t worst = 0;
#pragma unroll
          for (int u = 0; u < kTiles16; ++u) {
            const bool seen = key0 + u * 16 < in_use && it.span.sees_some(key0 + u * 16, 16);
            ks[u] = seen ? __uint_as_float(wa[u]) : 1.f;
            vs[u] = seen ? __uint_as_float(wb[u]) : 1.f;
            worst = max(worst, beyond_range(vs[u]));
          }
          if (worst > kScaleRange) report_status(p.status, EAGLE_ERR_SCALE);
        }
        if (!(key0 + kKeys - 1 <= it.L + it.first && (key0 >= low_last || key0 + kKeys <= p.sinks))) {      // a tile that some row does not see whole
#pragma unroll
          for (int u = 0; u < kTiles16; ++u)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const int key = key0 + u * 16 + static_cast<int>(spread) + (e >> 1) * 8;
                if (key > limit[t][e & 1] || (key < low[t][e & 1] && key >= p.sinks)) sc[t][u][e] = -INFINITY;
              }
        }
        // column maxima in the log2 domain
        bool outgrown = false;
        float top[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            float x = -INFINITY;
#pragma unroll
            for (int u = 0; u < kTiles16; ++u) {
              const float z = fmaf(max3_nan(sc[t][u][j], sc[t][u][2 + j], -INFINITY), score_factor(ks[u], scale[t][j]), fast_log2(vs[u]));
              if (!(z < INFINITY)) l[t][j] = __uint_as_float(0x7fffffffu);      // NaN or +inf makes the row NaN
              x = fmaxf(x, z);
            }
            top[t][j] = fmaxf(m[t][j], column_max(x));
            outgrown |= top[t][j] != m[t][j];
          }
        if (__any_sync(0xffffffffu, outgrown)) {
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            const float f0 = fast_exp2(m[t][0] - (top[t][0] == -INFINITY ? 0.f : top[t][0]));      // m = -inf: nothing summed yet, the factor is 0
            const float f1 = fast_exp2(m[t][1] - (top[t][1] == -INFINITY ? 0.f : top[t][1]));
            l[t][0] *= f0;
            l[t][1] *= f1;
#pragma unroll
            for (int d = 0; d < D / 16; ++d) {
              o[t][d][0] *= f0;
              o[t][d][1] *= f1;
              o[t][d][2] *= f0;
              o[t][d][3] *= f1;
            }
            m[t][0] = top[t][0];
            m[t][1] = top[t][1];
          }
        }
        uint32_t pb[NT][kTiles16][2];
#pragma unroll
        for (int u = 0; u < kTiles16; ++u) {
          const float lv = fast_log2(vs[u]) + kHalfShift, iv = fast_rcp(vs[u]);
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            const float a0 = score_factor(ks[u], scale[t][0]), a1 = score_factor(ks[u], scale[t][1]);
            const float c0 = lv - (m[t][0] == -INFINITY ? 0.f : m[t][0]), c1 = lv - (m[t][1] == -INFINITY ? 0.f : m[t][1]);
            const float p0 = fast_exp2(fmaf(sc[t][u][0], a0, c0)), p1 = fast_exp2(fmaf(sc[t][u][1], a1, c1));
            const float p2 = fast_exp2(fmaf(sc[t][u][2], a0, c0)), p3 = fast_exp2(fmaf(sc[t][u][3], a1, c1));
            l[t][0] = fmaf(p0 + p2, iv, l[t][0]);
            l[t][1] = fmaf(p1 + p3, iv, l[t][1]);
            pb[t][u][0] = transposed(pack_half(p0, p1));
            pb[t][u][1] = transposed(pack_half(p2, p3));
          }
        }
        if (key0 + kKeys > in_use || !it.span.sees_all(key0, kKeys)) {
          // values of slots that the unit does not see may be anything, and 0 * garbage must not reach O
          for (int j = lane; j < kKeys * 8; j += 32) {
            const int key = key0 + (j >> 3);
            if (key >= in_use || !it.span.sees(key)) *reinterpret_cast<uint4*>(smem + slot * S::kStage + S::kTile + j * 16) = make_uint4(0u, 0u, 0u, 0u);
          }
          fence_proxy_async();                             // (the slot's next copy is ordered behind these stores)
          __syncwarp();
        }
#pragma unroll
        for (int u = 0; u < kTiles16; ++u) {
#pragma unroll
          for (int d = 0; d < D / 32; ++d) {               // 32 columns: two pieces of 16 codes
            uint32_t vb[4];                                // keys 0 .. 7 and 8 .. 15 of the first piece, then of the second
            load_matrices_t(vb, v_at + u * 2048 + v_row + (((d * 2 + v_piece) ^ v_key) << 4));
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              uint32_t a0, a1, a2, a3;
              half_of_codes(__byte_perm(vb[2 * h], vb[2 * h + 1], 0x6420), a0, a2);
              half_of_codes(__byte_perm(vb[2 * h], vb[2 * h + 1], 0x7531), a1, a3);
#pragma unroll
              for (int t = 0; t < NT; ++t) mma_16x8x16(o[t][2 * d + h], a0, a1, a2, a3, pb[t][u]);
            }
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(empty(slot));
      }
      before += it.steps;

      // ---- the warps' parts are joined: m* = max m_w, l* = sum l_w 2^(m_w - m*), out = sum o_w 2^(m_w - m*) / l*.  (After an abort
      // every warp still comes to the barriers.)
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int row = warp * S::kRows + t * 8 + 2 * quad + j;
          const float sum = column_sum(l[t][j]);
          if (sub == 0) ml[row] = make_float2(m[t][j], sum);
#pragma unroll
          for (int d = 0; d < D / 16; ++d) *reinterpret_cast<float2*>(acc + row * S::kAccRow + d * 16 + 2 * sub) = make_float2(o[t][d][j], o[t][d][2 + j]);
        }
      asm volatile("bar.sync 1, %0;" ::"n"(32 * kWarps) : "memory");
      {
        constexpr int kLanes = 32 * kWarps / S::kRows;     // threads to a row
        const int r = tid / kLanes, c = (tid % kLanes) * 4, tok = r / G, head = r - tok * G, token = it.first + tok;
        if (tok < p.tpt && token < it.n) {
          float2 part[kWarps];
          float top = -INFINITY, sum = 0.f;
#pragma unroll
          for (int w = 0; w < kWarps; ++w) {
            part[w] = ml[w * S::kRows + r];
            top = fmaxf(top, part[w].x);
          }
          const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
          for (int w = 0; w < kWarps; ++w) {
            part[w].x = fast_exp2(part[w].x - base);
            sum = fmaf(part[w].y, part[w].x, sum);
          }
          const float inv = sum > 0.f ? 1.f / sum : (sum == 0.f ? 0.f : sum);                   // a NaN sum stays one
#pragma unroll
          for (int e = 0; e < D; e += 4 * kLanes) {
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
              const float4 a = *reinterpret_cast<const float4*>(acc + (w * S::kRows + r) * S::kAccRow + e + c);
              v = make_float4(fmaf(a.x, part[w].x, v.x), fmaf(a.y, part[w].x, v.y), fmaf(a.z, part[w].x, v.z), fmaf(a.w, part[w].x, v.w));
            }
            if (it.slot < 0)
              *reinterpret_cast<uint2*>(p.out + (static_cast<size_t>(it.start + token) * p.Hq + it.g * G + head) * D + e + c) =
                  make_uint2(pack_bf16(v.x * inv, v.y * inv), pack_bf16(v.z * inv, v.w * inv));
            else
              *reinterpret_cast<float4*>(p.work.part_o + (static_cast<size_t>(it.slot) * (D / 4) + (e + c) / 4) * (S::kRows * 4) + r * 4) = v;
          }
          if (it.slot >= 0 && c == 0) p.work.part_ml[static_cast<size_t>(it.slot) * S::kRows + r] = make_float2(top, sum);
        }
      }
      asm volatile("bar.sync 1, %0;" ::"n"(32 * kWarps) : "memory");
    }
  }
  __syncthreads();
  if (*s_abort) {
    if (tid == 0) report_status(p.status, EAGLE_ERR_TIMEOUT);
    let_work_land();
  }
}

template <int NT>
cudaError_t launch(const ChunkParams& p, cudaStream_t stream) {
  using S = CodeSmem<NT>;
  CUtensorMap mk, mv;
  const bool paged = p.block_table != nullptr;
  const int box_rows = paged && p.page_size < kKeys ? p.page_size : kKeys;
  const long long n1 = paged ? p.page_size : (p.capacity > 0 ? p.capacity : 1);
  const long long n2 = paged ? static_cast<long long>(p.num_pages) * p.Hkv : static_cast<long long>(p.B) * p.Hkv;
  if (!map_codes_3d(&mk, p.k, n1, n2, 128, box_rows, true) || !map_codes_3d(&mv, p.v, n1, n2, 128, box_rows, true)) return cudaErrorInvalidValue;
  BehindLaunch at(p.num_workers, kThreads, S::kBytes, stream);
  auto kernel = p.stall_after_tiles >= 0 ? (paged ? window_codes_kernel<NT, true, true> : window_codes_kernel<NT, false, true>)
                                         : (paged ? window_codes_kernel<NT, true, false> : window_codes_kernel<NT, false, false>);
  return cudaLaunchKernelEx(&at.config, kernel, p, mk, mv);
}

template <int NT>
cudaError_t prepare() {
  for (auto kernel : {window_codes_kernel<NT, false, false>, window_codes_kernel<NT, true, false>, window_codes_kernel<NT, false, true>,
                      window_codes_kernel<NT, true, true>}) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, CodeSmem<NT>::kBytes);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace

cudaError_t window_codes_prepare() {
  const cudaError_t e = prepare<1>();
  return e == cudaSuccess ? prepare<2>() : e;
}
cudaError_t launch_window_codes(const ChunkParams& p, cudaStream_t stream) { return p.rows == 8 ? launch<1>(p, stream) : launch<2>(p, stream); }

}  // namespace eagle
