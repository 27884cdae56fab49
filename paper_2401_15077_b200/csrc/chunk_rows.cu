// Chunk attention of single tokens: 16 query rows of one (sequence, KV head) against the cache, streamed through a ring in
// shared memory.
//
// Bound by the reading of the cache: a key and its value are 4 D bytes for 4 G D operations, so the matrix work is small whatever
// unit does it, and the 128-row tiles of the tensor-memory path would spend a longer chain of waits per tile than the bytes take.
// Here one warp issues copies of 32 keys with their values as far ahead as shared memory allows (192 KB in flight per SM), and four
// warps take the tiles in turn, each with its own running maximum, sum and accumulator in registers (16-row matrix
// instructions: scores leave one as the operand of the next).  The four are joined when the item ends, which the copies of the next
// item do not wait for.
//
// 64 single tokens over 512 to 8192 slots (1.21 GB of keys and values, 32 heads over 8, D = 128): 203 us with planner and merge (from a
// graph; a call 212 us), 6.0 TB/s of the 6.6 TB/s that a plain copy reaches; one token over 65536 slots (268 MB, 64 heads over 8): 59.5 us,
// 4.5 TB/s (planner, merge and two launches are about 12 us of it).
#include "chunk.cuh"
#include "tc.cuh"

namespace eagle {

namespace {

using namespace tc;

constexpr int kRowWarps = 4, kRowThreads = 32 * (kRowWarps + 1);
constexpr int kRowKeys = 32;             // keys of a tile: a quarter of a K/V tile of the plan

template <int D>
struct RowSmem {
  static constexpr int kSlabs = D / 64;                      // 64 bf16 = one 128-byte swizzled row
  static constexpr int kSlab = kRowKeys * 128, kTile = kSlabs * kSlab, kStage = 2 * kTile;    // K, then V
  static constexpr int kStages = 12 * 128 / D;
  // A warp takes all uses of a slot: copies land in any order, and a warp that came to a slot's next use before another had seen
  // the last one would find its parity there already.
  static_assert(kStages % kRowWarps == 0, "a slot belongs to one warp");
  static constexpr int kAccRow = D + 8;                      // (rows 8 floats apart in the banks: 8-byte stores of four rows do not meet)
  static constexpr int kAcc = kStages * kStage;              // float [4 warps][16][kAccRow]
  static constexpr int kMl = kAcc + kRowWarps * kFewRows * kAccRow * 4;      // float2 [4 warps][16]: maximum and sum
  static constexpr int kBar = kMl + kRowWarps * kFewRows * 8;                // full [kStages], empty [kStages]
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
// c[16 x 8] += a[16 x 16] b[16 x 8]
__device__ __forceinline__ void mma_16x8x16(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float quad_max(float x) {
  x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
  return fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
}
__device__ __forceinline__ float quad_sum(float x) {
  x += __shfl_xor_sync(0xffffffffu, x, 1);
  return x + __shfl_xor_sync(0xffffffffu, x, 2);
}

template <int D, bool PAGED, bool STALL>                     // (STALL: of the test hook, as in chunk.cu)
__global__ void __launch_bounds__(kRowThreads, 1)
chunk_rows_kernel(ChunkParams p, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v) {
  using S = RowSmem<D>;
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
    for (int i = 0; i < S::kStages; ++i) { mbar_init(full(i), 1); mbar_init(empty(i), 1); }
    *s_abort = 0;
    *reinterpret_cast<volatile unsigned long long*>(smem + S::kMisc + 8) = p.wait_limit_ns;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  launch_dependents();
  wait_for_prerequisites();                // the plan is there
  const int4 mine = p.work.cta[blockIdx.x];              // whole units first, then this CTA's share of the rest
  const int n_items = mine.y + mine.w;
  struct Item {
    int b, g, first, start, n, L, key0, steps, slot;     // first: token of the chunk in row 0; keys from key0 on, `steps` tiles
  };
  auto item = [&](int i) {
    const int4* at = reinterpret_cast<const int4*>(p.work.items + (i < mine.y ? mine.x + i : mine.z + (i - mine.y)));
    const int4 a = at[0], b = at[1];
    const int first = a.z * p.tpt;
    const int keys = b.y + min(first + p.tpt, b.x);      // what the last row sees
    const long long end = static_cast<long long>(b.w) * kChunkTile < keys ? static_cast<long long>(b.w) * kChunkTile : keys;
    const int key0 = b.z * kChunkTile;
    return Item{a.x, a.y, first, a.w, b.x, b.y, key0, b.w > b.z ? static_cast<int>((end - key0 + kRowKeys - 1) / kRowKeys) : 0, at[2].x};
  };

  if (warp == kRowWarps) {
    // =========================================================================== copies
    // A lane per box (a page's rows x 64 columns, of K or of V); the page of a lane's next box is looked up while the box before it
    // is on its way.  A box past the sequence's last page fetches that page again (its rows are masked), so that a tile's byte count
    // never changes; an entry outside the pool reads page 0, and marks its sequence when the item ends (the merge kernel reports it and
    // zeroes the rows).
    const int box_rows = PAGED ? min(p.page_size, kRowKeys) : kRowKeys, per = S::kSlabs * (kRowKeys / box_rows);
    const bool is_v = lane >= per, active = lane < 2 * per;
    const int r0 = ((lane - (is_v ? per : 0)) / S::kSlabs) * box_rows, sl = lane % S::kSlabs;      // (per is a multiple of kSlabs)
    const uint32_t dst = sbase + (is_v ? S::kTile : 0) + sl * S::kSlab + r0 * 128;
    Item it = {};
    int i = -1, step = 0, y = 0, z = 0;
    bool more = true, wrong = false;                       // wrong: some entry of the item was outside the pool
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
      y = it.key0 + step * kRowKeys + r0;
      z = it.b;
      if (PAGED && active) {
        const int last = (it.L + it.n - 1) >> p.page_shift, pi = y >> p.page_shift;
        z = __ldg(p.block_table + static_cast<size_t>(it.b) * p.max_pages + (pi < last ? pi : last));
        y &= p.page_size - 1;
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
      ring.step();
      advance();
    }
  } else {
    // =========================================================================== scores, softmax, output
    // Lane l holds columns 2 (l % 4), + 1 of rows l / 4 and l / 4 + 8 of every 8 columns.  fp32 throughout, in the log2 domain; the
    // probabilities are rounded to bf16 for the second product (relative 2^-8 each), the sum that divides them is kept from
    // the unrounded ones.
    const int row = lane >> 2, col = (lane & 3) * 2, G = p.G;
    const int tok0 = row / G, tok1 = (row + 8) / G;        // tokens of this lane's rows within the tile
    const int head0 = row - tok0 * G, head1 = row + 8 - tok1 * G;
    const float scale_log2 = p.scale_log2;
    float* acc = reinterpret_cast<float*>(smem + S::kAcc);
    float2* ml = reinterpret_cast<float2*>(smem + S::kMl);
    // ldmatrix rows of this lane: K by (key, 16-byte piece), V by (key, 16-byte piece) too, transposed on the way
    const uint32_t k_row = (lane & 7) * 128, k_piece = lane >> 3, swz = lane & 7;
    const uint32_t v_row = (lane & 15) * 128, v_piece = lane >> 4;
    uint32_t before = 0;                                   // tiles of the items before
    bool ok = true;
    for (int i = 0; i < n_items; ++i) {
      const Item it = item(i);
      if (it.steps <= 0) continue;                         // (uniform over the CTA)
      const bool valid0 = tok0 < p.tpt && it.first + tok0 < it.n, valid1 = tok1 < p.tpt && it.first + tok1 < it.n;
      uint32_t qa[D / 16][4];
      {
        const uint32_t* q0 = reinterpret_cast<const uint32_t*>(p.q + (static_cast<size_t>(it.start + it.first + tok0) * p.Hq + it.g * G + head0) * D + col);
        const uint32_t* q1 = reinterpret_cast<const uint32_t*>(p.q + (static_cast<size_t>(it.start + it.first + tok1) * p.Hq + it.g * G + head1) * D + col);
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          qa[k][0] = valid0 ? __ldg(q0 + k * 8) : 0u;
          qa[k][1] = valid1 ? __ldg(q1 + k * 8) : 0u;
          qa[k][2] = valid0 ? __ldg(q0 + k * 8 + 4) : 0u;
          qa[k][3] = valid1 ? __ldg(q1 + k * 8 + 4) : 0u;
        }
      }
      float o[D / 8][4];
#pragma unroll
      for (int d = 0; d < D / 8; ++d) o[d][0] = o[d][1] = o[d][2] = o[d][3] = 0.f;
      float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;
      const int limit0 = it.L + it.first + tok0, limit1 = it.L + it.first + tok1;       // the last key a row sees
      for (int s = static_cast<int>((warp - before) & (kRowWarps - 1)); s < it.steps && ok; s += kRowWarps) {
        const uint32_t gs = before + s, slot = gs % S::kStages, par = (gs / S::kStages) & 1u;
        const uint32_t k_at = sbase + slot * S::kStage, v_at = k_at + S::kTile;
        const int key0 = it.key0 + s * kRowKeys;
        ok = mbar_wait_warp(full(slot), par, s_abort);
        if (!ok) break;
        float sc[kRowKeys / 8][4];
#pragma unroll
        for (int j = 0; j < kRowKeys / 8; ++j) {
          sc[j][0] = sc[j][1] = sc[j][2] = sc[j][3] = 0.f;
#pragma unroll
          for (int k = 0; k < D / 32; ++k) {               // 32 columns of 8 keys: two steps of 16
            uint32_t kb[4];
            load_matrices(kb, k_at + (k >> 1) * S::kSlab + j * 1024 + k_row + ((((k & 1) * 4 + k_piece) ^ swz) << 4));
            mma_16x8x16(sc[j], qa[2 * k], kb[0], kb[1]);
            mma_16x8x16(sc[j], qa[2 * k + 1], kb[2], kb[3]);
          }
        }
        if (key0 + kRowKeys - 1 > it.L + it.first) {       // a tile that some row does not see whole
#pragma unroll
          for (int j = 0; j < kRowKeys / 8; ++j) {
            const int key = key0 + j * 8 + col;
            if (key > limit0) sc[j][0] = -INFINITY;
            if (key + 1 > limit0) sc[j][1] = -INFINITY;
            if (key > limit1) sc[j][2] = -INFINITY;
            if (key + 1 > limit1) sc[j][3] = -INFINITY;
          }
        }
        float t0 = -INFINITY, t1 = -INFINITY;
#pragma unroll
        for (int j = 0; j < kRowKeys / 8; ++j) {
          t0 = max3(t0, sc[j][0], sc[j][1]);
          t1 = max3(t1, sc[j][2], sc[j][3]);
        }
        const float n0 = fmaxf(m0, quad_max(t0) * scale_log2), n1 = fmaxf(m1, quad_max(t1) * scale_log2);      // scale > 0
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
        for (int j = 0; j < kRowKeys / 8; ++j) {
          const float p0 = fast_exp2(fmaf(sc[j][0], scale_log2, b0)), p1 = fast_exp2(fmaf(sc[j][1], scale_log2, b0));
          const float p2 = fast_exp2(fmaf(sc[j][2], scale_log2, b1)), p3 = fast_exp2(fmaf(sc[j][3], scale_log2, b1));
          l0 += p0 + p1;
          l1 += p2 + p3;
          pa[j >> 1][(j & 1) * 2] = pack_bf16(p0, p1);
          pa[j >> 1][(j & 1) * 2 + 1] = pack_bf16(p2, p3);
        }
        const int in_use = it.L + it.n - key0;             // keys of the tile that belong to the sequence
        if (in_use < kRowKeys) {
          // the rows of V past the sequence may hold anything, and 0 * garbage must not reach O
          for (int sl = 0; sl < S::kSlabs; ++sl)
            for (int j = in_use * 8 + lane; j < kRowKeys * 8; j += 32)
              *reinterpret_cast<uint4*>(smem + slot * S::kStage + S::kTile + sl * S::kSlab + j * 16) = make_uint4(0u, 0u, 0u, 0u);
          fence_proxy_async();                             // (the slot's next copy is ordered behind these stores)
          __syncwarp();
        }
#pragma unroll
        for (int d = 0; d < D / 16; ++d) {
#pragma unroll
          for (int k = 0; k < kRowKeys / 16; ++k) {        // 16 keys of 16 columns
            uint32_t vb[4];
            load_matrices_t(vb, v_at + (d >> 2) * S::kSlab + k * 2048 + v_row + ((((d & 3) * 2 + v_piece) ^ swz) << 4));
            mma_16x8x16(o[2 * d], pa[k], vb[0], vb[1]);
            mma_16x8x16(o[2 * d + 1], pa[k], vb[2], vb[3]);
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(empty(slot));
      }
      before += it.steps;

      // ---- the four warps' parts are joined: m* = max m_w, l* = sum l_w 2^(m_w - m*), out = sum o_w 2^(m_w - m*) / l*.  (After an abort
      // every warp still comes to the barriers.)
      l0 = quad_sum(l0);
      l1 = quad_sum(l1);
      if ((lane & 3) == 0) {
        ml[warp * kFewRows + row] = make_float2(m0, l0);
        ml[warp * kFewRows + row + 8] = make_float2(m1, l1);
      }
#pragma unroll
      for (int d = 0; d < D / 8; ++d) {
        *reinterpret_cast<float2*>(acc + (warp * kFewRows + row) * S::kAccRow + d * 8 + col) = make_float2(o[d][0], o[d][1]);
        *reinterpret_cast<float2*>(acc + (warp * kFewRows + row + 8) * S::kAccRow + d * 8 + col) = make_float2(o[d][2], o[d][3]);
      }
      asm volatile("bar.sync 1, %0;" ::"n"(32 * kRowWarps) : "memory");
      {
        const int r = tid >> 3, c = (tid & 7) * 4, tok = r / G, head = r - tok * G, token = it.first + tok;
        if (tok < p.tpt && token < it.n) {
          float2 part[kRowWarps];
          float m = -INFINITY, l = 0.f;
#pragma unroll
          for (int w = 0; w < kRowWarps; ++w) {
            part[w] = ml[w * kFewRows + r];
            m = fmaxf(m, part[w].x);
          }
          const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
          for (int w = 0; w < kRowWarps; ++w) {
            part[w].x = fast_exp2(part[w].x - base);
            l = fmaf(part[w].y, part[w].x, l);
          }
          const float inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);                   // a NaN sum stays one
#pragma unroll
          for (int e = 0; e < D; e += 32) {
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kRowWarps; ++w) {
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
      asm volatile("bar.sync 1, %0;" ::"n"(32 * kRowWarps) : "memory");
    }
  }
  __syncthreads();
  if (*s_abort) {
    if (tid == 0) report_status(p.status, EAGLE_ERR_TIMEOUT);
    let_work_land();
  }
}

template <int D>
cudaError_t launch(const ChunkParams& p, cudaStream_t stream) {
  CUtensorMap mk, mv;
  const bool paged = p.block_table != nullptr;
  const int box_rows = paged && p.page_size < kRowKeys ? p.page_size : kRowKeys;
  const long long n1 = paged ? p.page_size : (p.capacity > 0 ? p.capacity : 1);
  const long long n2 = paged ? static_cast<long long>(p.num_pages) * p.Hkv : static_cast<long long>(p.B) * p.Hkv;
  if (!map_bf16_3d(&mk, p.k, D, n1, n2, 64, box_rows, 1) || !map_bf16_3d(&mv, p.v, D, n1, n2, 64, box_rows, 1)) return cudaErrorInvalidValue;
  BehindLaunch at(p.num_workers, kRowThreads, RowSmem<D>::kBytes, stream);
  auto kernel = p.stall_after_tiles >= 0 ? (paged ? chunk_rows_kernel<D, true, true> : chunk_rows_kernel<D, false, true>)
                                         : (paged ? chunk_rows_kernel<D, true, false> : chunk_rows_kernel<D, false, false>);
  return cudaLaunchKernelEx(&at.config, kernel, p, mk, mv);
}

template <int D>
cudaError_t prepare() {
  for (auto kernel : {chunk_rows_kernel<D, false, false>, chunk_rows_kernel<D, true, false>, chunk_rows_kernel<D, false, true>, chunk_rows_kernel<D, true, true>}) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, RowSmem<D>::kBytes);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace

cudaError_t chunk_rows_prepare(int head_dim) { return head_dim == 128 ? prepare<128>() : prepare<64>(); }
cudaError_t launch_chunk_rows(const ChunkParams& p, cudaStream_t stream) { return p.D == 128 ? launch<128>(p, stream) : launch<64>(p, stream); }

}  // namespace eagle
