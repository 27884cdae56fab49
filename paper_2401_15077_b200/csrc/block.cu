// Rotary positions of new tokens, fused with the write of their keys and values into a cache of e4m3 codes with a scale for each block of
// slots and KV head.
//
// The scale of a block is the least power of two 2^e with max |x| <= 448 * 2^e over what goes into it (rotated keys, values), so all new
// tokens of a block are seen before the first of them is stored: one warp takes a head's part of a block (of a whole tree in the tree
// form, whose blocks share a scale), reads its rows twice, once for the maximum and once for the codes, and finds the second time in L1 or
// L2.  Where older slots lie in the block and the scale has grown, the same warp stores their codes again.  So nothing is shared between warps but
// the sines and cosines, which a CTA computes once for the tokens of its block.  Queries are turned by CTAs of their own, a warp per
// token, behind those in the same launch.
//
// A CTA of the chunk form looks for the blocks that begin (for this call) within `span` rows: with long chunks a span is a block, with few
// tokens it is a row, so that every token has CTAs of its own.
#include "block.cuh"

namespace eagle {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int D = 128, kLanes = D / 16;          // lanes of a head's row, each with two 16-byte vectors (those of eight pairs in halves)
constexpr int kRowsAtOnce = 32 / kLanes;
constexpr int kMaxBlock = 128;                   // rows of a block, and more than a tree's nodes
constexpr int kMaxTouched = kMaxTree / 16 + 1;   // blocks that a tree's slots can lie in

// 2^e, the least e in [-40, 120] with a <= 448 * 2^e = 1.75 * 2^(8 + e).
__device__ __forceinline__ float scale_for(float a) {
  const uint32_t u = __float_as_uint(a);
  const int e = static_cast<int>(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  return __uint_as_float(static_cast<uint32_t>(min(max(e, -40), 120) + 127) << 23);
}
__device__ __forceinline__ float finite_magnitude(float x) {
  const float a = fabsf(x);
  return a < INFINITY ? a : 0.f;                 // (NaN: 0)
}
// Values of sixteen codes.
__device__ __forceinline__ void decode(const uint4& c, float* f) {
  const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(i & 1 ? w[i >> 1] >> 16 : w[i >> 1] & 0xffffu), __NV_E4M3);
    const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&h));
    f[2 * i] = v.x;
    f[2 * i + 1] = v.y;
  }
}

template <bool INTERLEAVED>
__device__ __forceinline__ void rotate(float (&x)[8], float (&y)[8], const float2* cs) {
  if constexpr (INTERLEAVED) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float x0 = x[2 * e], x1 = x[2 * e + 1], y0 = y[2 * e], y1 = y[2 * e + 1];
      const float2 c = cs[e], d = cs[4 + e];
      x[2 * e] = x0 * c.x - x1 * c.y;
      x[2 * e + 1] = x1 * c.x + x0 * c.y;
      y[2 * e] = y0 * d.x - y1 * d.y;
      y[2 * e + 1] = y1 * d.x + y0 * d.y;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float x0 = x[e], y0 = y[e];
      const float2 c = cs[e];
      x[e] = x0 * c.x - y0 * c.y;
      y[e] = y0 * c.x + x0 * c.y;
    }
  }
}
__device__ __forceinline__ float2 turn_by(const RopeParams& p, int pos, int m) {
  double turns = static_cast<double>(pos) * (p.freqs[m] * 0.15915494309189535);      // 1 / (2 pi)
  turns -= rint(turns);
  float sn, cs;
  sincospif(2.0f * static_cast<float>(turns), &sn, &cs);
  return make_float2(cs * p.amplitude, sn * p.amplitude);
}

// A tree's validity, and the depth of node `lane` and of node `lane + 32` (a warp; top-level nodes have depth 1).
struct TreeOf {
  int n, L;
  bool bad, no_room;
  int depth[2];
};
__device__ __forceinline__ TreeOf tree_of(const RopeParams& p, int b, int lane) {
  TreeOf t;
  const int32_t* parent = p.tree_parent + (p.shared_tree ? 0 : static_cast<size_t>(b) * p.T);
  t.n = p.tree_sizes ? p.tree_sizes[p.shared_tree ? 0 : b] : p.T;
  t.L = p.seq_lens[b];
  const bool size_ok = t.n >= 0 && t.n <= p.T;
  int up[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) up[i] = size_ok && lane + 32 * i < t.n ? parent[lane + 32 * i] : -1;
  t.bad = __any_sync(0xffffffffu, !size_ok || up[0] < -1 || up[0] >= lane || up[1] < -1 || up[1] >= lane + 32);
  t.no_room = t.n > 0 && (t.L < 0 || static_cast<long long>(t.L) + t.n > p.capacity);
  if (!size_ok) t.n = -1;
  t.depth[0] = t.depth[1] = 1;
  if (!t.bad) {
    // all paths go up together: a step adds 1 and moves on, until every node has come to the context
    int at[2] = {up[0], up[1]};
    while (__any_sync(0xffffffffu, at[0] >= 0 || at[1] >= 0)) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int lo = __shfl_sync(0xffffffffu, up[0], at[i] & 31), hi = __shfl_sync(0xffffffffu, up[1], at[i] & 31);
        if (at[i] >= 0) {
          ++t.depth[i];
          at[i] = at[i] < 32 ? lo : hi;
        }
      }
    }
  }
  return t;
}

// What a CTA stores at once: `n` new rows of one sequence, which share a scale per head.
struct Rows {
  int first;                     // row of q, k and v
  int n;
  int old;                       // slots of the first block that are older
  int blocks;                    // blocks they lie in
};

enum Form { kChunks, kTrees, kSingles };

template <Form FORM, bool INTERLEAVED>
__global__ void __launch_bounds__(kThreads) block_kernel(BlockParams p) {
  constexpr bool TREE = FORM == kTrees;
  // sines and cosines of [rows or depths], the eight pairs of a lane in four 16-byte pieces [4][kLanes] (eight lanes of a read are then neighbours);
  // for queries [warps][R / 2]
  extern __shared__ __align__(16) float2 s_cs[];
  __shared__ long long s_row[kMaxBlock];                   // cache row (KV head 0) of each new row, -1: not stored
  __shared__ long long s_scale[kMaxTouched];               // each block's place among the scales (KV head 0), -1: none
  __shared__ int s_pos[kMaxBlock];                         // position of a row; in the tree form, of a depth
  __shared__ int s_turn[kMaxBlock];                        // place of a row in the table
  __shared__ float s_top[kWarps];
  const RopeParams& r = p.r;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, half = r.R / 2;
  const int u = lane & (kLanes - 1), sub = lane / kLanes;
  const bool turn = 16 * u < r.R;                          // this lane's two vectors hold eight whole pairs
  const int va = !turn ? 16 * u : (INTERLEAVED ? 16 * u : 8 * u);
  const int vb = !turn ? 16 * u + 8 : (INTERLEAVED ? 16 * u + 8 : half + 8 * u);

  if (!TREE && blockIdx.x == 0) {                          // the list of starts has to ascend within the tensor
    int bad = 0;
    for (int i = threadIdx.x; i <= r.B; i += kThreads) {
      const int s = r.token_start[i];
      if (s < 0 || s > r.N || (i < r.B && r.token_start[i + 1] < s)) bad = 1;
    }
    if (bad) report_status(r.status, EAGLE_ERR_SEQ);
  }

  if (static_cast<int>(blockIdx.x) >= p.store_ctas) {
    // ============================================================================================ queries: a warp per token and some heads
    const long long job = static_cast<long long>(blockIdx.x - p.store_ctas) * kWarps + warp;
    const long long token_of = job / r.head_chunks;
    const int h_lo = static_cast<int>(job - token_of * r.head_chunks) * r.heads_per_warp, h_hi = min(r.Hq, h_lo + r.heads_per_warp);
    if (token_of >= (TREE ? static_cast<long long>(r.B) * r.T : r.N)) return;
    const int t = static_cast<int>(token_of);
    const __nv_bfloat16* row = r.q + t * r.q_stride;
    struct Unit {
      uint4 a, b;
    } now, then;
    auto fetch = [&](Unit& x, int h) __attribute__((always_inline)) {
      if (h >= h_hi) return;
      x.a = *reinterpret_cast<const uint4*>(row + h * D + va);
      x.b = *reinterpret_cast<const uint4*>(row + h * D + vb);
    };
    int h = h_lo + sub;
    fetch(now, h);                                         // sets out before anything is known about the token
    int pos = 0;
    bool zero;
    if constexpr (TREE) {
      const int seq = t / r.T, i = t - seq * r.T;
      const TreeOf tree = tree_of(r, seq, lane);
      if (tree.n >= 0 && i >= tree.n) return;
      zero = tree.bad || tree.no_room;
      const int d0 = __shfl_sync(0xffffffffu, tree.depth[0], i & 31), d1 = __shfl_sync(0xffffffffu, tree.depth[1], i & 31);
      pos = tree.L + (i < 32 ? d0 : d1) - 1;
    } else {
      const int seq = owner_of(r.token_start, r.B, t, lane);
      const int s = r.token_start[seq], e = r.token_start[seq + 1], L = r.seq_lens[seq];
      if (s < 0 || s > t || t >= e || e > r.N) return;
      zero = L < 0 || static_cast<long long>(L) + (e - s) > r.capacity;
      if (!zero) pos = r.positions ? r.positions[t] : L + (t - s);
    }
    float2* mine = s_cs + warp * half;
    for (int m = lane; m < half; m += 32) mine[m] = turn_by(r, pos, m);
    __syncwarp();
    float2 cs[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) cs[e] = turn ? mine[8 * u + e] : make_float2(1.f, 0.f);
    auto work = [&](const Unit& in, int head) __attribute__((always_inline)) {
      if (head >= h_hi) return;
      uint4 a = in.a, b = in.b;
      if (turn) {
        float x[8], y[8];
        widen(a, x);
        widen(b, y);
        rotate<INTERLEAVED>(x, y, cs);
        a = narrow(x);
        b = narrow(y);
      }
      if (zero) a = b = make_uint4(0u, 0u, 0u, 0u);
      __nv_bfloat16* dst = r.q_out + (static_cast<long long>(t) * r.Hq + head) * D;
      *reinterpret_cast<uint4*>(dst + va) = a;
      *reinterpret_cast<uint4*>(dst + vb) = b;
    };
    for (; h < h_hi; h += 2 * kRowsAtOnce) {
      fetch(then, h + kRowsAtOnce);
      work(now, h);
      fetch(now, h + 2 * kRowsAtOnce);
      work(then, h + kRowsAtOnce);
    }
    return;
  }

  // Cache row and scale of a slot (KV head 0).
  auto scale_at = [&](int b, int slot) -> long long {
    if (!r.block_table) return static_cast<long long>(b) * r.Hkv * p.head_blocks + (slot >> p.block_shift);
    const int page = r.block_table[static_cast<size_t>(b) * r.max_pages + (slot >> r.page_shift)];
    if (page < 0 || page >= r.num_pages) return -1;
    return static_cast<long long>(page) * r.Hkv * p.head_blocks + ((slot & (r.page_size - 1)) >> p.block_shift);
  };
  // Codes of an older slot again, by a scale that has grown (16 of a lane).  The products have 28 bits: rounded to fp32, one next to a middle between two
  // codes would be taken for the middle.  So they are cut off, with the last bit set where something is missing, and rounded once.
  auto store_again = [&](uint8_t* at, float held, float scale) {
    const float ratio = held * __uint_as_float(0x7f000000u - __float_as_uint(scale));      // 1 / 2^e
    float f[16];
    decode(*reinterpret_cast<const uint4*>(at), f);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float cut = __fmul_rz(f[e], ratio);
      f[e] = __uint_as_float(__float_as_uint(cut) | (fmaf(f[e], ratio, -cut) != 0.f ? 1u : 0u));
    }
    const uint2 lo = codes(f, 1.f, 1.f), hi = codes(f + 8, 1.f, 1.f);
    *reinterpret_cast<uint4*>(at) = make_uint4(lo.x, lo.y, hi.x, hi.y);
  };

  if constexpr (FORM == kSingles) {
    // ============================================================================== keys and values of single tokens: a warp per row and some heads
    const long long job = static_cast<long long>(blockIdx.x) * kWarps + warp, token_of = job / p.store_groups;
    const int h_lo = static_cast<int>(job - token_of * p.store_groups) * p.store_heads, h_hi = min(2 * r.Hkv, h_lo + p.store_heads);
    if (token_of >= r.N) return;
    const int t = static_cast<int>(token_of), seq = owner_of(r.token_start, r.B, t, lane);
    const int s = r.token_start[seq], e = r.token_start[seq + 1], L = r.seq_lens[seq];
    if (s < 0 || s > t || t >= e || e > r.N) return;
    if (L < 0 || static_cast<long long>(L) + (e - s) > r.capacity) {
      if (lane == 0) report_status(r.status, EAGLE_ERR_SEQ);
      return;
    }
    const int slot = L + (t - s), in_block = slot & (p.block_size - 1), n = min(e - t, p.block_size - in_block);
    if (t != s && in_block != 0) return;                   // its block begins with an earlier row
    const long long row = rope_row(r, seq, slot), at = scale_at(seq, slot);
    if (row < 0) return;
    float2* mine = s_cs + warp * half;
    float2 cs[8];
    auto angles = [&](int i) {
      __syncwarp();
      for (int m = lane; m < half; m += 32) mine[m] = turn_by(r, r.positions ? r.positions[t + i] : slot + i, m);
      __syncwarp();
#pragma unroll
      for (int x = 0; x < 8; ++x) cs[x] = turn ? mine[8 * u + x] : make_float2(1.f, 0.f);
    };
    angles(0);
    for (int h0 = h_lo; h0 < h_hi; h0 += kRowsAtOnce) {
      const int head = h0 + sub;
      const bool live = head < h_hi, is_v = head >= r.Hkv;
      const int g = !live ? 0 : (is_v ? head - r.Hkv : head);
      const long long stride = is_v ? r.v_stride : r.k_stride;
      const __nv_bfloat16* src = (is_v ? r.v : r.k) + t * stride + g * D;
      uint8_t* cache = static_cast<uint8_t*>(is_v ? r.v_cache : r.k_cache) + (row + g * r.head_rows) * D;
      float* scale_to = (is_v ? p.v_scale : p.k_scale) + at + g * p.head_blocks;
      const float held = in_block > 0 && live ? *scale_to : 0.f;
      float x[8], y[8];
      auto fetch = [&](int i) {
        if (n > 1) angles(i);
        widen(*reinterpret_cast<const uint4*>(src + i * stride + va), x);
        widen(*reinterpret_cast<const uint4*>(src + i * stride + vb), y);
        if (turn && !is_v) rotate<INTERLEAVED>(x, y, cs);
      };
      float top = 0.f;
      for (int i = 0; i < n; ++i) {
        fetch(i);
#pragma unroll
        for (int k = 0; k < 8; ++k) top = fmaxf(top, fmaxf(finite_magnitude(x[k]), finite_magnitude(y[k])));
      }
#pragma unroll
      for (int o = 1; o < kLanes; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      const float need = scale_for(top);
      const bool grown = held > 0.f && need > held;
      const float scale = held > 0.f && !grown ? held : need;
      if (grown)
        for (int i = 1; i <= in_block; ++i) store_again(cache - i * D + 16 * u, held, scale);
      float inv;
      asm("rcp.approx.f32 %0, %1;" : "=f"(inv) : "f"(scale));
      for (int i = 0; i < n; ++i) {
        if (n > 1) fetch(i);
        if (!live) continue;
        *reinterpret_cast<uint2*>(cache + i * D + va) = codes(x, scale, inv);
        *reinterpret_cast<uint2*>(cache + i * D + vb) = codes(y, scale, inv);
      }
      if (live && u == 0) *scale_to = scale;
    }
    return;
  }

  // ================================================================================================ keys and values
  const int job = blockIdx.x / p.store_groups, h_lo = (blockIdx.x - job * p.store_groups) * p.store_heads;
  const int warps = kWarps / p.store_heads, part = warp % warps, head_of = h_lo + warp / warps;      // warps per head, this one's part and head
  const bool any_keys = h_lo < r.Hkv, some_head = head_of < 2 * r.Hkv;
  const int row0 = part * kRowsAtOnce + sub, step = warps * kRowsAtOnce;

  // One head's rows: the maximum, the scale, the codes.  (All warps of the CTA.)
  auto store_head = [&](const Rows& rows) {
    const int head = some_head ? head_of : 0;
    const bool is_v = head >= r.Hkv;
    const int g = is_v ? head - r.Hkv : head;
    const long long stride = is_v ? r.v_stride : r.k_stride;
    const __nv_bfloat16* src = (is_v ? r.v : r.k) + rows.first * stride + g * D;
    float* scales = is_v ? p.v_scale : p.k_scale;
    uint8_t* cache = static_cast<uint8_t*>(is_v ? r.v_cache : r.k_cache) + g * r.head_rows * D;
    auto fetch = [&](int i, float (&x)[8], float (&y)[8]) __attribute__((always_inline)) {
      const uint4 a = *reinterpret_cast<const uint4*>(src + i * stride + va), b = *reinterpret_cast<const uint4*>(src + i * stride + vb);
      widen(a, x);
      widen(b, y);
      if (turn && !is_v) {
        float2 cs[8];
        const float4* at = reinterpret_cast<const float4*>(s_cs) + s_turn[i] * (4 * kLanes) + u;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float4 c = at[e * kLanes];
          cs[2 * e] = make_float2(c.x, c.y);
          cs[2 * e + 1] = make_float2(c.z, c.w);
        }
        rotate<INTERLEAVED>(x, y, cs);
      }
    };
    const long long first_scale = s_scale[0];
    float held = 0.f;
    if (rows.old > 0 && first_scale >= 0) held = scales[first_scale + g * p.head_blocks];
    float top = 0.f;
    if (some_head) {
#pragma unroll 4
      for (int i = row0; i < rows.n; i += step) {
        float x[8], y[8];
        fetch(i, x, y);
#pragma unroll
        for (int e = 0; e < 8; ++e) top = fmaxf(top, fmaxf(finite_magnitude(x[e]), finite_magnitude(y[e])));
      }
    }
    top = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top)));      // (magnitudes order as their bits do)
    if (warps > 1) {
      if (lane == 0) s_top[warp] = top;
      __syncthreads();                                     // (the older scale has been read by all, too)
      for (int w = 0; w < warps; ++w) top = fmaxf(top, s_top[warp - part + w]);
    }
    if (!some_head) return;
    const float need = scale_for(top);
    const bool grown = held > 0.f && need > held;
    const float scale = held > 0.f && !grown ? held : need;
    if (grown) {
      uint8_t* old = cache + (s_row[0] - rows.old) * D;
      for (int i = row0; i < rows.old; i += step) store_again(old + i * D + 16 * u, held, scale);
    }
    float inv;
    asm("rcp.approx.f32 %0, %1;" : "=f"(inv) : "f"(scale));
#pragma unroll 2
    for (int i = row0; i < rows.n; i += step) {
      const long long to = s_row[i];
      if (to < 0) continue;
      float x[8], y[8];
      fetch(i, x, y);
      *reinterpret_cast<uint2*>(cache + to * D + va) = codes(x, scale, inv);
      *reinterpret_cast<uint2*>(cache + to * D + vb) = codes(y, scale, inv);
    }
    if (part == 0 && lane < rows.blocks && s_scale[lane] >= 0) scales[s_scale[lane] + g * p.head_blocks] = scale;
  };
  auto store = [&](const Rows& rows, int angles) {         // angles: positions in s_pos
    if (any_keys) {
      for (int i = threadIdx.x; i < angles * half; i += kThreads) {
        const int at = i / half, m = i - at * half;
        s_cs[((at * 4 + ((m >> 1) & 3)) * kLanes + (m >> 3)) * 2 + (m & 1)] = turn_by(r, s_pos[at], m);
      }
    }
    __syncthreads();
    store_head(rows);
  };

  if constexpr (TREE) {
    const int b = job;
    const TreeOf tree = tree_of(r, b, lane);
    if (tree.bad || tree.no_room) {
      if (threadIdx.x == 0) report_status(r.status, tree.bad ? EAGLE_ERR_TREE : EAGLE_ERR_SEQ);
      return;
    }
    if (tree.n == 0) return;
    const int blocks = ((tree.L + tree.n - 1) >> p.block_shift) - (tree.L >> p.block_shift) + 1;
    if (warp == 0) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (lane + 32 * i < tree.n) {
          s_row[lane + 32 * i] = rope_row(r, b, tree.L + lane + 32 * i);
          s_turn[lane + 32 * i] = tree.depth[i] - 1;
          s_pos[lane + 32 * i] = tree.L + lane + 32 * i;
        }
    } else if (warp == 1 && lane < blocks) {
      s_scale[lane] = scale_at(b, ((tree.L >> p.block_shift) + lane) << p.block_shift);
    }
    const int deepest = __reduce_max_sync(0xffffffffu, max(lane < tree.n ? tree.depth[0] : 0, lane + 32 < tree.n ? tree.depth[1] : 0));
    __syncthreads();
    store(Rows{b * r.T, tree.n, tree.L & (p.block_size - 1), blocks}, deepest);
  } else {
    const int end = min(r.N, (job + 1) * p.span);
    int t = job * p.span;
    int seq = owner_of(r.token_start, r.B, t, lane);
    while (t < end) {
      const int s = r.token_start[seq], e = r.token_start[seq + 1];
      if (t >= e && seq + 1 < r.B) {                       // (past a sequence, perhaps an empty one)
        ++seq;
        continue;
      }
      if (t < s || t >= e || s < 0 || e > r.N) {           // in no sequence
        ++t;
        continue;
      }
      const int L = r.seq_lens[seq];
      if (L < 0 || static_cast<long long>(L) + (e - s) > r.capacity) {
        if (threadIdx.x == 0) report_status(r.status, EAGLE_ERR_SEQ);
        t = e;
        continue;
      }
      const int slot = L + (t - s), in_block = slot & (p.block_size - 1), rest = min(e - t, p.block_size - in_block);
      if (t != s && in_block != 0) {                       // its block begins in another span
        t += rest;
        continue;
      }
      __syncthreads();                                     // (the tables of the rows before have been read)
      const long long row = rope_row(r, seq, slot);
      for (int i = threadIdx.x; i < rest; i += kThreads) {
        s_row[i] = row < 0 ? -1 : row + i;
        s_turn[i] = i;
        s_pos[i] = r.positions ? r.positions[t + i] : slot + i;
      }
      if (threadIdx.x == 0) s_scale[0] = scale_at(seq, slot);
      __syncthreads();
      if (row >= 0) store(Rows{t, rest, in_block, 1}, rest);      // (uniform: a block lies in one page)
      t += rest;
    }
  }
}

template <Form FORM>
cudaError_t launch(const BlockParams& p, unsigned blocks, size_t smem, cudaStream_t stream) {
  auto kernel = p.r.interleaved ? block_kernel<FORM, true> : block_kernel<FORM, false>;
  if (smem > 48 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
    if (e != cudaSuccess) return e;
  }
  kernel<<<blocks, kThreads, smem, stream>>>(p);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_block(const BlockParams& p_in, bool tree, int sm_count, cudaStream_t stream) {
  BlockParams p = p_in;
  RopeParams& r = p.r;
  const long long tokens = tree ? static_cast<long long>(r.B) * r.T : r.N;
  // keys and values: sixteen rows and more to a warp, up to four warps per head, eight warps to a CTA (64 trees of 16 to 64 nodes: 43 us with
  // a warp per head); the rows of a CTA are a block's, or fewer while two CTAs per SM are not there
  const long long each = tree ? r.T : (r.N + static_cast<long long>(r.B) - 1) / r.B, held = each < p.block_size || tree ? each : p.block_size;
  p.store_heads = held >= 64 ? 2 : (held >= 32 ? 4 : kWarps);
  p.store_groups = (2 * r.Hkv + p.store_heads - 1) / p.store_heads;
  p.span = p.block_size;
  while (!tree && p.span > 1 && (r.N + p.span - 1) / p.span * static_cast<long long>(p.store_groups) < 2 * sm_count) p.span /= 2;
  long long stores = (tree ? r.B : (r.N + static_cast<long long>(p.span) - 1) / p.span) * p.store_groups;
  const bool single = !tree && r.N <= r.B;
  if (single) {
    // as for the queries below: a row's heads go to several warps until there are sixteen warps per SM, or a warp has one step of heads
    int parts = 1;
    while (tokens * parts < 16ll * sm_count && 2 * r.Hkv > parts * kRowsAtOnce) parts *= 2;
    p.store_heads = ((2 * r.Hkv + parts - 1) / parts + kRowsAtOnce - 1) / kRowsAtOnce * kRowsAtOnce;
    p.store_groups = (2 * r.Hkv + p.store_heads - 1) / p.store_heads;
    stores = (tokens * p.store_groups + kWarps - 1) / kWarps;
  }
  // queries: a token's heads are split over several warps until there are sixteen warps per SM, or a warp has one step of heads
  int chunks = 1;
  while (tokens * chunks < 16ll * sm_count && r.Hq > chunks * kRowsAtOnce) chunks *= 2;
  r.heads_per_warp = r.Hq > 0 ? ((r.Hq + chunks - 1) / chunks + kRowsAtOnce - 1) / kRowsAtOnce * kRowsAtOnce : 1;
  r.head_chunks = r.Hq > 0 ? (r.Hq + r.heads_per_warp - 1) / r.heads_per_warp : 0;
  const long long turns = (tokens * r.head_chunks + kWarps - 1) / kWarps;
  if (stores + turns > 0x7fffffffll) return cudaErrorInvalidValue;
  p.store_ctas = static_cast<int>(stores);
  const long long most = tree ? r.T : (single ? 0 : (p.block_size < r.N ? p.block_size : r.N));
  const size_t smem = sizeof(float2) * (D / 2) * static_cast<size_t>(most > kWarps ? most : kWarps);
  const unsigned blocks = static_cast<unsigned>(stores + turns);
  const cudaError_t e = tree ? launch<kTrees>(p, blocks, smem, stream)
                        : (single ? launch<kSingles>(p, blocks, smem, stream) : launch<kChunks>(p, blocks, smem, stream));
  if (e != cudaSuccess) return e;
  count_launch();
  return cudaSuccess;
}

}  // namespace eagle
