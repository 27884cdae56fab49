// Rotary positions of new tokens, fused with the write of their keys and values into the cache.
//
// Token t of sequence b has position pos and cache slot L_b + i (i: its place among the sequence's new tokens).  Pair m of the
// rotated part of a head turns by the angle pos * freqs[m]:
//     (x, y) -> amplitude * (x cos - y sin, y cos + x sin),
// x and y half a rotated part apart (m, m + R/2) or next to one another (2m, 2m + 1).  Queries go to a dense tensor, keys to
// the cache, values to the cache as they are; an fp8 cache takes e4m3 codes of x / scale.
//
// The angle is taken in turns: pos * (freqs[m] / 2 pi) in fp64, its whole turns dropped there, the rest rounded to fp32 (error
// 2^-25 of a turn at any position) for sincospi.
//
// A warp takes one token (or some of its heads, when there are few tokens) and needs no other warp: it finds the token's sequence,
// computes the token's sines and cosines, two pairs a lane, and shares them out so that a lane holds the eight pairs that its
// place in a head needs, for every head.  A unit of work is two 16-byte vectors of one head, the two that a rotation of eight
// pairs in halves needs; units of the heads to come are on their way while one is turned.  (With tokens spread over a CTA and the
// sines read from shared memory for each unit, those reads, four-way bank conflicts among them, cost as much as the loads.)
// The kernel moves (2 Hq + 2 Hkv + 2 Hkv) * D elements a token and is bound by HBM for long chunks, by launch and memory
// latency for short ones.  From a graph, 8192 tokens, 64 heads over 8, D = 128 (336 MB): 58 us, 5.8 TB/s of the 6.6 TB/s that a plain copy reaches;
// 64 trees of 16 to 64 nodes, 32 heads over 8 (64 MB, one round of CTAs): 17 us, 3.7 TB/s; 6900 tokens into e4m3 codes (164 MB): 38 us,
// 4.3 TB/s, where the conversions' registers leave no room for more loads (some spill already); one token: 3.3 to 4.2 us.  Measured and no better: three units
// in flight (spills: 64 us for the 8192 tokens), 32 or 64 warps per SM asked for below (18.6 and 19.5 us for the trees).
#include "rope.cuh"

namespace eagle {

namespace {

constexpr int kRopeThreads = 256;
constexpr int kRopeWarps = kRopeThreads / 32;

template <bool TREE, bool FP8, bool INTERLEAVED, int D>
__global__ void __launch_bounds__(kRopeThreads, 4) rope_kernel(RopeParams p) {
  __shared__ float2 s_cs[kRopeWarps][D / 2];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long job = static_cast<long long>(blockIdx.x) * kRopeWarps + warp;
  const int chunks = p.head_chunks, H = p.Hq + 2 * p.Hkv, tokens = TREE ? p.B * p.T : p.N;
  const long long token_of = job / chunks;
  const int h_lo = static_cast<int>(job - token_of * chunks) * p.heads_per_warp, h_hi = min(H, h_lo + p.heads_per_warp);

  if (!TREE && blockIdx.x == 0) {                          // the list of starts has to ascend within the tensor
    int bad = 0;
    for (int i = threadIdx.x; i <= p.B; i += kRopeThreads) {
      const int s = p.token_start[i];
      if (s < 0 || s > p.N || (i < p.B && p.token_start[i + 1] < s)) bad = 1;
    }
    if (bad) report_status(p.status, EAGLE_ERR_SEQ);
  }
  if (token_of >= tokens) return;
  const int t = static_cast<int>(token_of);

  // ---- units: lane `l` has place l % U in the heads l / U, l / U + 32 / U, ...
  constexpr int U = D / 16, kStep = 32 / U;
  const int u = lane & (U - 1), half = p.R / 2;
  const bool turn = 16 * u < p.R;                          // its two vectors hold eight whole pairs
  const int va = !turn ? 16 * u : (INTERLEAVED ? 16 * u : 8 * u);
  const int vb = !turn ? 16 * u + 8 : (INTERLEAVED ? 16 * u + 8 : half + 8 * u);
  const __nv_bfloat16 *q_row = p.q + t * p.q_stride, *k_row = p.k + t * p.k_stride, *v_row = p.v + t * p.v_stride;
  struct Unit {
    uint4 a, b;
    float scale;
  };
  auto fetch = [&](Unit& x, int h) __attribute__((always_inline)) {
    if (h >= h_hi) return;
    const __nv_bfloat16* s = h < p.Hq ? q_row + h * D : (h < p.Hq + p.Hkv ? k_row + (h - p.Hq) * D : v_row + (h - p.Hq - p.Hkv) * D);
    x.a = *reinterpret_cast<const uint4*>(s + va);
    x.b = *reinterpret_cast<const uint4*>(s + vb);
  };
  Unit now, then;
  int h = h_lo + lane / U;
  fetch(now, h);                                           // sets out before anything is known about the token

  // ---- the token: sequence, position, cache row; a token without a sequence is left alone
  int seq, pos = 0;
  bool zero = false;                                       // its sequence is refused: the queries become zeros
  long long row = -1;                                      // cache row of its slot (KV head 0), -1: not stored
  if constexpr (TREE) {
    seq = t / p.T;
    const int i = t - seq * p.T;
    const int32_t* parent = p.tree_parent + (p.shared_tree ? 0 : static_cast<size_t>(seq) * p.T);
    const int n = p.tree_sizes ? p.tree_sizes[p.shared_tree ? 0 : seq] : p.T, L = p.seq_lens[seq];
    const bool size_ok = n >= 0 && n <= p.T;
    const int p0 = size_ok && lane < n ? parent[lane] : -1, p1 = size_ok && lane + 32 < n ? parent[lane + 32] : -1;
    const bool bad = __any_sync(0xffffffffu, !size_ok || p0 < -1 || p0 >= lane || p1 < -1 || p1 >= lane + 32);
    const bool no_room = n > 0 && (L < 0 || static_cast<long long>(L) + n > p.capacity);
    if (lane == 0 && i == 0 && (bad || no_room)) report_status(p.status, bad ? EAGLE_ERR_TREE : EAGLE_ERR_SEQ);
    if (size_ok && i >= n) return;
    zero = bad || no_room;
    if (!zero) {
      int depth = 0;
      for (int m = i; m >= 0; ++depth) m = m < 32 ? __shfl_sync(0xffffffffu, p0, m) : __shfl_sync(0xffffffffu, p1, m - 32);
      pos = L + depth - 1;
      row = rope_row(p, seq, L + i);
    }
  } else {
    seq = owner_of(p.token_start, p.B, t, lane);
    const int s = p.token_start[seq], e = p.token_start[seq + 1], L = p.seq_lens[seq];
    if (s < 0 || s > t || t >= e || e > p.N) return;
    zero = L < 0 || static_cast<long long>(L) + (e - s) > p.capacity;
    if (zero && lane == 0) report_status(p.status, EAGLE_ERR_SEQ);
    if (!zero) {
      pos = p.positions ? p.positions[t] : L + (t - s);
      row = rope_row(p, seq, L + (t - s));
    }
  }

  // ---- sines and cosines, times the amplitude
  for (int m = lane; m < half; m += 32) {
    double turns = static_cast<double>(pos) * (p.freqs[m] * 0.15915494309189535);      // 1 / (2 pi)
    turns -= rint(turns);
    float sn, cs;
    sincospif(2.0f * static_cast<float>(turns), &sn, &cs);
    s_cs[warp][m] = make_float2(cs * p.amplitude, sn * p.amplitude);
  }
  __syncwarp();
  float cs[8], sn[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float2 c = turn ? s_cs[warp][8 * u + e] : make_float2(1.f, 0.f);
    cs[e] = c.x;
    sn[e] = c.y;
  }

  auto rotate = [&](float (&x)[8], float (&y)[8]) __attribute__((always_inline)) {
    if constexpr (INTERLEAVED) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x0 = x[2 * e], x1 = x[2 * e + 1], y0 = y[2 * e], y1 = y[2 * e + 1];
        x[2 * e] = x0 * cs[e] - x1 * sn[e];
        x[2 * e + 1] = x1 * cs[e] + x0 * sn[e];
        y[2 * e] = y0 * cs[4 + e] - y1 * sn[4 + e];
        y[2 * e + 1] = y1 * cs[4 + e] + y0 * sn[4 + e];
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x0 = x[e], y0 = y[e];
        x[e] = x0 * cs[e] - y0 * sn[e];
        y[e] = y0 * cs[e] + x0 * sn[e];
      }
    }
  };
  auto work = [&](const Unit& in, int head) __attribute__((always_inline)) {
    if (head >= h_hi) return;
    const bool is_q = head < p.Hq, is_v = head >= p.Hq + p.Hkv;
    const int g = is_v ? head - p.Hq - p.Hkv : head - p.Hq;
    if (FP8 && !is_q) {
      if (row < 0) return;
      uint8_t* dst = static_cast<uint8_t*>(is_v ? p.v_cache : p.k_cache) + (row + g * p.head_rows) * D;
      float x[8], y[8], inv;
      asm("rcp.approx.f32 %0, %1;" : "=f"(inv) : "f"(in.scale));
      widen(in.a, x);
      widen(in.b, y);
      if (turn && !is_v) rotate(x, y);
      *reinterpret_cast<uint2*>(dst + va) = codes(x, in.scale, inv);
      *reinterpret_cast<uint2*>(dst + vb) = codes(y, in.scale, inv);
      return;
    }
    uint4 out_a = in.a, out_b = in.b;
    if (turn && !is_v) {
      float x[8], y[8];
      widen(in.a, x);
      widen(in.b, y);
      rotate(x, y);
      out_a = narrow(x);
      out_b = narrow(y);
    }
    __nv_bfloat16* dst;
    if (is_q) {
      if (zero) out_a = out_b = make_uint4(0u, 0u, 0u, 0u);
      dst = p.q_out + (static_cast<long long>(t) * p.Hq + head) * D;
    } else {
      if (row < 0) return;
      dst = static_cast<__nv_bfloat16*>(is_v ? p.v_cache : p.k_cache) + (row + g * p.head_rows) * D;
    }
    *reinterpret_cast<uint4*>(dst + va) = out_a;
    *reinterpret_cast<uint4*>(dst + vb) = out_b;
  };
  // (the scales need the sequence, so they follow the first unit's vectors and travel with those after it)
  auto scale_of = [&](Unit& x, int h) __attribute__((always_inline)) {
    if constexpr (FP8) {
      if (h >= p.Hq && h < h_hi) x.scale = __ldg((h < p.Hq + p.Hkv ? p.k_scale - p.Hq : p.v_scale - p.Hq - p.Hkv) + static_cast<size_t>(seq) * p.Hkv + h);
    }
  };
  scale_of(now, h);
  // (two units in turn, not moved along: a move would wait for the loads that have just set out)
  for (; h < h_hi; h += 2 * kStep) {
    fetch(then, h + kStep);
    scale_of(then, h + kStep);
    work(now, h);
    fetch(now, h + 2 * kStep);
    scale_of(now, h + 2 * kStep);
    work(then, h + kStep);
  }
}

template <bool TREE, bool FP8, int D>
void launch_kernel(const RopeParams& p, unsigned blocks, cudaStream_t stream) {
  if (p.interleaved) rope_kernel<TREE, FP8, true, D><<<blocks, kRopeThreads, 0, stream>>>(p);
  else rope_kernel<TREE, FP8, false, D><<<blocks, kRopeThreads, 0, stream>>>(p);
}

}  // namespace

cudaError_t launch_rope(const RopeParams& p_in, bool tree, int sm_count, cudaStream_t stream) {
  RopeParams p = p_in;
  const int H = p.Hq + 2 * p.Hkv, step = 32 / (p.D / 16);
  const long long tokens = tree ? static_cast<long long>(p.B) * p.T : p.N;
  // few tokens: a token's heads are split over several warps (each computes the same sines again) until there are
  // sixteen warps per SM, or a warp has a single step of heads
  int chunks = 1;
  while (tokens * chunks < 16ll * sm_count && H > chunks * step) chunks *= 2;
  p.heads_per_warp = ((H + chunks - 1) / chunks + step - 1) / step * step;
  p.head_chunks = (H + p.heads_per_warp - 1) / p.heads_per_warp;
  const long long jobs = tokens * p.head_chunks;
  const unsigned blocks = static_cast<unsigned>((jobs + kRopeWarps - 1) / kRopeWarps);
  if (p.k_scale) {                                         // codes: head_dim 128 only
    if (tree) launch_kernel<true, true, 128>(p, blocks, stream);
    else launch_kernel<false, true, 128>(p, blocks, stream);
  } else if (p.D == 128) {
    if (tree) launch_kernel<true, false, 128>(p, blocks, stream);
    else launch_kernel<false, false, 128>(p, blocks, stream);
  } else {
    if (tree) launch_kernel<true, false, 64>(p, blocks, stream);
    else launch_kernel<false, false, 64>(p, blocks, stream);
  }
  count_launch();
  return cudaGetLastError();
}

}  // namespace eagle
