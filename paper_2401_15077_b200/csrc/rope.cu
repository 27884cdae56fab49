// Rotary positions of new tokens, fused with the write of their keys and values into the cache.
//
// Token t of sequence b has position pos and cache slot L_b + i (i: its place among the sequence's new tokens).  Pair m of the
// rotated part of a head turns by the angle pos * freqs[m]:
//     (x, y) -> amplitude * (x cos - y sin, y cos + x sin),
// x and y half a rotated part apart (m, m + R/2) or next to one another (2m, 2m + 1).  Queries go to a dense tensor, keys to
// the cache, values to the cache as they are; an fp8 cache takes e4m3 codes of x / scale.
//
// The angle is taken in turns: pos * (freqs[m] / 2 pi) in fp64, its whole turns dropped there, the rest rounded to fp32 (error
// 2^-25 of a turn at any position) for sincospi.  It depends on the token and the pair only: a CTA takes a few tokens, computes
// their sines and cosines once into shared memory and uses them for every head.
//
// A unit of work is two 16-byte vectors of one head of one token, the two that a rotation of eight pairs in halves needs; a
// thread keeps its place in the head and walks over (token, head), two units in flight.  The kernel moves
// (2 Hq + 2 Hkv + 2 Hkv) * D elements a token and is bound by HBM for long chunks, by launch and memory latency for short ones.
#include <cuda_fp8.h>

#include "rope.cuh"

namespace eagle {

namespace {

constexpr int kRopeThreads = 256;
constexpr int kRopeTokens = 4;         // tokens per CTA

struct Vec2 {
  uint4 a, b;
};

__device__ __forceinline__ void widen(const uint4& v, float* f) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(w[i] << 16);
    f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ uint4 narrow(const float* f) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    __nv_bfloat162 v = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
    w[i] = *reinterpret_cast<uint32_t*>(&v);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// eight e4m3 codes (round to nearest even, magnitudes above 448 become 448, NaN stays NaN)
__device__ __forceinline__ uint2 codes(const float* f, float scale) {
  uint32_t w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float2 lo = make_float2(__fdiv_rn(f[4 * i], scale), __fdiv_rn(f[4 * i + 1], scale));
    const float2 hi = make_float2(__fdiv_rn(f[4 * i + 2], scale), __fdiv_rn(f[4 * i + 3], scale));
    w[i] = __nv_cvt_float2_to_fp8x2(lo, __NV_SATFINITE, __NV_E4M3) | (static_cast<uint32_t>(__nv_cvt_float2_to_fp8x2(hi, __NV_SATFINITE, __NV_E4M3)) << 16);
  }
  return make_uint2(w[0], w[1]);
}

// The sequence of packed token t: the last one that starts at or before it (a warp, 32 probes a round).
__device__ __forceinline__ int owner_of(const int32_t* start, int B, int t, int lane) {
  int lo = 0, n = B;
  while (n > 1) {
    const int step = (n + 31) >> 5, at = lane * step;
    const bool le = at < n && (lane == 0 || start[lo + at] <= t);
    const int last = 31 - __clz(__ballot_sync(0xffffffffu, le));
    lo += last * step;
    n = n - last * step < step ? n - last * step : step;
  }
  return lo;
}

template <bool TREE, bool FP8>
__global__ void __launch_bounds__(kRopeThreads) rope_kernel(RopeParams p) {
  __shared__ float2 s_cs[kRopeTokens][64];               // (cos, sin) of every pair of every token of the CTA
  __shared__ long long s_row[kRopeTokens];               // first cache row of the token's slot (KV head 0), -1: not stored
  __shared__ int s_seq[kRopeTokens], s_pos[kRopeTokens]; // sequence (-1: nothing to do), position
  __shared__ int s_zero[kRopeTokens];                    // its sequence is refused: the queries become zeros
  __shared__ int s_parent[kMaxTree];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  int t0;                                                // first token (row of q, k, v) of this CTA
  int n_tok = kRopeTokens;

  if constexpr (TREE) {
    const int groups = (p.T + kRopeTokens - 1) / kRopeTokens;
    const int b = blockIdx.x / groups, i0 = (blockIdx.x - b * groups) * kRopeTokens;
    t0 = b * p.T + i0;
    const int32_t* parent = p.tree_parent + (p.shared_tree ? 0 : static_cast<size_t>(b) * p.T);
    const int n = p.tree_sizes ? p.tree_sizes[p.shared_tree ? 0 : b] : p.T;
    const int L = p.seq_lens[b];
    const bool size_ok = n >= 0 && n <= p.T;
    int bad = !size_ok;
    if (size_ok && tid < n) {
      const int m = parent[tid];
      s_parent[tid] = m;
      bad = m < -1 || m >= tid;
    }
    bad = __syncthreads_or(bad);
    const bool no_room = L < 0 || static_cast<long long>(L) + n > p.capacity;
    if (tid == 0 && i0 == 0 && (bad || (no_room && n > 0))) report_status(p.status, bad ? EAGLE_ERR_TREE : EAGLE_ERR_SEQ);
    if (tid < kRopeTokens) {
      const int i = i0 + tid, nodes = size_ok ? n : p.T;
      const bool here = i < nodes && i < p.T, refused = bad || no_room;
      int depth = 0;
      if (here && !refused)
        for (int m = i; m >= 0; m = s_parent[m]) ++depth;
      s_seq[tid] = here ? b : -1;
      s_zero[tid] = refused;
      s_pos[tid] = L + depth - 1;
      s_row[tid] = here && !refused ? rope_row(p, b, L + i) : -1;
    }
  } else {
    t0 = blockIdx.x * kRopeTokens;
    if (warp < kRopeTokens) {
      const int t = t0 + warp;
      int b = -1, zero = 0, pos = 0;
      long long row = -1;
      if (t < p.N) {
        const int o = owner_of(p.token_start, p.B, t, lane);
        const int s = p.token_start[o], e = p.token_start[o + 1];
        if (s >= 0 && s <= t && t < e && e <= p.N) {
          const int L = p.seq_lens[o];
          b = o;
          zero = L < 0 || static_cast<long long>(L) + (e - s) > p.capacity;
          if (zero && lane == 0) report_status(p.status, EAGLE_ERR_SEQ);
          pos = p.positions ? p.positions[t] : L + (t - s);
          if (!zero) row = rope_row(p, o, L + (t - s));
        }
      }
      if (lane == 0) {
        s_seq[warp] = b;
        s_zero[warp] = zero;
        s_pos[warp] = pos;
        s_row[warp] = row;
      }
    } else if (blockIdx.x == 0 && blockIdx.y == 0) {
      // the list of starts has to ascend within the tensor
      int bad = 0;
      for (int b = tid - 32 * kRopeTokens; b <= p.B; b += kRopeThreads - 32 * kRopeTokens) {
        const int s = p.token_start[b];
        if (s < 0 || s > p.N || (b < p.B && p.token_start[b + 1] < s)) bad = 1;
      }
      if (bad) report_status(p.status, EAGLE_ERR_SEQ);
    }
  }
  __syncthreads();

  const int half = p.R / 2;
  for (int i = tid; i < kRopeTokens * half; i += kRopeThreads) {
    const int t = i / half, m = i - t * half;
    double turns = static_cast<double>(s_pos[t]) * (p.freqs[m] * 0.15915494309189535);      // 1 / (2 pi)
    turns -= rint(turns);
    float sn, cs;
    sincospif(2.0f * static_cast<float>(turns), &sn, &cs);
    s_cs[t][m] = make_float2(cs * p.amplitude, sn * p.amplitude);
  }
  __syncthreads();

  // ---- units: `u` is the place within a head, fixed for the thread; (token, head) advances by `step` heads
  const int U = p.D / 16, u = tid & (U - 1), step = kRopeThreads / U;
  const int h_lo = blockIdx.y * p.heads_per_block, H = p.Hq + 2 * p.Hkv;
  const int heads = min(p.heads_per_block, H - h_lo);
  // element offsets of the unit's two vectors; `turn`: they hold eight whole pairs
  const bool turn = 16 * u < p.R;
  const int va = !turn ? 16 * u : (p.interleaved ? 16 * u : 8 * u);
  const int vb = !turn ? 16 * u + 8 : (p.interleaved ? 16 * u + 8 : half + 8 * u);
  int tok = 0, h = tid / U;
  while (h >= heads && tok < n_tok) { h -= heads; ++tok; }

  auto source = [&](int t, int head) -> const uint4* {
    const __nv_bfloat16* s = head < p.Hq              ? p.q + (t0 + t) * p.q_stride + static_cast<long long>(head) * p.D
                             : head < p.Hq + p.Hkv    ? p.k + (t0 + t) * p.k_stride + static_cast<long long>(head - p.Hq) * p.D
                                                      : p.v + (t0 + t) * p.v_stride + static_cast<long long>(head - p.Hq - p.Hkv) * p.D;
    return reinterpret_cast<const uint4*>(s);
  };
  auto live = [&](int t, int head) { return s_seq[t] >= 0 && (head < p.Hq || s_row[t] >= 0); };
  auto finish = [&](int t, int head, const Vec2& in) {
    const bool is_q = head < p.Hq, is_v = head >= p.Hq + p.Hkv;
    float x[8], y[8];
    Vec2 out = in;
    if (turn && !is_v) {
      widen(in.a, x);
      widen(in.b, y);
      if (p.interleaved) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 c = s_cs[t][8 * u + e], d = s_cs[t][8 * u + 4 + e];
          const float x0 = x[2 * e], x1 = x[2 * e + 1], y0 = y[2 * e], y1 = y[2 * e + 1];
          x[2 * e] = x0 * c.x - x1 * c.y;
          x[2 * e + 1] = x1 * c.x + x0 * c.y;
          y[2 * e] = y0 * d.x - y1 * d.y;
          y[2 * e + 1] = y1 * d.x + y0 * d.y;
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float2 c = s_cs[t][8 * u + e];
          const float x0 = x[e], y0 = y[e];
          x[e] = x0 * c.x - y0 * c.y;
          y[e] = y0 * c.x + x0 * c.y;
        }
      }
      if (is_q || !FP8) {
        out.a = narrow(x);
        out.b = narrow(y);
      }
    } else if (FP8 && !is_q) {
      widen(in.a, x);
      widen(in.b, y);
    }
    if (is_q) {
      if (s_zero[t]) out.a = out.b = make_uint4(0u, 0u, 0u, 0u);
      __nv_bfloat16* dst = p.q_out + (static_cast<long long>(t0 + t) * p.Hq + head) * p.D;
      *reinterpret_cast<uint4*>(dst + va) = out.a;
      *reinterpret_cast<uint4*>(dst + vb) = out.b;
      return;
    }
    const int g = is_v ? head - p.Hq - p.Hkv : head - p.Hq;
    const long long row = s_row[t] + g * p.head_rows;
    if constexpr (FP8) {
      const float scale = (is_v ? p.v_scale : p.k_scale)[static_cast<size_t>(s_seq[t]) * p.Hkv + g];
      uint8_t* dst = static_cast<uint8_t*>(is_v ? p.v_cache : p.k_cache) + row * p.D;
      *reinterpret_cast<uint2*>(dst + va) = codes(x, scale);
      *reinterpret_cast<uint2*>(dst + vb) = codes(y, scale);
    } else {
      __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(is_v ? p.v_cache : p.k_cache) + row * p.D;
      *reinterpret_cast<uint4*>(dst + va) = out.a;
      *reinterpret_cast<uint4*>(dst + vb) = out.b;
    }
  };
  auto advance = [&]() {
    h += step;
    while (h >= heads && tok < n_tok) { h -= heads; ++tok; }
  };
  while (tok < n_tok) {
    int ts[2], hs[2];
    bool on[2];
    Vec2 in[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      ts[i] = tok;
      hs[i] = h_lo + h;
      on[i] = tok < n_tok && live(tok, hs[i]);
      if (on[i]) {
        const uint4* s = source(ts[i], hs[i]);
        in[i].a = s[va / 8];
        in[i].b = s[vb / 8];
      }
      if (tok < n_tok) advance();
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (on[i]) finish(ts[i], hs[i], in[i]);
  }
}

}  // namespace

cudaError_t launch_rope(const RopeParams& p_in, bool tree, int sm_count, cudaStream_t stream) {
  RopeParams p = p_in;
  const int H = p.Hq + 2 * p.Hkv;
  const long long groups = tree ? static_cast<long long>(p.B) * ((p.T + kRopeTokens - 1) / kRopeTokens) : (static_cast<long long>(p.N) + kRopeTokens - 1) / kRopeTokens;
  // few tokens: the heads are split over several CTAs (each computes the same sines again) until there are two CTAs per SM
  int splits = 1;
  while (groups * splits < 2ll * sm_count && H > splits * (kRopeThreads / (p.D / 16)) / kRopeTokens && splits < 64) splits *= 2;
  p.heads_per_block = (H + splits - 1) / splits;
  const dim3 grid(static_cast<unsigned>(groups), static_cast<unsigned>((H + p.heads_per_block - 1) / p.heads_per_block));
  const bool fp8 = p.k_scale != nullptr;
  if (tree) {
    if (fp8) rope_kernel<true, true><<<grid, kRopeThreads, 0, stream>>>(p);
    else rope_kernel<true, false><<<grid, kRopeThreads, 0, stream>>>(p);
  } else {
    if (fp8) rope_kernel<false, true><<<grid, kRopeThreads, 0, stream>>>(p);
    else rope_kernel<false, false><<<grid, kRopeThreads, 0, stream>>>(p);
  }
  count_launch();
  return cudaGetLastError();
}

}  // namespace eagle
