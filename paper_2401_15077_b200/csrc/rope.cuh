// Parameters of the rotary append (rope.cu), and what it shares with the append into a block-scaled cache (block.cu).
#pragma once
#include <cuda_fp8.h>

#include "common.cuh"

namespace eagle {

struct RopeParams {
  const __nv_bfloat16* q;        // rows of `*_stride` elements
  const __nv_bfloat16* k;
  const __nv_bfloat16* v;
  long long q_stride, k_stride, v_stride;
  __nv_bfloat16* q_out;          // dense [rows, Hq, D]
  void* k_cache;                 // bf16, or codes when the scales are set
  void* v_cache;
  const float* k_scale;          // [B, Hkv] or null
  const float* v_scale;
  const int32_t* block_table;    // paged cache, or null
  int32_t page_size, page_shift, max_pages, num_pages;
  long long capacity;            // slots per sequence
  long long head_rows;           // cache rows from one KV head to the next
  const int32_t* seq_lens;       // [B]
  const int32_t* token_start;    // [B + 1] (chunk form)
  const int32_t* positions;      // [N] or null (chunk form)
  const int32_t* tree_parent;    // tree form
  const int32_t* tree_sizes;
  const double* freqs;           // [R / 2] radians per position
  float amplitude;
  int32_t B, N, T, Hq, Hkv, D, R;
  int32_t interleaved, shared_tree;
  int32_t heads_per_warp, head_chunks;
  int32_t* status;
};

// Cache row (of KV head 0) of a sequence's slot; -1, and EAGLE_ERR_PAGE, when its block-table entry is outside the pool.
__device__ __forceinline__ long long rope_row(const RopeParams& p, int b, int slot) {
  if (!p.block_table) return static_cast<long long>(b) * p.Hkv * p.capacity + slot;
  const int page = p.block_table[static_cast<size_t>(b) * p.max_pages + (slot >> p.page_shift)];
  if (page < 0 || page >= p.num_pages) {
    report_status(p.status, EAGLE_ERR_PAGE);
    return -1;
  }
  return static_cast<long long>(page) * p.Hkv * p.page_size + (slot & (p.page_size - 1));
}

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
// Eight e4m3 codes of f / scale (round to nearest even, magnitudes above 448 become 448, NaN stays NaN).
// With q = f * inv, up to two steps of fp32 off, what is missing is exactly (f - q scale) / scale, and f - q scale is a number of fp32:
// adding it times `inv` leaves an error of 2^-44 before the sum is rounded to fp32.  So a value at the middle between two codes is
// seen to be there.  Where q is large its magnitude is cut at 1024 first (the sum is large all the same): an infinite one would
// make f - q scale infinite, too.
__device__ __forceinline__ float2 quotients(float2 f, float scale, float inv) {
  float2 q = make_float2(f.x * inv, f.y * inv);
  asm("min.NaN.xorsign.abs.f32 %0, %0, %1;" : "+f"(q.x) : "f"(1024.f));      // (of the magnitudes; the sign stays)
  asm("min.NaN.xorsign.abs.f32 %0, %0, %1;" : "+f"(q.y) : "f"(1024.f));
  return make_float2(fmaf(-fmaf(q.x, scale, -f.x), inv, q.x), fmaf(-fmaf(q.y, scale, -f.y), inv, q.y));      // (these signs keep that of a zero)
}
__device__ __forceinline__ uint2 codes(const float* f, float scale, float inv) {
  uint32_t w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float2 lo = quotients(make_float2(f[4 * i], f[4 * i + 1]), scale, inv);
    const float2 hi = quotients(make_float2(f[4 * i + 2], f[4 * i + 3]), scale, inv);
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

cudaError_t launch_rope(const RopeParams& p, bool tree, int sm_count, cudaStream_t stream);

}  // namespace eagle
