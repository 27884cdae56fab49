// Parameters of the rotary append (rope.cu).
#pragma once
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

cudaError_t launch_rope(const RopeParams& p, bool tree, int sm_count, cudaStream_t stream);

}  // namespace eagle
