// Parameters of the append into a block-scaled cache (block.cu).
#pragma once
#include "rope.cuh"

namespace eagle {

struct BlockParams {
  RopeParams r;                  // (k_scale and v_scale of it are not used; D = 128)
  float* k_scale;                // one per block and KV head
  float* v_scale;
  int32_t block_size, block_shift;
  long long head_blocks;         // blocks from one KV head to the next
  int32_t span;                  // chunk form: rows whose blocks a CTA takes
  int32_t store_heads;           // keys' and values' heads that a CTA takes (single tokens: a warp)
  int32_t store_groups, store_ctas;      // CTAs (single tokens: warps) per span or tree, and CTAs in all; the queries' CTAs come behind them
};

cudaError_t launch_block(const BlockParams& p, bool tree, int sm_count, cudaStream_t stream);

}  // namespace eagle
