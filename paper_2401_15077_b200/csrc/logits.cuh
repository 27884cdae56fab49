// Parameters of the logit adjustment (logits.cu).
#pragma once
#include "common.cuh"

namespace eagle {

constexpr int kMaxBias = 1024;

struct LogitsParams {
  const void* logits;            // [B, T + 1, V] fp32 or bf16
  float* out;                    // [B, T + 1, V]
  const int32_t* draft_tokens;   // [B, T]
  const int32_t* tree_parent;    // [B, T] or [T]
  const int32_t* tree_sizes;
  const int32_t* history;        // [B, H] or null
  const int32_t* history_len;    // [B]
  const int32_t* prompt_len;     // [B] or null
  const float* repetition;       // [B] or null
  const float* presence;
  const float* frequency;
  const int32_t* bias_tokens;    // [B, max_bias] or null
  const float* bias_values;
  const int32_t* bias_len;       // [B] or null
  const uint32_t* allowed;       // [B, T + 1, ceil(V / 32)] or null
  int32_t B, T, V, H, max_bias;
  int32_t bf16, shared_tree;
  int32_t rows_per_block;
  int32_t* status;
};

cudaError_t launch_logits(const LogitsParams& p, int sm_count, cudaStream_t stream);

}  // namespace eagle
