// Parameters of the sampler (sample.cu).
#pragma once
#include "common.cuh"

namespace eagle {

struct SampleParams {
  const void* logits;            // [B, R, V] fp32 or bf16
  const float* uniforms;         // [B, R] (with tokens)
  int32_t* tokens;               // [B, R] or null
  float* probs;                  // [B, R, V] or null
  const int32_t* num_rows;       // [B] or null
  const float* temperature;      // [B] or null
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  int32_t B, R, V;
  int32_t bf16;
  int32_t* status;
};

cudaError_t launch_sample(const SampleParams& p, int sm_count, cudaStream_t stream);

}  // namespace eagle
