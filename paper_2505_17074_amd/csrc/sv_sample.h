// Internal declarations of sampling.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sv {

struct SampleParams {
  const void* logits;
  int64_t stride;
  const float* temperature;
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  const float* uniforms;
  int32_t* tokens;
  void* rows;
  int64_t rows_stride;
  int32_t V;
  int32_t kind;                        // spec_sample_rows_t
};

hipError_t launch_sample(const SampleParams& p, int num_rows, bool f32, hipStream_t s);

}  // namespace sv
