// Host interface of sample.hip: words drawn from scores. All arguments are
// validated by the caller.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace w2v {

struct SampleArgs {
  const void* logits;     // rows x V, stride ld
  const float* uniforms;  // rows x V, stride ldu, or NULL (greedy)
  int64_t ld, ldu;
  int32_t rows, V, dtype;
  // per-row settings, or NULL: the scalar for every row
  const float* temperatures;
  const int32_t* top_ks;
  const float* top_ps;
  const float* min_ps;
  float temperature;
  int32_t top_k;
  float top_p, min_p;
  int32_t* ids;
  float* logprob;  // or NULL
  int32_t* status;
};

size_t sample_workspace_bytes(int32_t rows, int32_t V);
hipError_t launch_sample(const SampleArgs& a, void* workspace, hipStream_t s);

}  // namespace w2v
