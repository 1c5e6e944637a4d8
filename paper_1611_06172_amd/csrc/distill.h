// Host interface of distill.hip: distillation from a teacher's top logits.
// All arguments are validated by the caller.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace w2v {

struct DistillArgs {
  const void* logits;  // rows x V, stride ld
  int64_t ld;
  int32_t rows, V, dtype;
  const int32_t* ids;   // rows x K, -1 absent
  const void* teacher;  // rows x K, type teacher_dtype
  int32_t K, teacher_dtype;
  const int32_t* labels;  // rows, -1 none, or NULL
  float temperature, soft, hard;
  const float* row_weight;  // rows, or NULL: 1
  float* loss;              // rows, or NULL
  float* stats;             // rows x 3; an input of the backward pass
  void* grad;               // rows x V, stride ldg, or NULL
  int64_t ldg;
  int32_t* status;
};

size_t distill_workspace_bytes(int32_t rows, int32_t V, int32_t dtype);
// Loss and statistics, and the gradient where a.grad is given.
hipError_t launch_distill(const DistillArgs& a, void* workspace, hipStream_t s);
// The gradient from a.stats.
hipError_t launch_distill_backward(const DistillArgs& a, hipStream_t s);

}  // namespace w2v
