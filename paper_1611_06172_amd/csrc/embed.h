// Host interface of embed.hip: rows of a matrix by word, and their gradient. All
// arguments are validated by the caller.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace w2v {

struct EmbedArgs {
  const int32_t* ids;  // n words, -1 absent
  const void* weight;  // V x D, stride ldw
  void* y;             // n x D, stride ldy
  int64_t ldw, ldy;
  int32_t n, V, D, dtype, out_dtype;
  float scale;
  int32_t* status;
};

struct EmbedBackwardArgs {
  const void* dy;      // n x D, stride lddy
  const int32_t* ids;
  void* grad;          // V x D, stride ldg
  int64_t lddy, ldg;
  int32_t n, V, D, dtype, grad_dtype;
  bool accumulate;
  float scale;
  int32_t* status;
};

hipError_t launch_embed(const EmbedArgs& a, hipStream_t s);
size_t embed_backward_workspace_bytes(int32_t n, int32_t V, int32_t D);
hipError_t launch_embed_backward(const EmbedBackwardArgs& a, void* workspace, hipStream_t s);

}  // namespace w2v
