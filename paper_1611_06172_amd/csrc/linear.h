// Host interface of linear.hip: products with the vocabulary head's epilogue
// and their gradients. All arguments are validated by the caller.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace w2v {

struct LinearArgs {
  const void* x;      // M x K, stride ldx
  const void* w;      // N x K, stride ldw
  const float* bias;  // N or NULL
  const void* residual;
  void* y;
  void* pre;  // z before the activation, or NULL
  int64_t ldx, ldw, ldr, ldy, ldp;
  int32_t M, N, K;
  int32_t dtype, out_dtype, activation;
};

struct LinearBackwardArgs {
  const void* dy;
  const void* x;
  const void* w;
  const void* pre;
  void* dx;
  void* dw;
  float* db;
  int64_t lddy, ldx, ldw, ldp, lddx, lddw;
  int32_t M, N, K;
  int32_t dtype, activation;
};

// Whether the product's blocks, or those of both gradients' products, fit a grid,
// whose threads are counted in 32 bits.
bool linear_fits(int32_t M, int32_t N, int32_t K, int32_t dtype, bool backward);
size_t linear_workspace_bytes(int32_t M, int32_t N, int32_t K, int32_t dtype);
size_t linear_backward_workspace_bytes(int32_t M, int32_t N, int32_t K, int32_t dtype,
                                       int32_t activation);
hipError_t launch_linear(const LinearArgs& a, void* workspace, hipStream_t s);
hipError_t launch_linear_backward(const LinearBackwardArgs& a, void* workspace,
                                  hipStream_t s);

}  // namespace w2v
