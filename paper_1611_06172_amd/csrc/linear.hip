// Matrix products of the vocabulary head: workspace sizes and the choice of
// the element type's kernels (linear_kernels.h).
#include "linear_plan.h"

namespace w2v {

size_t linear_workspace_bytes(int32_t M, int32_t N, int32_t K, int32_t dtype) {
  if (M == 0 || few_rows(M, K)) return 0;
  return partial_bytes(plan_product(M, N, K, dtype, false), M, N) +
         copy_bytes(M, M, N, K, dtype) + copy_bytes(N, M, N, K, dtype);
}

size_t linear_backward_workspace_bytes(int32_t M, int32_t N, int32_t K, int32_t dtype,
                                       int32_t activation) {
  const BackwardPlan b = plan_backward(M, N, K, dtype, activation);
  return b.dz + b.partial + b.sums + b.x;
}

hipError_t launch_linear(const LinearArgs& a, void* workspace, hipStream_t s) {
  switch (a.dtype) {
    case W2V_DTYPE_F32:
      return launch_linear_f32(a, workspace, s);
    case W2V_DTYPE_BF16:
      return launch_linear_bf16(a, workspace, s);
    default:
      return launch_linear_f16(a, workspace, s);
  }
}

hipError_t launch_linear_backward(const LinearBackwardArgs& a, void* workspace,
                                  hipStream_t s) {
  switch (a.dtype) {
    case W2V_DTYPE_F32:
      return launch_backward_f32(a, workspace, s);
    case W2V_DTYPE_BF16:
      return launch_backward_bf16(a, workspace, s);
    default:
      return launch_backward_f16(a, workspace, s);
  }
}

}  // namespace w2v
