// Matrix products of the vocabulary head: workspace sizes and the choice of
// the element type's kernels (linear_kernels.h).
#include "linear_plan.h"

namespace w2v {

bool linear_fits(int32_t M, int32_t N, int32_t K, int32_t dtype, bool backward) {
  constexpr int64_t kMost = UINT32_MAX / 256;
  if (M == 0) return true;
  if (!backward && few_rows(M, K)) return ceil_div(N, 64) <= kMost;
  // (the smallest tiles settle it for all but the largest outputs, and a product
  // that is split has no more than kSlots blocks)
  const int64_t m = ceil_div(M, 64), n = ceil_div(N, 64), k = ceil_div(K, 64);
  if ((backward ? (m > n ? m : n) * k : m * n) <= kMost) return true;
  auto blocks = [](const Plan& p) { return (int64_t)p.tiles_m * p.tiles_n * p.splits; };
  if (!backward) return blocks(plan_product(M, N, K, dtype, false)) <= kMost;
  const BackwardPlan b = plan_backward(M, N, K, dtype, W2V_ACTIVATION_NONE);
  return blocks(b.dx) <= kMost && blocks(b.dw) <= kMost;
}

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
