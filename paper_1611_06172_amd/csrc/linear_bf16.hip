// The vocabulary head's matrix products of bfloat16 operands.
#include "linear_kernels.h"

namespace w2v {

hipError_t launch_linear_bf16(const LinearArgs& l, void* workspace, hipStream_t s) {
  return l.out_dtype == W2V_DTYPE_F32 ? launch_linear_as<bf16_t, float>(l, workspace, s)
                                      : launch_linear_as<bf16_t, bf16_t>(l, workspace, s);
}

hipError_t launch_backward_bf16(const LinearBackwardArgs& l, void* workspace, hipStream_t s) {
  return launch_backward_as<bf16_t>(l, workspace, s);
}

}  // namespace w2v
