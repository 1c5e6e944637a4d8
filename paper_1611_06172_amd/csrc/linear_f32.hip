// The vocabulary head's matrix products of float32 operands.
#include "linear_kernels.h"

namespace w2v {

hipError_t launch_linear_f32(const LinearArgs& l, void* workspace, hipStream_t s) {
  return launch_linear_as<float, float>(l, workspace, s);
}

hipError_t launch_backward_f32(const LinearBackwardArgs& l, void* workspace, hipStream_t s) {
  return launch_backward_as<float>(l, workspace, s);
}

}  // namespace w2v
