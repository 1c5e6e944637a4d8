// Host interface of dropout.hip. All arguments are validated by the caller.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace w2v {

struct DropoutArgs {
  const void* x;         // rows x cols, stride ldx
  const void* residual;  // or NULL; stride ldr
  void* y;               // stride ldy; may be x or the residual
  int64_t ldx, ldr, ldy;
  int32_t rows, cols, dtype;
  uint64_t below;        // elements whose number is below it are dropped (<= 2^32)
  float scale;           // of the others
  uint64_t seed, offset;
  const int64_t* offset_dev;  // or NULL: added to offset
};

hipError_t launch_dropout(const DropoutArgs& a, hipStream_t s);

}  // namespace w2v
