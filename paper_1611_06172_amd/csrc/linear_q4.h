// Host interface of linear_q4.hip: a matrix in 4 bits, and products with it. All
// arguments are validated by the caller.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace w2v {

// The layout of a matrix in 4 bits: rows in tiles of 16, columns in blocks of 32
// and in groups of 1, 2 or 4 blocks, each group with one scale.
struct Q4Shape {
  int32_t N, K, group;
  int64_t tiles;    // of 16 rows
  int32_t groups;   // of a row
  int32_t blocks;   // of a row
};

inline Q4Shape q4_shape(int32_t N, int32_t K, int32_t group) {
  Q4Shape q;
  q.N = N;
  q.K = K;
  q.group = group;
  q.tiles = ((int64_t)N + 15) / 16;
  q.groups = (int32_t)(((int64_t)K + group - 1) / group);
  q.blocks = q.groups * (group / 32);
  return q;
}

struct QuantizeArgs {
  const void* w;  // N x K, stride ldw
  int64_t ldw;
  int32_t dtype;
  uint32_t* packed;
  void* scales;  // bfloat16
};

struct LinearQ4Args {
  const void* x;  // M x K, stride ldx
  const uint32_t* packed;
  const void* scales;
  const float* bias;  // or NULL
  void* y;            // M x N, stride ldy
  int64_t ldx, ldy;
  int32_t M, dtype, out_dtype;
};

hipError_t launch_quantize_q4(const QuantizeArgs& a, const Q4Shape& q, hipStream_t s);
hipError_t launch_linear_q4(const LinearQ4Args& a, const Q4Shape& q, hipStream_t s);

}  // namespace w2v
