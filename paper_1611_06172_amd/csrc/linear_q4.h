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

// What a wavefront's loads of W may reach, in bytes from its first tile: those of the
// `most` tiles from `tile` on that lie before `end`, nothing where there are none.
struct Q4Range {
  int32_t words, scales, bias;
};
__host__ __device__ __forceinline__ Q4Range q4_range(const Q4Shape& q, int64_t tile, int64_t end,
                                                     int most, bool bias) {
  const int64_t left = end - tile, rows = q.N - tile * 16;
  const int count = left >= most ? most : left > 0 ? (int)left : 0;
  return {count * q.blocks * 256, count * q.groups * 32,
          !bias || rows <= 0 ? 0 : (rows < most * 16 ? (int32_t)rows : most * 16) * 4};
}

// Where the loads for tile t of these begin, in bytes, of the step at column block
// `block`: a lane's words, the scales of its row from group `group` on, its row's bias.
// Blocks lie in fours, the rest together, and so do groups. All of it is the lane's
// offset, which the range check counts; one in a scalar register it need not.
__host__ __device__ __forceinline__ int32_t q4_words_at(const Q4Shape& q, int t, int block,
                                                        int lane) {
  const int rest = q.blocks - block;
  return (t * q.blocks + block) * 256 + lane * (rest >= 4 ? 16 : rest * 4);
}
__host__ __device__ __forceinline__ int32_t q4_scales_at(const Q4Shape& q, int t, int group,
                                                         int row) {
  const int first = group & ~3, rest = q.groups - first;
  return t * q.groups * 32 + first * 32 + (group - first) * 2 + row * (rest >= 4 ? 8 : rest * 2);
}
__host__ __device__ __forceinline__ int32_t q4_bias_at(int t, int row) { return t * 64 + row * 4; }

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
