// Element types, wide loads and stores, activations and launch helpers shared
// by the kernels of the vocabulary head (linear.hip, distill.hip,
// sample.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "w2v_internal.h"

namespace w2v {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(bf16_t v) {
  return __builtin_bit_cast(float, (uint32_t)__builtin_bit_cast(uint16_t, v) << 16);
}
__device__ __forceinline__ float to_f32(f16_t v) { return (float)v; }

// One rounding to nearest even from 32 bits.
template <typename T>
__device__ __forceinline__ T from_f32(float v) {
  return (T)v;
}

// N consecutive elements at an address aligned to one element. gfx950 loads
// and stores up to 16 bytes at any alignment in one instruction, so rows of
// odd strides take the same path as aligned ones.
template <typename T, int N>
struct Pack {
  T v[N];
};

template <typename T, int N>
__device__ __forceinline__ Pack<T, N> load_pack(const T* p) {
  Pack<T, N> out;
  __builtin_memcpy(&out, p, sizeof(out));
  return out;
}

// 16 bytes in four registers: elements that are only moved stay packed.
__device__ __forceinline__ uint4 load_16(const void* p) {
  uint4 v;
  __builtin_memcpy(&v, p, 16);
  return v;
}

// The elements of 16 bytes, taken from whole words: the pack stays in four
// registers.
template <typename T>
__device__ __forceinline__ void unpack_words(uint4 w, float (&out)[16 / (int)sizeof(T)]) {
  const uint32_t word[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; i++) {
    if constexpr (sizeof(T) == 4) {
      out[i] = __builtin_bit_cast(float, word[i]);
    } else {
      const uint16_t lo = (uint16_t)word[i], hi = (uint16_t)(word[i] >> 16);
      out[2 * i] = to_f32(__builtin_bit_cast(T, lo));
      out[2 * i + 1] = to_f32(__builtin_bit_cast(T, hi));
    }
  }
}

template <typename T, int N>
__device__ __forceinline__ void store_pack(T* p, const Pack<T, N>& v) {
  __builtin_memcpy(p, &v, sizeof(v));
}

// The first n (0..N) elements at p, the others 0.
template <typename T, int N>
__device__ __forceinline__ Pack<T, N> load_some(const T* p, int64_t n) {
  if (n >= N) return load_pack<T, N>(p);
  Pack<T, N> out;
#pragma unroll
  for (int i = 0; i < N; i++) out.v[i] = i < n ? p[i] : T(0.0f);
  return out;
}

template <typename T, int N>
__device__ __forceinline__ void store_some(T* p, int64_t n, const Pack<T, N>& v) {
  if (n >= N) {
    store_pack<T, N>(p, v);
    return;
  }
#pragma unroll
  for (int i = 0; i < N; i++)
    if (i < n) p[i] = v.v[i];
}

constexpr float kLog2e = 1.44269504088896341f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// erfc(|x|) as exp(-x^2) times a polynomial in t = 1 / (1 + p |x|), fitted to
// exp(x^2) erfc(x) over [0, 10] for the least relative error, 1e-7, so that the
// tail, where gelu is all of erfc, is as exact as the rest: with the roundings
// gelu is within 5 units of 2^-24 of z, and within 5e-6 of itself where it is far
// smaller than z. A fifth of the library function's instructions.
__device__ __forceinline__ float erfc_of_abs(float x) {
  x = fabsf(x);
  const float t = __builtin_amdgcn_rcpf(1.0f + 0.43f * x);
  float poly = 0.07314582f;
  poly = poly * t - 0.30809563f;
  poly = poly * t + 0.37988725f;
  poly = poly * t - 0.08230429f;
  poly = poly * t + 0.24508066f;
  poly = poly * t + 0.2054725f;
  poly = poly * t + 0.24429382f;
  poly = poly * t + 0.24251983f;
  return poly * t * exp2_fast(x * x * -kLog2e);
}

// FAST: with the hardware's exponential and reciprocal and the polynomial
// above, for results that are rounded to 16 bits: before that rounding they are
// within 1e-5 of their value, 0.02 units of fp16 and 0.003 of bf16 (and bf16's
// below 2^-126 may be 0).
template <bool FAST>
__device__ __forceinline__ float activate(float z, int activation) {
  switch (activation) {
    case W2V_ACTIVATION_RELU:
      return z < 0.0f ? 0.0f : z;  // NaN stays NaN
    case W2V_ACTIVATION_GELU: {
      if (!FAST) return 0.5f * z * erfcf(z * -0.70710678118654752f);
      const float half = 0.5f * erfc_of_abs(z * 0.70710678118654752f);
      return z * (z < 0.0f ? half : 1.0f - half);
    }
    case W2V_ACTIVATION_SILU:
      return FAST ? z * __builtin_amdgcn_rcpf(1.0f + exp2_fast(z * -kLog2e))
                  : z / (1.0f + expf(-z));
    case W2V_ACTIVATION_TANH:
      return tanhf(z);
    case W2V_ACTIVATION_SIGMOID:
      return FAST ? __builtin_amdgcn_rcpf(1.0f + exp2_fast(z * -kLog2e))
                  : 1.0f / (1.0f + expf(-z));
    default:
      return z;
  }
}

// Derivative of `activate` at z. relu's at 0 is 0.
__device__ __forceinline__ float activation_slope(float z, int activation) {
  switch (activation) {
    case W2V_ACTIVATION_RELU:
      return z > 0.0f ? 1.0f : (z <= 0.0f ? 0.0f : z);
    case W2V_ACTIVATION_GELU:
      return 0.5f * erfcf(z * -0.70710678118654752f) +
             z * expf(-0.5f * z * z) * 0.39894228040143268f;
    case W2V_ACTIVATION_SILU: {
      const float p = 1.0f / (1.0f + expf(-z));
      const float q = 1.0f / (1.0f + expf(z));  // 1 - p without cancellation
      return p + z * p * q;
    }
    case W2V_ACTIVATION_TANH: {
      const float e = expf(-2.0f * fabsf(z));  // 1 - tanh^2 without cancellation
      return 4.0f * e / ((1.0f + e) * (1.0f + e));
    }
    case W2V_ACTIVATION_SIGMOID:
      return (1.0f / (1.0f + expf(-z))) * (1.0f / (1.0f + expf(z)));
    default:
      return 1.0f;
  }
}

// Records that a row was skipped for a list, a label or a setting out of range.
__device__ __forceinline__ void report_row(int32_t* status) {
  __hip_atomic_store(status, kStatusBadRow, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
}

// Rows of one launch of a block a row: a grid's threads, up to 1024 a row, are
// counted in 32 bits. Calls with more rows are made of even parts.
constexpr int kLaunchRows = 1 << 21;
inline int rows_of_launch(int rows) {
  const int parts = (rows + kLaunchRows - 1) / kLaunchRows;
  return (rows + parts - 1) / parts;
}
inline const void* row_at(const void* p, int64_t row, int64_t ld, int32_t dtype) {
  return p == nullptr ? p : (const char*)p + row * ld * (dtype == W2V_DTYPE_F32 ? 4 : 2);
}
template <typename V>
inline V* row_at(V* p, int64_t row, int64_t ld = 1) {
  return p == nullptr ? p : p + row * ld;
}

// Reductions over a wavefront and over a block of up to 16 of them; every
// thread gets the result. `scratch`: 16 floats of LDS, free again on return.
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
  return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}
// Two values at once; `scratch`: 32 floats.
__device__ __forceinline__ void block_sums(float& a, float& b, float* scratch) {
  a = wave_sum(a);
  b = wave_sum(b);
  const int w = threadIdx.x >> 6, waves = blockDim.x >> 6;
  if ((threadIdx.x & 63) == 0) {
    scratch[w] = a;
    scratch[16 + w] = b;
  }
  __syncthreads();
  a = scratch[0];
  b = scratch[16];
  for (int i = 1; i < waves; i++) {
    a += scratch[i];
    b += scratch[16 + i];
  }
  __syncthreads();
}
__device__ __forceinline__ void block_maxima(float& a, float& b, float* scratch) {
  a = wave_max(a);
  b = wave_max(b);
  const int w = threadIdx.x >> 6, waves = blockDim.x >> 6;
  if ((threadIdx.x & 63) == 0) {
    scratch[w] = a;
    scratch[16 + w] = b;
  }
  __syncthreads();
  a = scratch[0];
  b = scratch[16];
  for (int i = 1; i < waves; i++) {
    a = fmaxf(a, scratch[i]);
    b = fmaxf(b, scratch[16 + i]);
  }
  __syncthreads();
}
__device__ __forceinline__ float block_sum(float v, float* scratch) {
  v = wave_sum(v);
  if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = v;
  __syncthreads();
  v = scratch[0];
  for (int w = 1; w < (int)(blockDim.x >> 6); w++) v += scratch[w];
  __syncthreads();
  return v;
}
__device__ __forceinline__ float block_max(float v, float* scratch) {
  v = wave_max(v);
  if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = v;
  __syncthreads();
  v = scratch[0];
  for (int w = 1; w < (int)(blockDim.x >> 6); w++) v = fmaxf(v, scratch[w]);
  __syncthreads();
  return v;
}

}  // namespace w2v
