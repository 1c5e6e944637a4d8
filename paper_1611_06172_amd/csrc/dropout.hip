// Dropout whose mask is never stored: element i of a matrix, counted row by row
// whatever the stride, is kept where the 32-bit number r_i is at least `below`,
//
//   y_i = [r_i >= below] x_i 2^32 / (2^32 - below) + residual_i,
//
// and r_i comes from Philox4x32-10 (Salmon, Moraes, Dror, Shaw, SC'11), so the
// backward pass forms the same numbers again. x (and the residual) is read once
// and y written once; the generator has to keep up with that.
//
// One block of the generator holds the upper 16 bits of eight elements' numbers,
// another one the lower 16. The second one is formed only where an upper half
// equals below's, which alone does not decide: for one element in 65,536. A
// number of 32 bits costs as much as one of 16 that way: 2.5 wide
// multiplications an element. Measured: 65,536 x 600 bf16 with a residual in 45 us, 5.2
// TB/s, which is a copy's rate; 64 x 300 fp32 9 us, 2.9 of them in the kernel.
#include "dropout.h"
#include "head_types.h"

namespace w2v {
namespace {

constexpr int kBlock = 256;
constexpr int kE = 8;  // elements of a generator's block

struct Words {
  uint32_t v[4];
};

// Constants: the multipliers and Weyl increments published for Philox4x32.
__device__ __forceinline__ Words philox4x32_10(Words c, uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int r = 0; r < 10; r++) {
    const uint64_t a = (uint64_t)c.v[0] * 0xD2511F53u;
    const uint64_t b = (uint64_t)c.v[2] * 0xCD9E8D57u;
    c = {{(uint32_t)(b >> 32) ^ c.v[1] ^ k0, (uint32_t)b, (uint32_t)(a >> 32) ^ c.v[3] ^ k1,
          (uint32_t)a}};
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return c;
}

// The halves of words: element j has word j / 2, the low half first.
__device__ __forceinline__ uint32_t half_of(const Words& w, int j) {
  return j & 1 ? w.v[j / 2] >> 16 : w.v[j / 2] & 0xffffu;
}

// Which of elements 8 block to 8 block + 7 stay, as bits.
__device__ __forceinline__ uint32_t kept(const DropoutArgs& a, uint64_t offset, uint64_t block) {
  const uint32_t k0 = (uint32_t)a.seed, k1 = (uint32_t)(a.seed >> 32);
  Words counter = {{(uint32_t)block, (uint32_t)(block >> 32), (uint32_t)offset,
                    (uint32_t)(offset >> 32)}};
  const Words high = philox4x32_10(counter, k0, k1);
  const uint32_t edge = (uint32_t)(a.below >> 16), rest = (uint32_t)a.below & 0xffffu;
  uint32_t keep = 0, open = 0;
#pragma unroll
  for (int j = 0; j < kE; j++) {
    const uint32_t h = half_of(high, j);
    keep |= h >= edge ? 1u << j : 0u;
    open |= h == edge ? 1u << j : 0u;
  }
  // with rest 0 every lower half is at least it
  if (rest != 0 && open != 0) {
    counter.v[1] |= 0x80000000u;
    const Words low = philox4x32_10(counter, k0, k1);
#pragma unroll
    for (int j = 0; j < kE; j++)
      if ((open >> j & 1) != 0 && half_of(low, j) < rest) keep &= ~(1u << j);
  }
  return keep;
}

__device__ __forceinline__ uint64_t call_offset(const DropoutArgs& a) {
  return a.offset + (a.offset_dev != nullptr ? (uint64_t)*a.offset_dev : 0);
}

template <bool RESIDUAL, typename T>
__device__ __forceinline__ T dropped(T x, bool keep, float scale, T residual) {
  const float r = RESIDUAL ? to_f32(residual) : 0.0f;
  const float v = RESIDUAL ? fmaf(to_f32(x), scale, r) : to_f32(x) * scale;
  return from_f32<T>(keep ? v : r);
}

// Rows without a gap between them: one row of n elements.
template <typename T, bool RESIDUAL>
__global__ __launch_bounds__(kBlock) void k_dropout(DropoutArgs a, int64_t n) {
  const uint64_t offset = call_offset(a);
  const T* x = (const T*)a.x;
  const T* r = (const T*)a.residual;
  T* y = (T*)a.y;
  const int64_t blocks = (n + kE - 1) / kE, step = (int64_t)gridDim.x * kBlock;
  for (int64_t b = (int64_t)blockIdx.x * kBlock + threadIdx.x; b < blocks; b += step) {
    const int64_t i = b * kE;
    const Pack<T, kE> in = load_some<T, kE>(x + i, n - i);
    Pack<T, kE> res{};
    if constexpr (RESIDUAL) res = load_some<T, kE>(r + i, n - i);
    const uint32_t keep = kept(a, offset, (uint64_t)b);
    Pack<T, kE> out;
#pragma unroll
    for (int e = 0; e < kE; e++)
      out.v[e] = dropped<RESIDUAL>(in.v[e], (keep >> e & 1) != 0, a.scale, res.v[e]);
    store_some<T, kE>(y + i, n - i, out);
  }
}

// Rows with gaps: a generator's block may lie over the end of a row, or over
// several short ones.
template <typename T, bool RESIDUAL>
__global__ __launch_bounds__(kBlock) void k_dropout_rows(DropoutArgs a, int64_t n,
                                                         Divisor by_cols) {
  const uint64_t offset = call_offset(a);
  const T* x = (const T*)a.x;
  const T* r = (const T*)a.residual;
  T* y = (T*)a.y;
  const int64_t blocks = (n + kE - 1) / kE;
  for (int64_t b0 = (int64_t)blockIdx.x * kBlock; b0 < blocks; b0 += (int64_t)gridDim.x * kBlock) {
    const int64_t b = b0 + threadIdx.x;
    if (b >= blocks) break;
    // from the row of the thread block's first element, which all share
    const int64_t row0 = b0 * kE / a.cols;
    uint32_t col = (uint32_t)(b0 * kE - row0 * a.cols) + threadIdx.x * kE;
    const uint32_t rows = divided(col, by_cols);
    int64_t row = row0 + rows;
    col -= rows * (uint32_t)a.cols;
    const int count = (int)(n - b * kE < kE ? n - b * kE : kE);
    const uint32_t keep = kept(a, offset, (uint64_t)b);
    if (col + count <= (uint32_t)a.cols && count == kE) {
      const Pack<T, kE> in = load_pack<T, kE>(x + row * a.ldx + col);
      Pack<T, kE> res{};
      if constexpr (RESIDUAL) res = load_pack<T, kE>(r + row * a.ldr + col);
      Pack<T, kE> out;
#pragma unroll
      for (int e = 0; e < kE; e++)
        out.v[e] = dropped<RESIDUAL>(in.v[e], (keep >> e & 1) != 0, a.scale, res.v[e]);
      store_pack<T, kE>(y + row * a.ldy + col, out);
    } else {
      // element by element, with all loads under way together; past the end the
      // last one again (65,536 x 290 fp32 with gaps: 46 us one after the other)
      int64_t at_x[kE], at_r[kE], at_y[kE];
#pragma unroll
      for (int e = 0; e < kE; e++) {
        at_x[e] = row * a.ldx + col;
        at_y[e] = row * a.ldy + col;
        at_r[e] = RESIDUAL ? row * a.ldr + col : 0;
        const bool on = e + 1 < count, end = col + 1 == (uint32_t)a.cols;
        row += on && end ? 1 : 0;
        col = on ? (end ? 0 : col + 1) : col;
      }
      T in[kE], res[kE] = {};
#pragma unroll
      for (int e = 0; e < kE; e++) {
        in[e] = x[at_x[e]];
        if constexpr (RESIDUAL) res[e] = r[at_r[e]];
      }
#pragma unroll
      for (int e = 0; e < kE; e++)
        if (e < count)
          y[at_y[e]] = dropped<RESIDUAL>(in[e], (keep >> e & 1) != 0, a.scale, res[e]);
    }
  }
}

template <typename T, bool RESIDUAL>
hipError_t launch(const DropoutArgs& a, hipStream_t s) {
  const int64_t n = (int64_t)a.rows * a.cols;
  const int64_t threads = (n + kE - 1) / kE, most = 1 << 22;
  const int64_t blocks = (threads + kBlock - 1) / kBlock;
  const dim3 grid((unsigned)(blocks < most ? blocks : most));
  const bool flat = a.rows <= 1 || (a.ldx == a.cols && a.ldy == a.cols &&
                                    (!RESIDUAL || a.ldr == a.cols));
  if (flat) {
    hipLaunchKernelGGL((k_dropout<T, RESIDUAL>), grid, dim3(kBlock), 0, s, a, n);
  } else {
    hipLaunchKernelGGL((k_dropout_rows<T, RESIDUAL>), grid, dim3(kBlock), 0, s, a, n,
                       divisor_of((uint32_t)a.cols));
  }
  return hipGetLastError();
}

template <typename T>
hipError_t launch(const DropoutArgs& a, hipStream_t s) {
  return a.residual != nullptr ? launch<T, true>(a, s) : launch<T, false>(a, s);
}

}  // namespace

hipError_t launch_dropout(const DropoutArgs& a, hipStream_t s) {
  switch (a.dtype) {
    case W2V_DTYPE_F32:
      return launch<float>(a, s);
    case W2V_DTYPE_BF16:
      return launch<bf16_t>(a, s);
    default:
      return launch<f16_t>(a, s);
  }
}

}  // namespace w2v
