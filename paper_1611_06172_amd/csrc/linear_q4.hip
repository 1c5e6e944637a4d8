// Products with a matrix held in 4 bits with a scale for each group of a row:
//
//   y = x W^T + bias,   W_nk = s_n,g(k) (q_nk - 8),   q in 0..15,
//
// for few rows of x: the matrix is read once, which is what the product costs.
//
// A wavefront takes tiles of 16 rows of W and multiplies them on 16 x 16 x 32
// matrix instructions, 32 columns at a time, with x as the other operand (16 rows
// a tile, zeros where there are fewer). The layout is made for that: lane 16 q + r
// of a wavefront finds the eight codes of row r that the instruction wants from it
// in one word, the words of four blocks of columns in 16 bytes.
//
// A code becomes a 16-bit float by a shift and one and-or: 16 + q is 2^4 (1 + q /
// 16), whose fraction's upper bits are q. The product with x is thus 24 sum(x) too
// large in every group; the accumulator begins at minus that. The products are
// exact and are summed in fp32, and so is the correction, which makes the rounding
// error of a group that of sums of 31 |x| instead of 8 |x|, still 2^-24 of them.
// The group's sum times its scale is added in fp32.
//
// fp32 x is taken apart into three bfloat16 pieces of 8 bits each, which hold all
// of its 24 bits: three instructions for one, and nothing is rounded.
#include "head_types.h"
#include "linear_q4.h"

namespace w2v {
namespace {

constexpr int kWave = 64;
constexpr int kBlock = 256;
constexpr int kWaves = kBlock / kWave;
constexpr int kMaxGrid = 1 << 22;

// Where block b of a tile's columns has lane l's word, from the tile's beginning:
// blocks lie in fours, the rest together.
__host__ __device__ __forceinline__ int64_t word_at(int blocks, int b, int l) {
  const int fours = blocks & ~3;
  return b < fours ? (int64_t)(b >> 2) * 256 + l * 4 + (b & 3)
                   : (int64_t)fours * 64 + l * (blocks - fours) + (b - fours);
}
// The same for the scale of row r's group g.
__host__ __device__ __forceinline__ int64_t scale_at(int groups, int g, int r) {
  const int fours = groups & ~3;
  return g < fours ? (int64_t)(g >> 2) * 64 + r * 4 + (g & 3)
                   : (int64_t)fours * 16 + r * (groups - fours) + (g - fours);
}

// ------------------------------------------------------------ quantisation --

// One wavefront a tile and group. Column 8 q + j of a block is in nibble j / 2 of
// lane 16 q + r's word for even j, 4 + j / 2 for odd j, so that a shift leaves two
// neighbours in the halves of a register. s = max|w| / 7, rounded to bfloat16
// before the codes are taken with it.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_quantize(QuantizeArgs a, Q4Shape q) {
  const int lane = threadIdx.x & 63, r = lane & 15, quad = lane >> 4;
  const int of_group = q.group / 32;
  const int64_t units = q.tiles * q.groups;
  for (int64_t u = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6); u < units;
       u += (int64_t)gridDim.x * kWaves) {
    const int64_t tile = u / q.groups, row = tile * 16 + r;
    const int g = (int)(u - tile * q.groups);
    float v[4][8];
    float most = 0.0f;
    bool finite = true;
#pragma unroll
    for (int b = 0; b < 4; b++) {
      const int64_t k = ((int64_t)g * of_group + b) * 32 + quad * 8;
      const bool some = b < of_group && row < q.N && k < q.K;
      Pack<T, 8> in;
#pragma unroll
      for (int j = 0; j < 8; j++) in.v[j] = T(0.0f);
      if (some) in = load_some<T, 8>((const T*)a.w + row * a.ldw + k, q.K - k);
#pragma unroll
      for (int j = 0; j < 8; j++) {
        v[b][j] = to_f32(in.v[j]);
        most = fmaxf(most, fabsf(v[b][j]));
        finite &= fabsf(v[b][j]) <= 3.402823466e38f;
      }
    }
    most = fmaxf(most, __shfl_xor(most, 16));
    most = fmaxf(most, __shfl_xor(most, 32));
    // all four lanes of a row know of a value that is not finite
    const uint64_t bad = __ballot(!finite);
    const bool spoilt = ((bad >> r | bad >> (r + 16) | bad >> (r + 32) | bad >> (r + 48)) & 1) != 0;
    const bf16_t scale = from_f32<bf16_t>(spoilt ? __builtin_nanf("") : most / 7.0f);
    const float s = to_f32(scale);
#pragma unroll
    for (int b = 0; b < 4; b++) {
      if (b >= of_group) break;
      uint32_t word = 0;
#pragma unroll
      for (int j = 0; j < 8; j++) {
        const float code = s > 0.0f ? fminf(fmaxf(rintf(v[b][j] / s), -8.0f), 7.0f) : 0.0f;
        word |= (uint32_t)((int)code + 8) << (4 * (j / 2 + 4 * (j & 1)));
      }
      a.packed[tile * q.blocks * 64 + word_at(q.blocks, g * of_group + b, lane)] = word;
    }
    if (quad == 0)
      ((bf16_t*)a.scales)[tile * 16 * q.groups + scale_at(q.groups, g, r)] = scale;
  }
}

// ---------------------------------------------------------------- products --

template <typename T>
struct Operand {  // of fp32 x: pieces in bfloat16
  typedef bf16x8 Vec;
  typedef bf16_t Element;
  static constexpr int kPieces = 3;
};
template <>
struct Operand<bf16_t> {
  typedef bf16x8 Vec;
  typedef bf16_t Element;
  static constexpr int kPieces = 1;
};
template <>
struct Operand<f16_t> {
  typedef f16x8 Vec;
  typedef f16_t Element;
  static constexpr int kPieces = 1;
};

// 16 + q for the eight codes of a word.
template <typename Vec>
__device__ __forceinline__ Vec codes_of(uint32_t u) {
  uint4 w;
  if constexpr (__is_same(Vec, f16x8)) {
    w.x = (u << 6 & 0x03C003C0u) | 0x4C004C00u;
    w.y = (u << 2 & 0x03C003C0u) | 0x4C004C00u;
    w.z = (u >> 2 & 0x03C003C0u) | 0x4C004C00u;
    w.w = (u >> 6 & 0x03C003C0u) | 0x4C004C00u;
  } else {
    w.x = (u << 3 & 0x00780078u) | 0x41804180u;
    w.y = (u >> 1 & 0x00780078u) | 0x41804180u;
    w.z = (u >> 5 & 0x00780078u) | 0x41804180u;
    w.w = (u >> 9 & 0x00780078u) | 0x41804180u;
  }
  return __builtin_bit_cast(Vec, w);
}

__device__ __forceinline__ f32x4 multiply(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 multiply(f16x8 a, f16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// The upper 16 bits of v: the piece that is taken off, never larger than v.
__device__ __forceinline__ uint32_t upper(float v) {
  return __builtin_bit_cast(uint32_t, v) >> 16;
}

template <typename T>
__device__ __forceinline__ void store_as(void* y, int64_t at, float v) {
  ((T*)y)[at] = from_f32<T>(v);
}

// x in LDS as the instruction wants it, for `blocks` blocks of columns at a time:
// [block][tile of rows][piece][lane] of 16 bytes, and behind these -24 sum(x) of
// each group and row.
template <typename T, int MT, int GB>
__device__ __forceinline__ void stage(const LinearQ4Args& a, const Q4Shape& q, int m0, int b0,
                                      int blocks, uint4* frags, float* sums) {
  typedef Operand<T> Op;
  const int lane = threadIdx.x & 63, r = lane & 15, quad = lane >> 4;
  for (int u = threadIdx.x >> 6; u < blocks / GB * MT; u += kWaves) {
    const int g = u / MT, mt = u % MT, m = m0 + mt * 16 + r;
    float sum = 0.0f;
#pragma unroll
    for (int b = 0; b < GB; b++) {
      const int block = g * GB + b;
      const int64_t k = ((int64_t)b0 + block) * 32 + quad * 8;
      Pack<T, 8> in;
#pragma unroll
      for (int j = 0; j < 8; j++) in.v[j] = T(0.0f);
      if (m < a.M && k < q.K) in = load_some<T, 8>((const T*)a.x + m * a.ldx + k, q.K - k);
      uint4* to = frags + ((block * MT + mt) * Op::kPieces) * kWave + lane;
      if constexpr (Op::kPieces == 1) {
        to[0] = __builtin_bit_cast(uint4, in);
#pragma unroll
        for (int j = 0; j < 8; j++) sum += to_f32(in.v[j]);
      } else {
        uint32_t piece[3][8];
#pragma unroll
        for (int j = 0; j < 8; j++) {
          float v = in.v[j];
          sum += v;
#pragma unroll
          for (int p = 0; p < 3; p++) {
            piece[p][j] = upper(v);
            v -= __builtin_bit_cast(float, piece[p][j] << 16);
          }
        }
#pragma unroll
        for (int p = 0; p < 3; p++) {
          uint32_t w[4];
#pragma unroll
          for (int j = 0; j < 4; j++) w[j] = piece[p][2 * j] | piece[p][2 * j + 1] << 16;
          to[p * kWave] = make_uint4(w[0], w[1], w[2], w[3]);
        }
      }
    }
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    if (quad == 0) sums[(g * MT + mt) * 16 + r] = -24.0f * sum;
  }
}

// GB blocks of a group: the words of NT tiles against MT tiles of x.
template <typename T, int MT, int NT, int GB>
__device__ __forceinline__ void add_group(const uint4* frags, const float* sums, int block,
                                          const uint32_t (&word)[NT][GB], const float (&scale)[NT],
                                          f32x4 (&acc)[NT][MT]) {
  typedef Operand<T> Op;
  typedef typename Op::Vec Vec;
  const int lane = threadIdx.x & 63;
  f32x4 part[NT][MT];
#pragma unroll
  for (int mt = 0; mt < MT; mt++) {
    const f32x4 first = *(const f32x4*)(sums + (block / GB * MT + mt) * 16 + (lane >> 4) * 4);
#pragma unroll
    for (int t = 0; t < NT; t++) part[t][mt] = first;
  }
#pragma unroll
  for (int b = 0; b < GB; b++) {
    Vec w[NT];
#pragma unroll
    for (int t = 0; t < NT; t++) w[t] = codes_of<Vec>(word[t][b]);
#pragma unroll
    for (int mt = 0; mt < MT; mt++)
#pragma unroll
      for (int p = 0; p < Op::kPieces; p++) {
        const Vec x = __builtin_bit_cast(
            Vec, frags[(((block + b) * MT + mt) * Op::kPieces + p) * kWave + lane]);
#pragma unroll
        for (int t = 0; t < NT; t++) part[t][mt] = multiply(x, w[t], part[t][mt]);
      }
  }
#pragma unroll
  for (int t = 0; t < NT; t++)
#pragma unroll
    for (int mt = 0; mt < MT; mt++)
#pragma unroll
      for (int i = 0; i < 4; i++) acc[t][mt][i] = fmaf(scale[t], part[t][mt][i], acc[t][mt][i]);
}

// The blocks [b0, b0 + blocks) of NT tiles; `words` and `scales` are the first
// tile's, `next` tiles on (0 where there is no second one).
template <typename T, int MT, int NT, int GB>
__device__ __forceinline__ void add_blocks(const Q4Shape& q, const uint32_t* words,
                                           const bf16_t* scales, int next, int b0, int blocks,
                                           const uint4* frags, const float* sums,
                                           f32x4 (&acc)[NT][MT]) {
  const int lane = threadIdx.x & 63, r = lane & 15;
  const int64_t word_step = (int64_t)next * q.blocks * 64, scale_step = (int64_t)next * q.groups * 16;
  int b = 0;
  for (; b + 4 <= blocks; b += 4) {
    uint4 w[NT];
    float s[NT][4 / GB];
#pragma unroll
    for (int t = 0; t < NT; t++) {
      w[t] = load_16(words + t * word_step + (int64_t)((b0 + b) >> 2) * 256 + lane * 4);
#pragma unroll
      for (int g = 0; g < 4 / GB; g++)
        s[t][g] = to_f32(scales[t * scale_step + scale_at(q.groups, (b0 + b) / GB + g, r)]);
    }
#pragma unroll
    for (int g = 0; g < 4 / GB; g++) {
      uint32_t word[NT][GB];
      float scale[NT];
#pragma unroll
      for (int t = 0; t < NT; t++) {
        const uint32_t four[4] = {w[t].x, w[t].y, w[t].z, w[t].w};
#pragma unroll
        for (int i = 0; i < GB; i++) word[t][i] = four[g * GB + i];
        scale[t] = s[t][g];
      }
      add_group<T, MT, NT, GB>(frags, sums, b + g * GB, word, scale, acc);
    }
  }
  // the rest of a row's blocks: none where a group has four
  if constexpr (GB < 4) {
    for (; b < blocks; b += GB) {
      uint32_t word[NT][GB];
      float scale[NT];
#pragma unroll
      for (int t = 0; t < NT; t++) {
#pragma unroll
        for (int i = 0; i < GB; i++)
          word[t][i] = words[t * word_step + word_at(q.blocks, b0 + b + i, lane)];
        scale[t] = to_f32(scales[t * scale_step + scale_at(q.groups, (b0 + b) / GB, r)]);
      }
      add_group<T, MT, NT, GB>(frags, sums, b, word, scale, acc);
    }
  }
}

// One block: sets of kWaves x NT tiles of W, against MT tiles of x (blockIdx.y).
// `span` blocks of columns are in LDS at once; where that is all of them they are
// put there once.
template <typename T, int MT, int NT, int GB>
__global__ __launch_bounds__(kBlock) void k_linear_q4(LinearQ4Args a, Q4Shape q, int span) {
  extern __shared__ uint4 frags[];
  float* sums = (float*)(frags + (int64_t)span * MT * Operand<T>::kPieces * kWave);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15;
  const int m0 = blockIdx.y * MT * 16;
  const bool once = span >= q.blocks;
  if (once) {
    stage<T, MT, GB>(a, q, m0, 0, q.blocks, frags, sums);
    __syncthreads();
  }
  const int64_t sets = (q.tiles + kWaves * NT - 1) / (kWaves * NT);
  for (int64_t set = blockIdx.x; set < sets; set += gridDim.x) {
    const int64_t tile = (set * kWaves + wave) * NT;
    const bool any = tile < q.tiles;
    const uint32_t* words = a.packed + (any ? tile : 0) * q.blocks * 64;
    const bf16_t* scales = (const bf16_t*)a.scales + (any ? tile : 0) * q.groups * 16;
    const int next = tile + 1 < q.tiles ? 1 : 0;
    f32x4 acc[NT][MT] = {};
    if (once) {
      if (any)
        add_blocks<T, MT, NT, GB>(q, words, scales, next, 0, q.blocks, frags, sums, acc);
    } else {
      for (int b0 = 0; b0 < q.blocks; b0 += span) {
        const int blocks = q.blocks - b0 < span ? q.blocks - b0 : span;
        __syncthreads();
        stage<T, MT, GB>(a, q, m0, b0, blocks, frags, sums);
        __syncthreads();
        if (any) add_blocks<T, MT, NT, GB>(q, words, scales, next, b0, blocks, frags, sums, acc);
      }
    }
#pragma unroll
    for (int t = 0; t < NT; t++) {
      const int64_t n = (tile + t) * 16 + r;
      if (n >= q.N) continue;
      const float bias = a.bias != nullptr ? a.bias[n] : 0.0f;
#pragma unroll
      for (int mt = 0; mt < MT; mt++)
#pragma unroll
        for (int i = 0; i < 4; i++) {
          const int m = m0 + mt * 16 + (lane >> 4) * 4 + i;
          if (m >= a.M) continue;
          const int64_t at = m * a.ldy + n;
          const float v = acc[t][mt][i] + bias;
          if (a.out_dtype == W2V_DTYPE_F32) {
            store_as<float>(a.y, at, v);
          } else {
            store_as<typename Operand<T>::Element>(a.y, at, v);
          }
        }
    }
  }
}

constexpr int kMostLds = 128 << 10;

template <typename T, int MT, int NT, int GB>
hipError_t launch(const LinearQ4Args& a, const Q4Shape& q, hipStream_t s) {
  constexpr int kBlockBytes = MT * Operand<T>::kPieces * kWave * 16 + MT * 16 * 4 / GB;
  const int most = kMostLds / kBlockBytes & ~3;
  const int span = q.blocks < most ? q.blocks : most;
  const int bytes = span * kBlockBytes + 64;
  const int64_t sets = (q.tiles + kWaves * NT - 1) / (kWaves * NT);
  // as many blocks as the card holds at once: each puts x into LDS for itself
  const int64_t held = (160 << 10) / bytes, fit = 256 * (held < 6 ? held : 6);
  const dim3 grid((unsigned)(sets < fit ? sets : fit), (unsigned)((a.M + MT * 16 - 1) / (MT * 16)));
  if (bytes > (64 << 10)) {
    const hipError_t e = hipFuncSetAttribute((const void*)k_linear_q4<T, MT, NT, GB>,
                                             hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((k_linear_q4<T, MT, NT, GB>), grid, dim3(kBlock), bytes, s, a, q, span);
  return hipGetLastError();
}

template <typename T, int MT, int NT>
hipError_t launch(const LinearQ4Args& a, const Q4Shape& q, hipStream_t s) {
  switch (q.group) {
    case 32:
      return launch<T, MT, NT, 1>(a, q, s);
    case 64:
      return launch<T, MT, NT, 2>(a, q, s);
    default:
      return launch<T, MT, NT, 4>(a, q, s);
  }
}

template <typename T>
hipError_t launch(const LinearQ4Args& a, const Q4Shape& q, hipStream_t s) {
  if (a.M <= 16) return launch<T, 1, 2>(a, q, s);
  if (a.M <= 32 || Operand<T>::kPieces > 1) return launch<T, 2, 2>(a, q, s);
  return launch<T, 4, 2>(a, q, s);
}

}  // namespace

hipError_t launch_quantize_q4(const QuantizeArgs& a, const Q4Shape& q, hipStream_t s) {
  const int64_t blocks = (q.tiles * q.groups + kWaves - 1) / kWaves;
  const dim3 grid((unsigned)(blocks < kMaxGrid ? blocks : kMaxGrid));
  switch (a.dtype) {
    case W2V_DTYPE_F32:
      hipLaunchKernelGGL(k_quantize<float>, grid, dim3(kBlock), 0, s, a, q);
      break;
    case W2V_DTYPE_BF16:
      hipLaunchKernelGGL(k_quantize<bf16_t>, grid, dim3(kBlock), 0, s, a, q);
      break;
    default:
      hipLaunchKernelGGL(k_quantize<f16_t>, grid, dim3(kBlock), 0, s, a, q);
  }
  return hipGetLastError();
}

hipError_t launch_linear_q4(const LinearQ4Args& a, const Q4Shape& q, hipStream_t s) {
  switch (a.dtype) {
    case W2V_DTYPE_F32:
      return launch<float>(a, q, s);
    case W2V_DTYPE_BF16:
      return launch<bf16_t>(a, q, s);
    default:
      return launch<f16_t>(a, q, s);
  }
}

}  // namespace w2v
