// Products with a matrix held in 4 bits with a scale for each group of a row:
//
//   y = x W^T + bias,   W_nk = s_n,g(k) (q_nk - 8),   q in 0..15,
//
// for few rows of x: the matrix is read once, which is what the product costs.
// Measured: 16 x 10^6 x 300 fp32 61 us (238 MB at 3.9 TB/s), 61 x 100,000 x 600 fp16 in
// groups of 64 20 to 21 us (44.8 MB, 7.3 GFLOP), 1 x 71,290 x 300 bf16 12 us, 8 of them in
// the kernel.
//
// A wavefront takes tiles of 16 rows of W and multiplies them on 16 x 16 x 32
// matrix instructions, 32 columns at a time, with x as the other operand (16 rows
// a tile, zeros where there are fewer). The layout is made for that: lane 16 q + r
// of a wavefront finds the eight codes of row r that the instruction wants from it
// in one word, the words of four blocks of columns in 16 bytes.
//
// What is multiplied is q - 8, which both 16-bit types hold, so that products are exact
// and a group's sum is rounded as one of fp32 numbers is, in whatever order the
// instruction takes them. (Codes of 16 + q, a shift and an and-or, with a correction of
// -24 sum(x) are 7 instructions fewer a word of bfloat16 and 4 of fp16, but their sums
// are tens of times the result where x has a mean. 384 columns of mean 1 in groups of
// 128: errors of 1.9e-6, 1.9e-6 and 4.3e-6 of the result's size with fp32, bf16 and fp16
// x, so 1.2e-7, 3.6e-8 and 3.9e-8, a product in fp32 3.2e-7, 9e-8 and 2.2e-7. 16 x 10^6 x
// 300 fp32 62 us both ways, bf16 48, so 52.) The group's sum times its scale is added in
// fp32.
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

// One wavefront a tile and group, of which it reads 16 rows of 32 to 128 columns: 10^6 x
// 300 fp32 in groups of 32 in 389 us (1.4 GB at 3.5 TB/s), bf16 380, fp16 in groups of 128
// 271; bound by instruction issue, a division a weight and four blocks whatever the group
// has. Column 8 q + j of a block is in nibble j / 2 of
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

// e4m3 of the codes less 8 in the bytes of q, each 0 to 15. A byte selection takes one
// of eight bytes for 0 to 7, and for 8 to 15 zeros, ones or the sign of a byte, which are
// known. So one looks up the negative numbers and one, by q ^ 8, the others; each table
// is taken exclusive-or with what the other selection gives there.
__device__ __forceinline__ uint32_t numbers_of(uint32_t q) {
  const uint32_t negative = __builtin_amdgcn_perm(0x473F3BC8u, 0x3533CED0u, q);
  const uint32_t others = __builtin_amdgcn_perm(0xB1B3B548u, 0x444038FFu, q ^ 0x08080808u);
  return negative ^ others;
}

// q - 8 for the eight codes of a word: of bfloat16 in the order 0, 4, 1, 5, 2, 6, 3, 7
// of the columns. fp16: 16 + q is 2^4 (1 + q / 16), whose fraction's upper bits are q.
template <typename Vec>
__device__ __forceinline__ Vec codes_of(uint32_t u) {
  if constexpr (__is_same(Vec, f16x8)) {
    uint4 w;
    w.x = (u << 6 & 0x03C003C0u) | 0x4C004C00u;
    w.y = (u << 2 & 0x03C003C0u) | 0x4C004C00u;
    w.z = (u >> 2 & 0x03C003C0u) | 0x4C004C00u;
    w.w = (u >> 6 & 0x03C003C0u) | 0x4C004C00u;
    return __builtin_bit_cast(Vec, w) - (f16_t)24.0f;
  } else {
    const uint32_t low = numbers_of(u & 0x0F0F0F0Fu), high = numbers_of(u >> 4 & 0x0F0F0F0Fu);
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(low, 1.0f, false);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(low, 1.0f, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(high, 1.0f, false);
    const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(high, 1.0f, true);
    return Vec{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
  }
}
// Which of eight columns is in a place of the operands.
template <typename T>
__device__ __forceinline__ constexpr int column_at(int place) {
  return __is_same(T, f16_t) ? place : place / 2 + place % 2 * 4;
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

// Eight 16-bit x, with a NaN among them if there is an infinity: the row becomes NaN
// whatever codes it meets. Products with 0 find it, two in an instruction. (The pieces of
// an infinite fp32 x are that and inf - inf.)
template <typename T>
__device__ __forceinline__ uint4 not_infinite(uint4 x) {
  typedef T Two __attribute__((ext_vector_type(2)));
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  float zero = 0.0f;
#pragma unroll
  for (int i = 0; i < 4; i++) {
    if constexpr (__is_same(T, f16_t)) {
      zero = __builtin_amdgcn_fdot2(__builtin_bit_cast(Two, w[i]), Two{}, zero, false);
    } else {
      zero = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(Two, w[i]), Two{}, zero, false);
    }
  }
  if (zero != zero) x.x |= 0x7FFFu;
  return x;
}

// x in LDS as the instruction wants it, for `blocks` blocks of columns at a time:
// [block][tile of rows][piece][lane] of 16 bytes.
// A wavefront takes kUnits blocks of 16 rows at a time, whose loads are on their way
// together (fewer between products, where the registers are taken); only the end of a
// row is loaded with a test.
template <typename T, int MT, int GB, int WAVES, bool ONCE>
__device__ __forceinline__ void stage(const LinearQ4Args& a, const Q4Shape& q, int m0, int b0,
                                      int blocks, uint4* frags) {
  typedef Operand<T> Op;
  constexpr int kUnits = ONCE ? 4 : GB;
  const int lane = threadIdx.x & 63, r = lane & 15, quad = lane >> 4;
  const int units = blocks * MT;
  const T* x = (const T*)a.x;
  for (int u0 = threadIdx.x >> 6; u0 < units; u0 += WAVES * kUnits) {
    Pack<T, 8> in[kUnits];
    int64_t from[kUnits];
    int there[kUnits];
#pragma unroll
    for (int i = 0; i < kUnits; i++) {
      const int u = u0 + i * WAVES, m = m0 + u % MT * 16 + r;
      const int64_t k = ((int64_t)b0 + u / MT) * 32 + quad * 8;
      const bool some = u < units && m < a.M && k < q.K;
      there[i] = !some ? 0 : q.K - k < 8 ? (int)(q.K - k) : 8;
      from[i] = some ? m * a.ldx + k : 0;
      if (q.K >= 8) in[i] = load_pack<T, 8>(x + (there[i] == 8 ? from[i] : 0));
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < kUnits; i++) {
      const int u = u0 + i * WAVES;
      if (u >= units) break;
      Pack<T, 8> v = in[i];
      if (there[i] < 8) {
        if (there[i] > 0) {
          v = load_some<T, 8>(x + from[i], there[i]);
        } else {
#pragma unroll
          for (int j = 0; j < 8; j++) v.v[j] = T(0.0f);
        }
      }
      uint4* to = frags + (int64_t)u * Op::kPieces * kWave + lane;
      if constexpr (Op::kPieces == 1) {
        Pack<T, 8> placed;
#pragma unroll
        for (int j = 0; j < 8; j++) placed.v[j] = v.v[column_at<T>(j)];
        to[0] = not_infinite<T>(__builtin_bit_cast(uint4, placed));
      } else {
        uint32_t piece[3][8];
#pragma unroll
        for (int j = 0; j < 8; j++) {
          float left = v.v[column_at<T>(j)];
#pragma unroll
          for (int p = 0; p < 3; p++) {
            piece[p][j] = upper(left);
            left -= __builtin_bit_cast(float, piece[p][j] << 16);
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
  }
}

// GB blocks of a group: the words of NT tiles against MT tiles of x.
template <typename T, int MT, int NT, int GB>
__device__ __forceinline__ void add_group(const uint4* frags, int block,
                                          const uint32_t (&word)[NT][GB], const float (&scale)[NT],
                                          f32x4 (&acc)[NT][MT]) {
  typedef Operand<T> Op;
  typedef typename Op::Vec Vec;
  const int lane = threadIdx.x & 63;
  f32x4 part[NT][MT] = {};
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
  for (int mt = 0; mt < MT; mt++)
#pragma unroll
    for (int t = 0; t < NT; t++)
#pragma unroll
      for (int i = 0; i < 4; i++) acc[t][mt][i] = fmaf(scale[t], part[t][mt][i], acc[t][mt][i]);
}

// Cache policy of the words, which are read once: they do not drive x and the scales
// out (1 x 10^6 x 300: 57 to 52 us).
constexpr int kNonTemporal = 2;

// Range-checked access to `bytes` bytes: loads whose lane's offset is past them are 0.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t checked(const void* p, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc((void*)p, (short)0, bytes, 0x00020000);
}

// Four blocks of columns of NT tiles (the last of a row: the rest): a lane's words
// and the scales of its row. Four scales that lie together come in one load, others
// one by one; which it was is only looked at when they are used. What a rest's loads
// take in of other lanes and rows is not used.
template <int NT, int GB>
struct Step {
  word4 w[NT];
  static constexpr int kSingle = 4 / GB < 3 ? 4 / GB : 3;
  uint32_t four[NT][2];
  uint16_t single[NT][kSingle];
  float bias[NT];

  __device__ __forceinline__ float scale(int t, int g, bool whole) const {
    const uint32_t bits = GB == 1 && whole ? four[t][g / 2] >> (16 * (g & 1))
                                           : single[t][g < kSingle ? g : 0];
    return __builtin_bit_cast(float, bits << 16);
  }
};

// Whether the scales of a step that begins with `block` lie in fours.
template <int GB>
__device__ __forceinline__ bool whole_scales(const Q4Shape& q, int block) {
  return q.groups - (block / GB & ~3) >= 4;
}

// The next NT tiles of a wavefront, with what they have of words, scales and bias
// in range: nothing for tiles that there are not.
template <int NT, int GB>
struct Tiles {
  __amdgpu_buffer_rsrc_t words, scales, bias;

  __device__ __forceinline__ void begin(const LinearQ4Args& a, const Q4Shape& q, int64_t tile,
                                        int64_t end) {
    const Q4Range range = q4_range(q, tile, end, NT, a.bias != nullptr);
    words = checked(a.packed + tile * q.blocks * 64, range.words);
    scales = checked((const bf16_t*)a.scales + tile * q.groups * 16, range.scales);
    bias = checked(a.bias + tile * 16, range.bias);
  }
  __device__ __forceinline__ void load(const Q4Shape& q, int block, Step<NT, GB>& step) const {
    const int lane = threadIdx.x & 63, r = lane & 15;
    const int rest = q.blocks - block, group = block / GB;
    const bool whole = whole_scales<GB>(q, block);
    step = Step<NT, GB>{};  // nothing of the step before is kept alive
#pragma unroll
    for (int t = 0; t < NT; t++) {
      const int from = q4_words_at(q, t, block, lane);
      if (rest >= 4) {
        step.w[t] = __builtin_amdgcn_raw_buffer_load_b128(words, from, 0, kNonTemporal);
      } else {
        step.w[t].x = __builtin_amdgcn_raw_buffer_load_b32(words, from, 0, 0);
        step.w[t].y = __builtin_amdgcn_raw_buffer_load_b32(words, from + 4, 0, 0);
        step.w[t].z = __builtin_amdgcn_raw_buffer_load_b32(words, from + 8, 0, 0);
      }
      const int at = q4_scales_at(q, t, group, r);
      if (GB == 1 && whole) {
        const auto four = __builtin_amdgcn_raw_buffer_load_b64(scales, at, 0, 0);
        step.four[t][0] = four[0];
        step.four[t][1] = four[1];
      } else {
#pragma unroll
        for (int g = 0; g < Step<NT, GB>::kSingle; g++)
          step.single[t][g] = __builtin_amdgcn_raw_buffer_load_b16(scales, at + 2 * g, 0, 0);
      }
      // in time for the step that ends the tile; with larger groups a test costs more
      // than the load (61 x 100,000 x 600 in groups of 64: 31 to 29 us)
      if (GB > 1 || rest <= 4)
        step.bias[t] = __builtin_bit_cast(
            float, __builtin_amdgcn_raw_buffer_load_b32(bias, q4_bias_at(t, r), 0, 0));
    }
  }
};

// Wavefronts of a SIMD that the registers are to allow, 128 each. That takes one tile
// of W at a time with several of x (61 x 100,000 x 600 fp16 in groups of 64: 23 us,
// with two at 2 wavefronts 26), and of fp32 x in groups of 128 (1 x 100,000 x 1,000 17
// us, with two 22); else, with one of x, two share its readings from LDS (16 x 10^6 x
// 300 fp32: 61, with one 65).
constexpr int kResident = 4;
constexpr int kAll = 4 * kResident, kHalf = kAll / 2;
constexpr int tiles_at_once(int mt, int pieces, int gb) {
  return mt > 1 || (pieces > 1 && gb == 4) ? 1 : 2;
}

// One block: NT tiles of W at a time and wavefront, against MT tiles of x
// (blockIdx.y). `span` blocks of columns of x are in LDS at once; where that is all of
// them (ONCE) they are put there once, and the wavefronts do not wait for each other.
// A wavefront goes through the steps of all its tiles with the next one's loads on
// their way.
// Small blocks take sets of neighbouring tiles in turn: W is read in its order (16 x
// 10^6 x 300 fp32 3 us less than with a stretch for each block). Large ones, one a
// CU, take a stretch each, all of one length: 391 sets for 256 blocks would be two
// rounds (61 x 100,000 x 600 fp16 in groups of 64: 23.0 to 21.7 us).
template <typename T, int MT, int NT, int GB, int WAVES, bool ONCE>
__global__ __launch_bounds__(WAVES* kWave, WAVES == kHalf ? kResident / 2 : kResident)
void k_linear_q4(LinearQ4Args a, Q4Shape q, int span) {
  extern __shared__ uint4 frags[];
  const int lane = threadIdx.x & 63, r = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int m0 = blockIdx.y * MT * 16;
  const int64_t b = blockIdx.x;
  int64_t first = b * WAVES * NT, end = q.tiles, step = (int64_t)gridDim.x * WAVES * NT;
  if (WAVES >= kHalf) {
    const int64_t units = (q.tiles + NT - 1) / NT, each = units / gridDim.x;
    const int64_t more = units - each * gridDim.x;
    first = (b * each + (b < more ? b : more)) * NT;
    end = first + (each + (b < more)) * NT;
    if (end > q.tiles) end = q.tiles;
    step = WAVES * NT;
  }
  f32x4 acc[NT][MT] = {};
  // where the loads and the products are, of the wavefront itself or of the block's
  // first one
  const int64_t start = ONCE ? first + wave * NT : first;
  const int own = ONCE ? 0 : wave * NT;
  int64_t load_tile = start, tile0 = start;
  int load_block = 0, block = 0;
  Tiles<NT, GB> tiles;
  tiles.begin(a, q, load_tile + own, end);
  const auto load = [&](Step<NT, GB>& to) {
    tiles.load(q, load_block, to);
    load_block += 4;
    if (load_block >= q.blocks) {
      load_block = 0;
      load_tile += step;
      tiles.begin(a, q, load_tile + own, end);
    }
  };
  const auto add = [&](const Step<NT, GB>& from) {
    const int staged = ONCE ? block : block % span;
    if (!ONCE && staged == 0) {
      __syncthreads();
      stage<T, MT, GB, WAVES, false>(a, q, m0, block, q.blocks - block < span ? q.blocks - block : span,
                                     frags);
      __syncthreads();
    }
    const bool whole = whole_scales<GB>(q, block);
#pragma unroll
    for (int g = 0; g < 4 / GB; g++) {
      if (block + g * GB >= q.blocks) break;
      uint32_t word[NT][GB];
      float scale[NT];
#pragma unroll
      for (int t = 0; t < NT; t++) {
#pragma unroll
        for (int i = 0; i < GB; i++) word[t][i] = from.w[t][g * GB + i];
        scale[t] = from.scale(t, g, whole);
      }
      add_group<T, MT, NT, GB>(frags, staged + g * GB, word, scale, acc);
    }
    block += 4;
    if (block < q.blocks) return;
    const int64_t tile = tile0 + own;
#pragma unroll
    for (int t = 0; t < NT; t++) {
      const int64_t n = (tile + t) * 16 + r;
      if (tile + t < end && n < q.N) {
#pragma unroll
        for (int mt = 0; mt < MT; mt++)
#pragma unroll
          for (int i = 0; i < 4; i++) {
            const int m = m0 + mt * 16 + (lane >> 4) * 4 + i;
            if (m >= a.M) continue;
            const int64_t at = m * a.ldy + n;
            const float v = acc[t][mt][i] + from.bias[t];
            if (a.out_dtype == W2V_DTYPE_F32) {
              store_as<float>(a.y, at, v);
            } else {
              store_as<typename Operand<T>::Element>(a.y, at, v);
            }
          }
      }
#pragma unroll
      for (int mt = 0; mt < MT; mt++) acc[t][mt] = f32x4{};
    }
    block = 0;
    tile0 += step;
  };
  Step<NT, GB> even, odd;
  load(even);
  if (ONCE) {
    stage<T, MT, GB, WAVES, true>(a, q, m0, 0, q.blocks, frags);
    __syncthreads();
  }
  while (tile0 < end) {
    load(odd);
    add(even);
    if (tile0 >= end) break;
    load(even);
    add(odd);
  }
}

constexpr int kMostLds = 128 << 10, kLds = 160 << 10;

// LDS of a block of columns of x.
template <typename T>
constexpr int block_bytes(int mt) {
  return mt * Operand<T>::kPieces * kWave * 16;
}
// Blocks of columns of x that LDS holds.
template <typename T>
constexpr int most_blocks(int mt) {
  return kMostLds / block_bytes<T>(mt) & ~3;
}

template <typename T, int MT, int GB, int WAVES, bool ONCE>
hipError_t launch(const LinearQ4Args& a, const Q4Shape& q, int span, hipStream_t s) {
  constexpr int NT = tiles_at_once(MT, Operand<T>::kPieces, GB);
  const int bytes = span * block_bytes<T>(MT);
  const int64_t sets = (q.tiles + WAVES * NT - 1) / (WAVES * NT);
  // as many blocks as the card holds at once, so that all end at the same time:
  // each puts x into LDS for itself
  const int64_t by_lds = kLds / bytes, by_registers = WAVES == kHalf ? 1 : kAll / WAVES;
  const int64_t fit = 256 * (by_lds < by_registers ? by_lds : by_registers);
  const dim3 grid((unsigned)(sets < fit ? sets : fit), (unsigned)((a.M + MT * 16 - 1) / (MT * 16)));
  if (bytes > (64 << 10)) {
    // the most of any call, since another thread's may lie between this and the launch
    const hipError_t e = hipFuncSetAttribute((const void*)k_linear_q4<T, MT, NT, GB, WAVES, ONCE>,
                                             hipFuncAttributeMaxDynamicSharedMemorySize, kMostLds);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((k_linear_q4<T, MT, NT, GB, WAVES, ONCE>), grid, dim3(WAVES * kWave), bytes,
                     s, a, q, span);
  return hipGetLastError();
}

// Blocks of four wavefronts while LDS holds as many of them as the registers do and has
// room left, else one block of all those wavefronts, which shares its x (1 x 100,000 x
// 1,000 fp32 20 us, with the four that LDS then allows 37; 64 x 100,000 x 300 bf16 15,
// with four that fill it 19). x in parts and groups of 128 take more registers: half the
// wavefronts (16 x 50,000 x 2,000 fp32 24 us, with all 43).
template <typename T, int MT, int GB>
hipError_t launch(const LinearQ4Args& a, const Q4Shape& q, hipStream_t s) {
  const int most = most_blocks<T>(MT);
  if (q.blocks > most) {
    if constexpr (MT == 1 || GB < 4)
      return launch<T, MT, GB, GB == 4 ? kHalf : kAll, false>(a, q, most, s);
    return hipErrorInvalidValue;
  }
  if (q.blocks * block_bytes<T>(MT) < kLds / kResident)
    return launch<T, MT, GB, 4, true>(a, q, q.blocks, s);
  return launch<T, MT, GB, kAll, true>(a, q, q.blocks, s);
}

template <typename T, int MT>
hipError_t launch(const LinearQ4Args& a, const Q4Shape& q, hipStream_t s) {
  switch (q.group) {
    case 32:
      return launch<T, MT, 1>(a, q, s);
    case 64:
      return launch<T, MT, 2>(a, q, s);
    default:
      return launch<T, MT, 4>(a, q, s);
  }
}

// Up to 64 rows of x to a reading of W (32 of fp32, which takes three times the LDS).
// Where these do not fit into LDS x is taken in parts, or half as many rows at a time:
// in groups of 128, for their registers (32 x 100,000 x 1,000 fp32 39 us, in parts
// 47); where that leaves fewer rows over (90 x 71,290 x 2,000 bf16 103 and 122); or
// where it takes more blocks to fill the card (64 x 30,000 x 1,100 bf16 16 and 21;
// else in parts: 64 x 100,000 x 1,100 47 and 41, 64 x 50,000 x 2,000 fp16 in groups of
// 64 39 and 30).
template <typename T>
hipError_t launch(const LinearQ4Args& a, const Q4Shape& q, hipStream_t s) {
  int mt = a.M <= 16 ? 1 : a.M <= 32 || Operand<T>::kPieces > 1 ? 2 : 4;
  const auto parts = [&](int tiles) { return (a.M + tiles * 16 - 1) / (tiles * 16); };
  const auto blocks = [&](int tiles) {
    const int64_t of = kAll * tiles_at_once(tiles, Operand<T>::kPieces, q.group / 32);
    return parts(tiles) * ((q.tiles + of - 1) / of);
  };
  while (mt > 1 && q.blocks > most_blocks<T>(mt)) {
    const bool fewer = 2 * parts(mt) > parts(mt / 2);
    const bool fuller = blocks(mt) < 192 && blocks(mt / 2) > blocks(mt);
    if (q.group < 128 && !fewer && !fuller) break;
    mt /= 2;
  }
  if (mt == 1) return launch<T, 1>(a, q, s);
  if (mt == 2) return launch<T, 2>(a, q, s);
  if constexpr (Operand<T>::kPieces == 1) return launch<T, 4>(a, q, s);
  return hipErrorInvalidValue;
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
