// Kernels of the vocabulary head's matrix products and their launches, for
// one element type: each linear_<type>.hip is these for its type.
//   y = act(x W^T + b) + r and its backward pass (dz = dy act'(z), dx = dz W,
//   dW = dz^T x, db = column sums of dz), with fp32 accumulation and one
//   rounding per output element.
#pragma once

#include "head_types.h"
#include "linear_plan.h"

namespace w2v {
namespace {

constexpr int kThreads = 256;
// A block's share of C[m][n] = sum_k A(m, k) B(n, k). An operand whose k runs
// along memory (kc) holds element (r, k) at p[r ld + k], the other kind at
// p[k ld + r].
struct ProductArgs {
  const void* a;
  const void* b;
  int64_t lda, ldb;
  int32_t M, N, K;
  int32_t tiles_m, tiles_n, splits, k_per_split;  // k tiles of a split
  const float* bias;
  const void* residual;
  void* y;
  void* pre;
  int64_t ldr, ldy, ldp;
  int32_t activation;
  float* partial;       // [splits][M][N] where splits > 1
  float* row_sums;      // sums of A over k, or NULL: float [M]
  float* partial_sums;  // [splits][M] where splits > 1
};

template <typename T>
struct Matrix;  // MFMA of one 16-byte granule per lane
template <>
struct Matrix<float> {
  static constexpr int kGranule = 4;
  static __device__ __forceinline__ f32x16 mac32(uint4 a, uint4 b, f32x16 c) {
    const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
    for (int j = 0; j < 4; j++) c = __builtin_amdgcn_mfma_f32_32x32x2f32(x[j], y[j], c, 0, 0, 0);
    return c;
  }
  static __device__ __forceinline__ f32x4 mac16(uint4 a, uint4 b, f32x4 c) {
    const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
    for (int j = 0; j < 4; j++) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[j], y[j], c, 0, 0, 0);
    return c;
  }
};
template <>
struct Matrix<bf16_t> {
  static constexpr int kGranule = 8;
  static __device__ __forceinline__ f32x16 mac32(uint4 a, uint4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x4 mac16(uint4 a, uint4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};
template <>
struct Matrix<f16_t> {
  static constexpr int kGranule = 8;
  static __device__ __forceinline__ f32x16 mac32(uint4 a, uint4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x4 mac16(uint4 a, uint4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
};

// Where granule g of a tile row r of G granules lies. Reads take one granule
// column over 32 consecutive rows, the transposing writes one column over rows
// four apart; the columns are turned so that 8 neighbouring lanes of a read
// fall on all 8 granules of 128 bytes, and those of a write on at least 4.
template <int G>
__device__ __forceinline__ int granule_at(int r, int g) {
  return G == 8 ? r * 8 + (g ^ ((r ^ (r >> 3)) & 7)) : r * 4 + (g ^ (((r >> 1) ^ (r >> 3)) & 3));
}

// N elements at `at`, of which the last `past` are beyond the end of a row of
// `length` and become 0. They are read 16 bytes up to the end and moved down: no
// lane waits for single elements. They are moved by halves of words and by words,
// not as one 128-bit number: a 64-bit shift whose amount lies in the last register
// of a wave's allocation takes another amount on this GPU, and the compiler did
// put it there.
template <typename T, int N>
__device__ __forceinline__ uint4 load_end(const T* at, int past, int length) {
  if (length < N) return __builtin_bit_cast(uint4, load_some<T, N>(at, N - past));
  const int by = past > 0 ? past : 0;
  const uint4 in = load_16(at - by);
  uint32_t a = in.x, b = in.y, c = in.z, d = in.w;
  int words = by;
  if constexpr (sizeof(T) == 2) {
    words = by >> 1;
    const bool half = by & 1;
    a = half ? a >> 16 | b << 16 : a;
    b = half ? b >> 16 | c << 16 : b;
    c = half ? c >> 16 | d << 16 : c;
    d = half ? d >> 16 : d;
  }
  const bool one = words & 1, two = words & 2, all = by >= N;
  a = one ? b : a;
  b = one ? c : b;
  c = one ? d : c;
  d = one ? 0 : d;
  a = two ? c : a;
  b = two ? d : b;
  return make_uint4(all ? 0 : a, all ? 0 : b, all || two ? 0 : c, all || two ? 0 : d);
}

// One operand's tile, ROWS rows by G granules of k, on its way through
// registers into LDS, and back into MFMA operands. Elements past the
// operand's edge in k are 0, and so are (or repeat the last row) those past
// its edge in rows, whose products are not stored.
//
// k runs along memory: granules of k, as the MFMA wants them.
template <typename T, bool KC, int ROWS, int G>
struct Stage {
  static constexpr int GE = Matrix<T>::kGranule, BK = GE * G;
  static constexpr int kPer = ROWS * G / kThreads;
  static_assert(ROWS * G % kThreads == 0, "whole turns");
  uint4 r[kPer];
  const T* at[kPer];

  // The tiles are loaded one after the other from k0 on.
  __device__ __forceinline__ void begin(const T* p, int64_t ld, int row0, int rows, int k0,
                                        int tid) {
#pragma unroll
    for (int i = 0; i < kPer; i++) {
      const int u = tid + i * kThreads;
      at[i] = p + (int64_t)min(row0 + u / G, rows - 1) * ld + k0 + u % G * GE;
    }
  }
  // A tile that does not hold the operand's last k.
  __device__ __forceinline__ void load_next(int64_t) {
#pragma unroll
    for (int i = 0; i < kPer; i++) {
      r[i] = load_16(at[i]);
      at[i] += BK;
    }
  }
  // Any tile; it begins at k0.
  __device__ __forceinline__ void load_any(int64_t, int, int, int k0, int K, int tid) {
#pragma unroll
    for (int i = 0; i < kPer; i++) {
      const int k = k0 + (tid + i * kThreads) % G * GE;
      r[i] = load_end<T, GE>(at[i], k + GE - K, K);
      at[i] += BK;
    }
  }
  __device__ __forceinline__ void store(uint4* lds, int tid) const {
#pragma unroll
    for (int i = 0; i < kPer; i++) {
      const int u = tid + i * kThreads;
      lds[granule_at<G>(u / G, u % G)] = r[i];
    }
  }
  // The operand of rows r0 .. r0 + 31 and granules g, g + 1 of k.
  static __device__ __forceinline__ uint4 read(const uint4* lds, int r0, int g, int lane) {
    return lds[granule_at<G>(r0 + (lane & 31), g + (lane >> 5))];
  }
  static constexpr int kSums = 1;
  __device__ __forceinline__ void add_rows(float*, int) const {}
  static __device__ __forceinline__ void put_sums(const float*, float*, int) {}
  static constexpr int kSumParts = 1;
};

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// Rows run along memory: the tile lies in LDS as in memory, row k of the tile
// after row k - 1, and is turned when it is read. 4-byte elements are read one
// by one, 32 neighbours by each half of the wave. 2-byte ones go through the
// transposing LDS read: of each 16 lanes, lane 4 i + q gives the address of 4
// elements q of k row i and lane j receives column j of the 4 x 16 block.
// Pieces of 32 elements of a k row are exchanged so that the k rows which are
// read at once (k and k + 4; 4 neighbouring ones) meet all LDS banks.
template <typename T, int ROWS, int G>
struct Stage<T, false, ROWS, G> {
  static constexpr int GE = Matrix<T>::kGranule, BK = GE * G;
  static constexpr int kWide = ROWS / GE;   // granules of a k row
  static constexpr int kPiece = 32 / GE;    // granules of a piece
  static constexpr int kPer = BK * kWide / kThreads;
  static_assert(BK * kWide % kThreads == 0 && kThreads % kWide == 0, "whole turns");
  uint4 r[kPer];
  const T* at[kPer];

  static __device__ __forceinline__ int turned(int k, int piece) {
    if (sizeof(T) == 4) return piece ^ ((k >> 2) & 1);
    return piece ^ (ROWS == 128 ? k & 3 : (k >> 1) & 1);
  }
  __device__ __forceinline__ void begin(const T* p, int64_t ld, int row0, int rows, int k0,
                                        int tid) {
#pragma unroll
    for (int i = 0; i < kPer; i++) {
      const int u = tid + i * kThreads, m = row0 + u % kWide * GE;
      at[i] = p + (int64_t)(k0 + u / kWide) * ld + (m < rows ? m : 0);
    }
  }
  // A granule that the edge of the rows cuts is read whole: what lies past the
  // edge is the row's padding or the next k row, which is there because the
  // tile does not hold the last one.
  __device__ __forceinline__ void load_next(int64_t ld) {
#pragma unroll
    for (int i = 0; i < kPer; i++) {
      r[i] = load_16(at[i]);
      at[i] += BK * ld;
    }
  }
  __device__ __forceinline__ void load_any(int64_t ld, int row0, int rows, int k0, int K,
                                           int tid) {
#pragma unroll
    for (int i = 0; i < kPer; i++) {
      const int u = tid + i * kThreads, m = row0 + u % kWide * GE;
      r[i] = make_uint4(0, 0, 0, 0);
      if (k0 + u / kWide < K && m < rows) r[i] = load_end<T, GE>(at[i], m + GE - rows, rows);
      at[i] += BK * ld;
    }
  }
  __device__ __forceinline__ void store(uint4* lds, int tid) const {
#pragma unroll
    for (int i = 0; i < kPer; i++) {
      const int u = tid + i * kThreads, g = u % kWide, k = u / kWide;
      lds[k * kWide + turned(k, g / kPiece) * kPiece + g % kPiece] = r[i];
    }
  }
  static __device__ __forceinline__ uint4 read(const uint4* lds, int r0, int g, int lane) {
    if constexpr (sizeof(T) == 4) {
      const int k = (g + (lane >> 5)) * 4;
      const float* at = (const float*)(lds + k * kWide) + turned(k, r0 >> 5) * 32 + (lane & 31);
      f32x4 out;
#pragma unroll
      for (int j = 0; j < 4; j++) out[j] = at[j * ROWS];
      return __builtin_bit_cast(uint4, out);
    } else {
      const int k = (g + (lane >> 5)) * 8 + ((lane & 15) >> 2);
      const int col = (lane & 16) + (lane & 3) * 4;
      union {
        s16x4 half[2];
        uint4 whole;
      } out;
#pragma unroll
      for (int h = 0; h < 2; h++) {
        const char* at = (const char*)(lds + (k + 4 * h) * kWide) +
                         turned(k + 4 * h, r0 >> 5) * 64 + col * 2;
        out.half[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at);
      }
      return out.whole;
    }
  }
  // Sums of the tile's rows over k: a thread's granules are of the same rows.
  static constexpr int kSums = GE, kSumParts = kThreads / kWide;
  __device__ __forceinline__ void add_rows(float* sums, int) const {
#pragma unroll
    for (int i = 0; i < kPer; i++) {
      const Pack<T, GE> v = __builtin_bit_cast(Pack<T, GE>, r[i]);
#pragma unroll
      for (int c = 0; c < GE; c++) sums[c] += to_f32(v.v[c]);
    }
  }
  static __device__ __forceinline__ void put_sums(const float* sums, float* part, int tid) {
#pragma unroll
    for (int c = 0; c < GE; c++) part[tid / kWide * ROWS + tid % kWide * GE + c] = sums[c];
  }
};

// bias, activation, residual and the rounding of the first n (1..N) of N
// neighbouring elements of one row. FULL: all of them, otherwise the bias.
template <typename T, typename TO, int N, bool FULL>
__device__ __forceinline__ void finish(const ProductArgs& a, int64_t m, int col, int n,
                                       Pack<float, N> z, const Pack<float, N>& bias) {
  if (a.y == nullptr) return;  // only the row sums are wanted
  if (a.bias != nullptr) {
#pragma unroll
    for (int i = 0; i < N; i++) z.v[i] += bias.v[i];
  }
  if constexpr (FULL) {
    Pack<TO, N> residual = {};
    if (a.residual != nullptr)
      residual = load_some<TO, N>((const TO*)a.residual + m * a.ldr + col, n);
    if (a.pre != nullptr) {
      Pack<T, N> out;
#pragma unroll
      for (int i = 0; i < N; i++) out.v[i] = from_f32<T>(z.v[i]);
      store_some<T, N>((T*)a.pre + m * a.ldp + col, n, out);
    }
    if (a.activation != W2V_ACTIVATION_NONE) {
#pragma unroll
      for (int i = 0; i < N; i++) z.v[i] = activate<sizeof(TO) == 2>(z.v[i], a.activation);
    }
    if (a.residual != nullptr) {
#pragma unroll
      for (int i = 0; i < N; i++) z.v[i] += to_f32(residual.v[i]);
    }
  }
  Pack<TO, N> out;
#pragma unroll
  for (int i = 0; i < N; i++) out.v[i] = from_f32<TO>(z.v[i]);
  store_some<TO, N>((TO*)a.y + m * a.ldy + col, n, out);
}

// The same with the bias still in memory.
template <typename T, typename TO, int N>
__device__ __forceinline__ void finish(const ProductArgs& a, int64_t m, int col, int n,
                                       const Pack<float, N>& z) {
  Pack<float, N> bias = {};
  if (a.bias != nullptr) bias = load_some<float, N>(a.bias + col, n);
  finish<T, TO, N, true>(a, m, col, n, z, bias);
}

// Orders a wave's own LDS accesses, which the hardware performs in order.
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Tile and split of the block. Blocks go round the 8 XCDs: each XCD gets a
// contiguous range of the tiles, so that its L2 sees neighbours; within it
// panels of 16 tiles in m are walked along n, split after split.
__device__ __forceinline__ void tile_of(const ProductArgs& a, int& tm, int& tn, int& split) {
  const int tiles = a.tiles_m * a.tiles_n, total = tiles * a.splits;
  const int per = total / 8, extra = total % 8, xcd = blockIdx.x % 8;
  int t = xcd * per + min(xcd, extra) + (int)blockIdx.x / 8;
  split = t / tiles;
  t -= split * tiles;
  const int panel = 16 * a.tiles_n;
  const int first = t / panel * 16, height = min(16, a.tiles_m - first);
  const int in = t % panel;
  tm = first + in % height;
  tn = in / height;
}

// One block of 2 x 2 waves, each (32 TM) x (32 TN) of a tile in 32 x 32 MFMA
// blocks. Operands come through registers into two LDS buffers of G granules
// of k: the next one's loads are in flight while this one is multiplied, and
// the PER_CU blocks of a CU fill each other's waits.
// FULL: an epilogue with activation, residual or pre; otherwise with a bias.
// Blocks of 128 x 128 with 64 bytes of k are the largest that leave room for
// four on a CU. With one 256-wide block on it, a k of 300 is over before its
// pipeline is full: bf16 4,096 x 71,290 x 300 617 us against 549 (both before
// the loads lost their branch).
// Measured, in traces: bf16 4,096 x 71,290 x 300 410 us and up (427 TFLOP/s,
// output at 1.4 TB/s), its gradients with 8,191 rows 894 us and up (dx, 392
// TFLOP/s) and 808 (dW, 434); 65,536 x 300 x 300 with bias, gelu and residual 62;
// fp32 512 x 10^6 x 300 2,542 and up (121 TFLOP/s, a library product of 8,192^3
// has 153). 16 bits are bound by waits: at a k of ten tiles the waves wait for
// memory, LDS and each other in 52 to 66% of their cycles, while MFMA is busy in
// 19 to 21% of the SIMDs' (10% with the whole epilogue) and LDS in 26 to 38% of the
// CUs'. fp32 is bound by MFMA, busy in 78%.
template <typename T, typename TO, bool AKC, bool BKC, bool FULL, int TM, int TN, int G,
          int PER_CU>
__global__ __launch_bounds__(kThreads, PER_CU) void k_product(ProductArgs a) {
  constexpr int BM = 64 * TM, BN = 64 * TN, BK = Matrix<T>::kGranule * G;
  constexpr int kTile = (BM + BN) * G;  // granules of one buffer
  constexpr int kOut = 32 * TN + (TN == 1 ? 4 : 0);  // floats of a staged output row
  constexpr int kStage = 4 * 32 * kOut / 4;
  __shared__ __align__(16) uint4 lds[2 * kTile > kStage ? 2 * kTile : kStage];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wm = wave >> 1, wn = wave & 1;
  int tm, tn, split;
  tile_of(a, tm, tn, split);
  const int m0 = tm * BM, n0 = tn * BN;
  const int k_tiles = (a.K + BK - 1) / BK;
  const int first = split * a.k_per_split, last = min(k_tiles, first + a.k_per_split);

  typedef Stage<T, AKC, BM, G> StageA;
  typedef Stage<T, BKC, BN, G> StageB;
  StageA sa;
  StageB sb;
  float sums[StageA::kSums] = {};
  const bool want_sums = !AKC && a.row_sums != nullptr && tn == 0;
  auto load_any = [&](int k) {
    sa.load_any(a.lda, m0, a.M, k * BK, a.K, tid);
    sb.load_any(a.ldb, n0, a.N, k * BK, a.K, tid);
  };
  auto load_next = [&]() {
    sa.load_next(a.lda);
    sb.load_next(a.ldb);
  };
  auto store = [&](int to) {
    sa.store(lds + to * kTile, tid);
    sb.store(lds + to * kTile + BM * G, tid);
    if (want_sums) sa.add_rows(sums, tid);
  };
  f32x16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; i++)
#pragma unroll
    for (int j = 0; j < TN; j++)
#pragma unroll
      for (int e = 0; e < 16; e++) acc[i][j][e] = 0.0f;
  auto multiply = [&](int buffer) {
    const uint4* from = lds + buffer * kTile;
#pragma unroll
    for (int g = 0; g < G; g += 2) {
      uint4 fa[TM], fb[TN];
#pragma unroll
      for (int i = 0; i < TM; i++) fa[i] = StageA::read(from, (wm * TM + i) * 32, g, lane);
#pragma unroll
      for (int j = 0; j < TN; j++)
        fb[j] = StageB::read(from + BM * G, (wn * TN + j) * 32, g, lane);
#pragma unroll
      for (int i = 0; i < TM; i++)
#pragma unroll
        for (int j = 0; j < TN; j++) acc[i][j] = Matrix<T>::mac32(fa[i], fb[j], acc[i][j]);
    }
  };
  // Tiles before the last k are loaded without a test (rows of a few elements
  // excepted, past whose end a granule would reach too far); a branch around
  // the loads would wait for them at its end.
  const int whole =
      a.lda < StageA::GE || a.ldb < StageB::GE ? 0 : min(max((a.K - 1) / BK - first, 0), last - first);
  sa.begin((const T*)a.a, a.lda, m0, a.M, first * BK, tid);
  sb.begin((const T*)a.b, a.ldb, n0, a.N, first * BK, tid);
  if (whole > 0)
    load_next();
  else
    load_any(first);
  store(0);
  __syncthreads();
  int buffer = 0, k = first + 1;
  for (; k < first + whole; k++) {
    load_next();
    multiply(buffer);
    store(buffer ^ 1);
    __syncthreads();
    buffer ^= 1;
  }
  for (; k < last; k++) {
    load_any(k);
    multiply(buffer);
    store(buffer ^ 1);
    __syncthreads();
    buffer ^= 1;
  }
  multiply(buffer);
  __syncthreads();  // every wave has read its operands

  if (want_sums) {  // uniform over the block
    float* part = (float*)lds;  // [kSumParts][BM]
    static_assert(StageA::kSumParts * BM * 4 <= 2 * kTile * 16, "the sums fit");
    StageA::put_sums(sums, part, tid);
    __syncthreads();
    for (int r = tid; r < BM; r += kThreads) {
      float v = 0.0f;
#pragma unroll
      for (int k = 0; k < StageA::kSumParts; k++) v += part[k * BM + r];
      if (m0 + r < a.M)
        (a.splits > 1 ? a.partial_sums + (int64_t)split * a.M : a.row_sums)[m0 + r] = v;
    }
    __syncthreads();
  }

  // Output: each wave turns 32 rows at a time through its own part of LDS, so
  // that a lane holds neighbouring columns of a row (the MFMA block gives it
  // 16 rows of one column): wide stores and residual loads. Rows 4 to 7 of
  // every 8 have their halves exchanged: the two halves of a wave write to
  // different banks.
  float* stage = (float*)lds + wave * 32 * kOut;
  constexpr int kTurn = TN == 1 ? 0 : 32;
  constexpr int OV = 16 / (int)sizeof(TO);
  constexpr int kLanes = 32 * TN / OV;  // lanes of a row
  constexpr int kRows = 64 / kLanes;    // rows that the wave writes at once
  const int c = (lane % kLanes) * OV, col = n0 + wn * TN * 32 + c, cols = a.N - col;
  Pack<float, OV> bias = {};
  if (a.bias != nullptr && a.splits == 1 && cols > 0)
    bias = load_some<float, OV>(a.bias + col, cols);
#pragma unroll
  for (int i = 0; i < TM; i++) {
#pragma unroll
    for (int j = 0; j < TN; j++)
#pragma unroll
      for (int e = 0; e < 16; e++)
        stage[((e & 3) + 8 * (e >> 2) + 4 * (lane >> 5)) * kOut +
              ((j * 32 + (lane & 31)) ^ (lane >> 5 ? kTurn : 0))] = acc[i][j][e];
    wave_fence();
#pragma unroll FULL ? 1 : 32 / kRows
    for (int r = lane / kLanes; r < 32; r += kRows) {
      const int m = m0 + (wm * TM + i) * 32 + r;
      const Pack<float, OV> z =
          *(const Pack<float, OV>*)(stage + r * kOut + (c ^ (r & 4 ? kTurn : 0)));
      if (m < a.M && cols > 0) {
        if (a.splits > 1)
          store_some<float, OV>(a.partial + ((int64_t)split * a.M + m) * a.N + col, cols, z);
        else
          finish<T, TO, OV, FULL>(a, m, col, cols, z, bias);
      }
    }
    wave_fence();
  }
}

// Joins the partial sums of a product that was split along k, in order.
template <typename T, typename TO>
__global__ __launch_bounds__(kThreads) void k_join(ProductArgs a) {
  const int64_t per_row = (a.N + 3) / 4, units = per_row * a.M;
  const int64_t step = (int64_t)gridDim.x * kThreads;
  const int64_t begin = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  for (int64_t u = begin; u < units; u += step) {
    const int64_t m = u / per_row;
    const int col = (int)(u % per_row) * 4, n = min(4, a.N - col);
    Pack<float, 4> z = {};
    for (int s = 0; s < a.splits; s++) {
      const Pack<float, 4> p =
          load_some<float, 4>(a.partial + ((int64_t)s * a.M + m) * a.N + col, n);
#pragma unroll
      for (int i = 0; i < 4; i++) z.v[i] += p.v[i];
    }
    finish<T, TO, 4>(a, m, col, n, z);
  }
  if (a.row_sums != nullptr) {
    for (int64_t m = begin; m < a.M; m += step) {
      float v = 0.0f;
      for (int s = 0; s < a.splits; s++) v += a.partial_sums[(int64_t)s * a.M + m];
      a.row_sums[m] = v;
    }
  }
}

// Few rows of x (M <= 16): nothing of W is used twice, so W goes from memory
// straight into MFMA registers, 16 of its rows a wave, with x's rows as the
// other operand. Bound by W's bytes: 1 x 71,290 x 200 fp32 12.5 us in a trace,
// 4.6 TB/s, k = 300 17.2 in a graph, 5.0.
template <typename T, typename TO>
__global__ __launch_bounds__(kThreads) void k_few_rows(ProductArgs a) {
  constexpr int GE = Matrix<T>::kGranule, STEP = 4 * GE, U = 4;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int n0 = (blockIdx.x * 4 + wave) * 16;
  if (n0 >= a.N) return;
  const int g = lane >> 4, r = lane & 15;
  const T* w = (const T*)a.b + (int64_t)min(n0 + r, a.N - 1) * a.ldb + g * GE;
  const T* x = (const T*)a.a + (int64_t)min(r, a.M - 1) * a.lda + g * GE;
  f32x4 acc = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  int k = 0;
  for (; k + U * STEP <= a.K; k += U * STEP) {
    uint4 fw[U], fx[U];
#pragma unroll
    for (int u = 0; u < U; u++) {
      fw[u] = __builtin_bit_cast(uint4, load_pack<T, GE>(w + k + u * STEP));
      fx[u] = __builtin_bit_cast(uint4, load_pack<T, GE>(x + k + u * STEP));
    }
#pragma unroll
    for (int u = 0; u < U; u++) acc = Matrix<T>::mac16(fw[u], fx[u], acc);
  }
  for (; k < a.K; k += STEP) {
    const int64_t n = a.K - k - g * GE;
    const uint4 fw = __builtin_bit_cast(uint4, load_some<T, GE>(w + k, n));
    acc = Matrix<T>::mac16(fw, __builtin_bit_cast(uint4, load_some<T, GE>(x + k, n)), acc);
  }
  // lane: columns n0 + 4 g .. + 3 of row r
  const int col = n0 + 4 * g;
  if (r < a.M && col < a.N) {
    Pack<float, 4> z;
#pragma unroll
    for (int i = 0; i < 4; i++) z.v[i] = acc[i];
    finish<T, TO, 4>(a, r, col, min(4, a.N - col), z);
  }
}

// dz = dy act'(z) in 32 bits: a value of its own, not fused with what follows, so
// that both kernels below round the same one.
__device__ __forceinline__ float slope_product(float dy, float z, int activation) {
  float d = dy * activation_slope(z, activation);
  asm("" : "+v"(d));
  return d;
}

// dz = dy act'(z), rounded once to the operands' type: the MFMA operands of
// both gradient products have it. Bound by memory: 4,096 x 600 fp32 8.7 us, 3.4
// TB/s.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_slope(const T* dy, int64_t lddy, const T* pre,
                                                     int64_t ldp, T* dz, int M, int N,
                                                     int activation) {
  constexpr int V = 16 / (int)sizeof(T);
  const int64_t per_row = (N + V - 1) / V, units = per_row * M;
  for (int64_t u = (int64_t)blockIdx.x * kThreads + threadIdx.x; u < units;
       u += (int64_t)gridDim.x * kThreads) {
    const int64_t m = u / per_row;
    const int col = (int)(u % per_row) * V, n = N - col;
    const Pack<T, V> g = load_some<T, V>(dy + m * lddy + col, n);
    const Pack<T, V> z = load_some<T, V>(pre + m * ldp + col, n);
    Pack<T, V> out;
#pragma unroll
    for (int i = 0; i < V; i++)
      out.v[i] = from_f32<T>(slope_product(to_f32(g.v[i]), to_f32(z.v[i]), activation));
    store_some<T, V>(dz + m * N + col, n, out);
  }
}

// The same where dz is of 16 bits and db is wanted: db is no product, so it sums
// dz in fp32 before the rounding. sums: [blocks in y][N]. A block has `rows` rows
// of a stripe `across` packs wide; a thread adds up every down-th row, the block
// its threads in order. 65,536 x 300 bf16 with gelu takes 46 us, 2.6 TB/s beside
// erfcf; 300 x 100,000 with silu 56, 3.2 TB/s; the sums' own sums 4 to 7.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_slope_sums(const T* dy, int64_t lddy,
                                                          const T* pre, int64_t ldp, T* dz,
                                                          int M, int N, int activation,
                                                          int across, int rows, float* sums) {
  constexpr int V = 16 / (int)sizeof(T);
  __shared__ float part[kThreads * V];
  const int tid = threadIdx.x, down = kThreads / across, width = across * V;
  const int lane = tid % across, first = tid / across;
  const int col = (blockIdx.x * across + lane) * V, n = N - col;
  const int m0 = blockIdx.y * rows, count = min(M - m0, rows);
  float total[V] = {};
  if (first < down && n > 0) {
    for (int r = first; r < count; r += down) {
      const int64_t m = m0 + r;
      const Pack<T, V> g = load_some<T, V>(dy + m * lddy + col, n);
      const Pack<T, V> z = load_some<T, V>(pre + m * ldp + col, n);
      Pack<T, V> out;
#pragma unroll
      for (int i = 0; i < V; i++) {
        const float d = slope_product(to_f32(g.v[i]), to_f32(z.v[i]), activation);
        total[i] += d;
        out.v[i] = from_f32<T>(d);
      }
      if (dz != nullptr) store_some<T, V>(dz + m * N + col, n, out);
    }
  }
  if (first < down) {
#pragma unroll
    for (int i = 0; i < V; i++) part[first * width + lane * V + i] = total[i];
  }
  __syncthreads();
  const int at = blockIdx.x * width + tid;
  if (tid < width && at < N) {
    float v = 0.0f;
    for (int d = 0; d < down; d++) v += part[d * width + tid];
    sums[(int64_t)blockIdx.y * N + at] = v;
  }
}

// Adds up `parts` rows of N sums: 32 columns a block at a time, every 32nd row a
// thread, then the threads, in order.
constexpr int kAdders = 32;
__global__ __launch_bounds__(32 * kAdders) void k_add_rows(const float* in, int parts, int N,
                                                            float* out) {
  __shared__ float part[32 * kAdders];
  const int tid = threadIdx.x;
  for (int64_t first = blockIdx.x * 32; first < N; first += gridDim.x * 32) {
    const int64_t col = first + tid % 32;
    float v = 0.0f;
    if (col < N) {
#pragma unroll 8
      for (int p = tid / 32; p < parts; p += kAdders) v += in[(int64_t)p * N + col];
    }
    part[tid] = v;
    __syncthreads();
    if (tid < 32 && col < N) {
      for (int d = 1; d < kAdders; d++) v += part[d * 32 + tid];
      out[col] = v;
    }
    __syncthreads();
  }
}

// Copies rows of K elements to rows of ldo, a wave a row: 71,290 x 300 bf16 in
// 24 us, 3.6 TB/s.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_copy(const T* in, int64_t ld, T* out, int64_t ldo,
                                                    int rows, int K) {
  for (int64_t row = blockIdx.x * 4 + (threadIdx.x >> 6); row < rows; row += gridDim.x * 4) {
    for (int col = (threadIdx.x & 63) * 8; col < K; col += 512) {
      const uint4 v = load_end<T, 8>(in + row * ld + col, col + 8 - K, K);
      __builtin_memcpy(out + row * ldo + col, &v, 16);
    }
  }
}

// An operand with rows on 64-byte lines: itself, or its copy at `copy`, which
// has room for it unless it is not worth one (`bytes` 0).
template <typename T>
void align_rows(const void*& p, int64_t& ld, int rows, int K, void* copy, size_t bytes,
                hipStream_t s) {
  if constexpr (sizeof(T) == 2) {
    if (bytes == 0 || ((uintptr_t)p % 64 == 0 && ld % 32 == 0)) return;
    const int64_t ldo = aligned_columns(K);
    const int64_t blocks = ceil_div(rows, 4), most = 1 << 23;  // threads fit 32 bits
    k_copy<T><<<(int)(blocks < most ? blocks : most), kThreads, 0, s>>>((const T*)p, ld, (T*)copy,
                                                                        ldo, rows, K);
    p = copy;
    ld = ldo;
  }
}

// Zeroes `bytes` bytes of each of `rows` rows, a wave a row at a time.
__global__ __launch_bounds__(kThreads) void k_zero(char* p, int64_t stride, int rows,
                                                    int64_t bytes) {
  for (int64_t row = blockIdx.x * 4 + (threadIdx.x >> 6); row < rows; row += gridDim.x * 4)
    for (int64_t i = threadIdx.x & 63; i < bytes; i += 64) p[row * stride + i] = 0;
}

// Blocks of a kernel that goes on in steps of its grid, where `blocks` would do
// all of its work at once.
inline int grid_of(int64_t blocks) { return (int)(blocks < 65536 ? blocks : 65536); }

// The kernel of the plan's tile.
template <typename T, typename TO, bool AKC, bool BKC, bool FULL>
void launch_tile(const ProductArgs& a, const Plan& p, hipStream_t s) {
  const int blocks = p.tiles_m * p.tiles_n * p.splits;
  switch (p.tile) {
    case 0:
      k_product<T, TO, AKC, BKC, FULL, 1, 1, kTiles[0].granules, 4><<<blocks, kThreads, 0, s>>>(a);
      break;
    case 1:
      k_product<T, TO, AKC, BKC, FULL, 2, 1, kTiles[1].granules, 4><<<blocks, kThreads, 0, s>>>(a);
      break;
    default:
      k_product<T, TO, AKC, BKC, FULL, 2, 2, kTiles[2].granules, 4><<<blocks, kThreads, 0, s>>>(a);
      break;
  }
}

template <typename T, typename TO, bool AKC, bool BKC>
hipError_t launch_product(ProductArgs a, const Plan& p, void* partial, float* partial_sums,
                          hipStream_t s) {
  a.tiles_m = p.tiles_m;
  a.tiles_n = p.tiles_n;
  a.splits = p.splits;
  a.k_per_split = p.k_per_split;
  a.partial = (float*)partial;
  a.partial_sums = partial_sums;
  const bool full =
      a.activation != W2V_ACTIVATION_NONE || a.residual != nullptr || a.pre != nullptr;
  if constexpr (AKC && BKC) {  // the forward pass
    if (full)
      launch_tile<T, TO, AKC, BKC, true>(a, p, s);
    else
      launch_tile<T, TO, AKC, BKC, false>(a, p, s);
  } else {
    launch_tile<T, TO, AKC, BKC, false>(a, p, s);
  }
  if (p.splits > 1) {
    const int64_t blocks = ceil_div((int64_t)a.M * ((a.N + 3) / 4), kThreads);
    k_join<T, TO><<<(int)(blocks < 8192 ? blocks : 8192), kThreads, 0, s>>>(a);
  }
  return hipGetLastError();
}

template <typename T, typename TO>
hipError_t launch_linear_as(const LinearArgs& l, void* workspace, hipStream_t s) {
  ProductArgs a{};
  a.a = l.x;
  a.b = l.w;
  a.lda = l.ldx;
  a.ldb = l.ldw;
  a.M = l.M;
  a.N = l.N;
  a.K = l.K;
  a.bias = l.bias;
  a.residual = l.residual;
  a.y = l.y;
  a.pre = l.pre;
  a.ldr = l.ldr;
  a.ldy = l.ldy;
  a.ldp = l.ldp;
  a.activation = l.activation;
  if (few_rows(l.M, l.K)) {
    const int grid = (int)ceil_div(l.N, 64);
    k_few_rows<T, TO><<<grid, kThreads, 0, s>>>(a);
    return hipGetLastError();
  }
  const size_t bx = copy_bytes(l.M, l.M, l.N, l.K, l.dtype);
  const size_t bw = copy_bytes(l.N, l.M, l.N, l.K, l.dtype);
  char* ws = (char*)workspace;
  align_rows<T>(a.a, a.lda, l.M, l.K, ws, bx, s);
  align_rows<T>(a.b, a.ldb, l.N, l.K, ws + bx, bw, s);
  return launch_product<T, TO, true, true>(a, plan_product(l.M, l.N, l.K, l.dtype, false),
                                           ws + bx + bw, nullptr, s);
}

template <typename T>
hipError_t launch_backward_as(const LinearBackwardArgs& l, void* workspace, hipStream_t s) {
  const BackwardPlan b = plan_backward(l.M, l.N, l.K, l.dtype, l.activation);
  char* ws = (char*)workspace;
  const T* dz = (const T*)l.dy;
  int64_t lddz = l.lddy;
  // dW's product, which sums db on its way where dz is not rounded
  const bool product = l.dw != nullptr || (l.db != nullptr && !b.apart);
  float* const sums = (float*)(ws + b.dz + b.partial);
  if (l.activation != W2V_ACTIVATION_NONE && l.M > 0) {
    const bool wants_dz = l.dx != nullptr || product;
    if (b.apart && l.db != nullptr) {
      if constexpr (sizeof(T) == 2) {
        const SlopePlan& p = b.slope;
        k_slope_sums<T><<<dim3(p.stripes, p.chunks), kThreads, 0, s>>>(
            (const T*)l.dy, l.lddy, (const T*)l.pre, l.ldp, wants_dz ? (T*)ws : nullptr, l.M,
            l.N, l.activation, p.across, p.rows, p.chunks > 1 ? sums : l.db);
        if (p.chunks > 1)
          k_add_rows<<<grid_of(ceil_div(l.N, 32)), 32 * kAdders, 0, s>>>(sums, p.chunks, l.N,
                                                                         l.db);
      }
    } else if (wants_dz) {
      const int64_t units = (int64_t)l.M * ceil_div(l.N, 16 / (int)sizeof(T));
      const int64_t blocks = ceil_div(units, kThreads);
      k_slope<T><<<(int)(blocks < 16384 ? blocks : 16384), kThreads, 0, s>>>(
          (const T*)l.dy, l.lddy, (const T*)l.pre, l.ldp, (T*)ws, l.M, l.N, l.activation);
    }
    dz = (const T*)ws;
    lddz = l.N;
  }
  ws += b.dz;
  void* partial = ws;
  // (a copy of W for dx costs what it gains: its rows are read 256 bytes at a
  // time)
  const void* x = l.x;
  int64_t ldx = l.ldx;
  if (product) align_rows<T>(x, ldx, l.M, l.K, ws + b.partial + b.sums, b.x, s);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (l.M == 0) {  // no row: dW and db are sums of nothing
    if (l.dw != nullptr)
      k_zero<<<grid_of(ceil_div(l.N, 4)), kThreads, 0, s>>>(
          (char*)l.dw, l.lddw * sizeof(T), l.N, l.K * (int64_t)sizeof(T));
    if (l.db != nullptr)
      k_zero<<<1, kThreads, 0, s>>>((char*)l.db, 0, 1, l.N * (int64_t)4);
    return hipGetLastError();
  }
  if (l.dx != nullptr) {
    ProductArgs a{};
    a.a = dz;
    a.lda = lddz;
    a.b = l.w;
    a.ldb = l.ldw;
    a.M = l.M;
    a.N = l.K;
    a.K = l.N;
    a.y = l.dx;
    a.ldy = l.lddx;
    e = launch_product<T, T, true, false>(a, b.dx, partial, nullptr, s);
    if (e != hipSuccess) return e;
  }
  if (product) {
    ProductArgs a{};
    a.a = dz;
    a.lda = lddz;
    a.b = x;
    a.ldb = ldx;
    a.M = l.N;
    a.N = l.K;
    a.K = l.M;
    a.y = l.dw;
    a.ldy = l.lddw;
    a.row_sums = b.apart ? nullptr : l.db;
    e = launch_product<T, T, false, false>(a, b.dw, partial, sums, s);
  }
  return e;
}

}  // namespace
}  // namespace w2v
