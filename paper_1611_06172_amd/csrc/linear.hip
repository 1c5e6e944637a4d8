// Matrix products of the vocabulary head: y = act(x W^T + b) + r and its
// backward pass (dz = dy act'(z), dx = dz W, dW = dz^T x, db = column sums of
// dz), with fp32 accumulation and one rounding per output element.
#include "linear.h"

#include "head_types.h"

namespace w2v {
namespace {

constexpr int kThreads = 256;
constexpr int kRowBytes = 128;  // of k per tile row in LDS
constexpr int kGranules = 8;    // 16-byte granules of a tile row

// A block's share of C[m][n] = sum_k A(m, k) B(n, k). An operand whose k runs
// along memory (kc) holds element (r, k) at p[r ld + k], the other kind at
// p[k ld + r].
struct ProductArgs {
  const void* a;
  const void* b;
  int64_t lda, ldb;
  int32_t M, N, K;
  int32_t tiles_m, tiles_n, splits, tiles_per_split;
  // epilogue (splits == 1)
  const float* bias;
  const void* residual;
  void* y;
  void* pre;
  int64_t ldr, ldy, ldp;
  int32_t activation;
  // partial sums (splits > 1): float [splits][M][N]
  float* partial;
  // sums of A over k, or NULL: float [splits][M]
  float* row_sums;
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

// Where granule g of tile row r lies. Reads take one granule column over 32
// consecutive rows, the transposing writes one column over rows four apart:
// both fall on all 8 columns for any 8 neighbouring lanes.
__device__ __forceinline__ int granule_at(int r, int g) {
  return r * kGranules + (g ^ ((r ^ (r >> 3)) & 7));
}

// One operand's tile, ROWS rows by kRowBytes of k, on its way through
// registers into LDS. Elements past the operand's edge in k are 0; rows past
// it repeat the last row or are 0 (their products are not stored).
template <typename T, bool KC, int ROWS>
struct Stage {
  static constexpr int GE = Matrix<T>::kGranule;
  static constexpr int BK = GE * kGranules;
  // KC: 16-byte granules along k. Otherwise units of GE k-rows by 4
  // neighbouring elements, turned in registers.
  static constexpr int kUnits = KC ? ROWS * kGranules : ROWS / 4 * kGranules;
  static constexpr int kPer = (kUnits + kThreads - 1) / kThreads;
  static constexpr int kRegs = KC ? 1 : 4;
  uint4 r[kPer][kRegs];

  __device__ __forceinline__ void load(const T* p, int64_t ld, int row0, int rows, int k0,
                                       int K, int tid) {
#pragma unroll
    for (int i = 0; i < kPer; i++) {
      const int u = tid + i * kThreads;
      if (kUnits % kThreads != 0 && u >= kUnits) break;
      if constexpr (KC) {
        const int row = min(row0 + (u >> 3), rows - 1), k = k0 + (u & 7) * GE;
        const T* at = p + (int64_t)row * ld + k;
        const Pack<T, GE> v =
            k0 + BK <= K ? load_pack<T, GE>(at) : load_some<T, GE>(at, K - k);
        r[i][0] = __builtin_bit_cast(uint4, v);
      } else {
        const int m = row0 + (u % (ROWS / 4)) * 4, k = k0 + (u / (ROWS / 4)) * GE;
        Pack<T, 4> v[GE];
        const T* at = p + (int64_t)k * ld + m;
        if (k0 + BK <= K && row0 + ROWS <= rows) {
#pragma unroll
          for (int j = 0; j < GE; j++) v[j] = load_pack<T, 4>(at + (int64_t)j * ld);
        } else {
#pragma unroll
          for (int j = 0; j < GE; j++)
            v[j] = load_some<T, 4>(at + (int64_t)j * ld, k + j < K ? rows - m : 0);
        }
        __builtin_memcpy(&r[i][0], v, sizeof(v));
      }
    }
  }

  // Adds the tile's elements of each of the unit's 4 rows over k.
  __device__ __forceinline__ void add_rows(float (&sums)[kPer][4], int tid) const {
    if constexpr (!KC) {
#pragma unroll
      for (int i = 0; i < kPer; i++) {
        if (kUnits % kThreads != 0 && tid + i * kThreads >= kUnits) break;
        Pack<T, 4> v[GE];
        __builtin_memcpy(v, &r[i][0], sizeof(v));
#pragma unroll
        for (int j = 0; j < GE; j++)
#pragma unroll
          for (int c = 0; c < 4; c++) sums[i][c] += to_f32(v[j].v[c]);
      }
    }
  }

  __device__ __forceinline__ void store(uint4* lds, int tid) const {
#pragma unroll
    for (int i = 0; i < kPer; i++) {
      const int u = tid + i * kThreads;
      if (kUnits % kThreads != 0 && u >= kUnits) break;
      if constexpr (KC) {
        lds[granule_at(u >> 3, u & 7)] = r[i][0];
      } else {
        Pack<T, 4> v[GE];
        __builtin_memcpy(v, &r[i][0], sizeof(v));
#pragma unroll
        for (int c = 0; c < 4; c++) {
          Pack<T, GE> out;
#pragma unroll
          for (int j = 0; j < GE; j++) out.v[j] = v[j].v[c];
          lds[granule_at((u % (ROWS / 4)) * 4 + c, u / (ROWS / 4))] =
              __builtin_bit_cast(uint4, out);
        }
      }
    }
  }
};

// bias, activation, residual and the rounding of n (1..N) neighbouring
// elements of one row.
template <typename T, typename TO, int N>
__device__ __forceinline__ void finish(const ProductArgs& a, int64_t m, int col, int n,
                                       Pack<float, N> z) {
  if (a.y == nullptr) return;  // only the row sums are wanted
  if (a.bias != nullptr) {
    const Pack<float, N> b = load_some<float, N>(a.bias + col, n);
#pragma unroll
    for (int i = 0; i < N; i++) z.v[i] += b.v[i];
  }
  if (a.pre != nullptr) {
    Pack<T, N> out;
#pragma unroll
    for (int i = 0; i < N; i++) out.v[i] = from_f32<T>(z.v[i]);
    store_some<T, N>((T*)a.pre + m * a.ldp + col, n, out);
  }
  if (a.activation != W2V_ACTIVATION_NONE) {
#pragma unroll
    for (int i = 0; i < N; i++) z.v[i] = activate(z.v[i], a.activation);
  }
  if (a.residual != nullptr) {
    const Pack<TO, N> r = load_some<TO, N>((const TO*)a.residual + m * a.ldr + col, n);
#pragma unroll
    for (int i = 0; i < N; i++) z.v[i] += to_f32(r.v[i]);
  }
  Pack<TO, N> out;
#pragma unroll
  for (int i = 0; i < N; i++) out.v[i] = from_f32<TO>(z.v[i]);
  store_some<TO, N>((TO*)a.y + m * a.ldy + col, n, out);
}

// Tile of the block: XCD x of the 8 that blocks go round takes a contiguous
// range of the tiles, so that its L2 sees neighbours; within it panels of 16
// tiles in m are walked along n.
__device__ __forceinline__ void tile_of(const ProductArgs& a, int& tm, int& tn, int& split) {
  const int tiles = a.tiles_m * a.tiles_n;
  const int total = tiles * a.splits;
  const int per = total / 8, extra = total % 8;
  const int xcd = blockIdx.x % 8, at = blockIdx.x / 8;
  int t = xcd * per + min(xcd, extra) + at;
  split = t / tiles;
  t -= split * tiles;
  const int panel = 16 * a.tiles_n;
  const int first = t / panel * 16, height = min(16, a.tiles_m - first);
  const int in = t % panel;
  tm = first + in % height;
  tn = in / height;
}

// One block of 4 waves, 2 x 2, each (32 TM) x (32 TN) of a tile of (64 TM) x
// (64 TN), in 32 x 32 MFMA blocks. Operands come through registers into two
// LDS buffers of 128 bytes of k: the next tile's loads are in flight while
// this one is multiplied.
template <typename T, typename TO, bool AKC, bool BKC, int TM, int TN>
__global__ __launch_bounds__(kThreads) void k_product(ProductArgs a) {
  constexpr int BM = 64 * TM, BN = 64 * TN, BK = Matrix<T>::kGranule * kGranules;
  constexpr int kTile = (BM + BN) * kGranules;  // granules of one buffer
  constexpr int kOut = 32 * TN + 4;             // floats of a staged output row
  constexpr int kLds =
      2 * kTile * 16 > 4 * 32 * kOut * 4 ? 2 * kTile * 16 : 4 * 32 * kOut * 4;
  __shared__ __align__(16) unsigned char memory[kLds];
  uint4* lds = (uint4*)memory;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wm = wave >> 1, wn = wave & 1;
  int tm, tn, split;
  tile_of(a, tm, tn, split);
  const int m0 = tm * BM, n0 = tn * BN;
  const int k_tiles = (a.K + BK - 1) / BK;
  const int first = split * a.tiles_per_split;
  const int count = min(a.tiles_per_split, k_tiles - first);

  f32x16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; i++)
#pragma unroll
    for (int j = 0; j < TN; j++)
#pragma unroll
      for (int e = 0; e < 16; e++) acc[i][j][e] = 0.0f;

  Stage<T, AKC, BM> sa;
  Stage<T, BKC, BN> sb;
  float sums[Stage<T, AKC, BM>::kPer][4] = {};
  const bool want_sums = !AKC && a.row_sums != nullptr && tn == 0;
  if (count > 0) {
    sa.load((const T*)a.a, a.lda, m0, a.M, first * BK, a.K, tid);
    sb.load((const T*)a.b, a.ldb, n0, a.N, first * BK, a.K, tid);
    if (want_sums) sa.add_rows(sums, tid);
    sa.store(lds, tid);
    sb.store(lds + BM * kGranules, tid);
  }
  __syncthreads();
  for (int t = 0; t < count; t++) {
    const uint4* at = lds + (t & 1) * kTile;
    if (t + 1 < count) {
      sa.load((const T*)a.a, a.lda, m0, a.M, (first + t + 1) * BK, a.K, tid);
      sb.load((const T*)a.b, a.ldb, n0, a.N, (first + t + 1) * BK, a.K, tid);
    }
#pragma unroll
    for (int g = 0; g < kGranules; g += 2) {
      uint4 fa[TM], fb[TN];
#pragma unroll
      for (int i = 0; i < TM; i++)
        fa[i] = at[granule_at((wm * TM + i) * 32 + (lane & 31), g + (lane >> 5))];
#pragma unroll
      for (int j = 0; j < TN; j++)
        fb[j] = at[BM * kGranules +
                   granule_at((wn * TN + j) * 32 + (lane & 31), g + (lane >> 5))];
#pragma unroll
      for (int i = 0; i < TM; i++)
#pragma unroll
        for (int j = 0; j < TN; j++) acc[i][j] = Matrix<T>::mac32(fa[i], fb[j], acc[i][j]);
    }
    if (t + 1 < count) {
      uint4* to = lds + ((t + 1) & 1) * kTile;
      if (want_sums) sa.add_rows(sums, tid);
      sa.store(to, tid);
      sb.store(to + BM * kGranules, tid);
    }
    __syncthreads();
  }

  if (want_sums) {  // uniform over the block
    float* part = (float*)memory;  // [8 k-units][BM]
#pragma unroll
    for (int i = 0; i < Stage<T, AKC, BM>::kPer; i++) {
      const int u = tid + i * kThreads;
      if (u < Stage<T, AKC, BM>::kUnits) {
#pragma unroll
        for (int c = 0; c < 4; c++)
          part[u / (BM / 4) * BM + (u % (BM / 4)) * 4 + c] = sums[i][c];
      }
    }
    __syncthreads();
    for (int r = tid; r < BM; r += kThreads) {
      float v = 0.0f;
#pragma unroll
      for (int k = 0; k < kGranules; k++) v += part[k * BM + r];
      if (m0 + r < a.M) a.row_sums[(int64_t)split * a.M + m0 + r] = v;
    }
    __syncthreads();
  }

  // Output: each wave turns 32 rows at a time through its own part of LDS, so
  // that a lane holds neighbouring columns of a row (the MFMA block gives it
  // 16 rows of one column): wide stores, bias and residual loads.
  float* stage = (float*)memory + wave * 32 * kOut;
  constexpr int OV = 16 / (int)sizeof(TO);
  constexpr int kLanes = 32 * TN / OV;  // lanes of a row
#pragma unroll
  for (int i = 0; i < TM; i++) {
#pragma unroll
    for (int j = 0; j < TN; j++)
#pragma unroll
      for (int e = 0; e < 16; e++)
        stage[((e & 3) + 8 * (e >> 2) + 4 * (lane >> 5)) * kOut + j * 32 + (lane & 31)] =
            acc[i][j][e];
    __syncthreads();
    const int c = (lane % kLanes) * OV, col = n0 + wn * TN * 32 + c;
#pragma unroll 2
    for (int r = lane / kLanes; r < 32; r += 64 / kLanes) {
      const int m = m0 + (wm * TM + i) * 32 + r;
      if (m < a.M && col < a.N) {
        const Pack<float, OV> z = *(const Pack<float, OV>*)(stage + r * kOut + c);
        if (a.partial != nullptr)
          store_some<float, OV>(a.partial + ((int64_t)split * a.M + m) * a.N + col,
                                a.N - col, z);
        else
          finish<T, TO, OV>(a, m, col, a.N - col, z);
      }
    }
    __syncthreads();
  }
}

// Joins the partial sums of a product that was split along k, in order.
template <typename T, typename TO>
__global__ __launch_bounds__(kThreads) void k_join(ProductArgs a) {
  const int64_t per_row = (a.N + 3) / 4, units = per_row * a.M;
  for (int64_t u = (int64_t)blockIdx.x * kThreads + threadIdx.x; u < units;
       u += (int64_t)gridDim.x * kThreads) {
    const int64_t m = u / per_row;
    const int col = (int)(u % per_row) * 4, n = min(4, a.N - col);
    Pack<float, 4> z = load_some<float, 4>(a.partial + m * a.N + col, n);
    for (int s = 1; s < a.splits; s++) {
      const Pack<float, 4> p =
          load_some<float, 4>(a.partial + ((int64_t)s * a.M + m) * a.N + col, n);
#pragma unroll
      for (int i = 0; i < 4; i++) z.v[i] += p.v[i];
    }
    finish<T, TO, 4>(a, m, col, n, z);
  }
}

__global__ __launch_bounds__(kThreads) void k_join_sums(const float* part, float* out,
                                                         int splits, int n) {
  const int i = blockIdx.x * kThreads + threadIdx.x;
  if (i >= n) return;
  float v = 0.0f;
  for (int s = 0; s < splits; s++) v += part[(int64_t)s * n + i];
  out[i] = v;
}

// Few rows of x (M <= 16 MF): nothing of W is used twice, so W goes from
// memory straight into MFMA registers, 16 of its rows a wave, with x's rows as
// the other operand.
template <typename T, typename TO, int MF>
__global__ __launch_bounds__(kThreads) void k_few_rows(ProductArgs a) {
  constexpr int GE = Matrix<T>::kGranule, STEP = 4 * GE, U = 4;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int n0 = (blockIdx.x * 4 + wave) * 16;
  if (n0 >= a.N) return;
  const int g = lane >> 4, r = lane & 15;
  const T* w = (const T*)a.b + (int64_t)min(n0 + r, a.N - 1) * a.ldb + g * GE;
  const T* x[MF];
  f32x4 acc[MF];
#pragma unroll
  for (int f = 0; f < MF; f++) {
    x[f] = (const T*)a.a + (int64_t)min(f * 16 + r, a.M - 1) * a.lda + g * GE;
    acc[f] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  int k = 0;
  for (; k + U * STEP <= a.K; k += U * STEP) {
    uint4 fw[U], fx[U][MF];
#pragma unroll
    for (int u = 0; u < U; u++) {
      fw[u] = __builtin_bit_cast(uint4, load_pack<T, GE>(w + k + u * STEP));
#pragma unroll
      for (int f = 0; f < MF; f++)
        fx[u][f] = __builtin_bit_cast(uint4, load_pack<T, GE>(x[f] + k + u * STEP));
    }
#pragma unroll
    for (int u = 0; u < U; u++)
#pragma unroll
      for (int f = 0; f < MF; f++) acc[f] = Matrix<T>::mac16(fw[u], fx[u][f], acc[f]);
  }
  for (; k < a.K; k += STEP) {
    const int64_t n = a.K - k - g * GE;
    const uint4 fw = __builtin_bit_cast(uint4, load_some<T, GE>(w + k, n));
#pragma unroll
    for (int f = 0; f < MF; f++)
      acc[f] = Matrix<T>::mac16(
          fw, __builtin_bit_cast(uint4, load_some<T, GE>(x[f] + k, n)), acc[f]);
  }
  // lane: columns n0 + 4 g .. + 3 of row r (+ 16 f)
  const int col = n0 + 4 * g;
#pragma unroll
  for (int f = 0; f < MF; f++) {
    const int m = f * 16 + r;
    if (m < a.M && col < a.N) {
      Pack<float, 4> z;
#pragma unroll
      for (int i = 0; i < 4; i++) z.v[i] = acc[f][i];
      finish<T, TO, 4>(a, m, col, min(4, a.N - col), z);
    }
  }
}

// dz = dy act'(z), rounded once to the operands' type: the MFMA operands of
// both gradient products have it.
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
      out.v[i] =
          from_f32<T>(to_f32(g.v[i]) * activation_slope(to_f32(z.v[i]), activation));
    store_some<T, V>(dz + m * N + col, n, out);
  }
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
size_t aligned(size_t bytes) { return (bytes + 255) / 256 * 256; }
int element_size(int32_t dtype) { return dtype == W2V_DTYPE_F32 ? 4 : 2; }

// Tile and split of a product.
struct Plan {
  bool large;  // 128 x 128 tiles, else 64 x 64
  int32_t tiles_m, tiles_n, splits, tiles_per_split;
};

// 128 x 128 tiles reuse every loaded element twice as often as 64 x 64 ones,
// which are for products too small to give each of the 256 CUs a large tile.
// A product with a long k and few tiles is split along k until there are two
// blocks for each CU, with at least 8 tiles of k each.
Plan plan_product(int32_t M, int32_t N, int32_t K, int32_t dtype) {
  Plan p;
  p.large = ceil_div(M, 128) * ceil_div(N, 128) >= 256 || (M > 64 && N > 64 && K > 8192);
  const int tile = p.large ? 128 : 64;
  p.tiles_m = (int32_t)ceil_div(M, tile);
  p.tiles_n = (int32_t)ceil_div(N, tile);
  const int64_t k_tiles = ceil_div(K, kRowBytes / element_size(dtype));
  const int64_t tiles = (int64_t)p.tiles_m * p.tiles_n;
  int64_t splits = tiles == 0 ? 1 : ceil_div(512, tiles);
  if (splits > k_tiles / 8) splits = k_tiles / 8;
  if (splits > 64) splits = 64;
  if (splits < 1) splits = 1;
  p.tiles_per_split = (int32_t)ceil_div(k_tiles, splits);
  if (p.tiles_per_split < 1) p.tiles_per_split = 1;
  p.splits = (int32_t)ceil_div(k_tiles, p.tiles_per_split);
  if (p.splits < 1) p.splits = 1;
  return p;
}

size_t partial_bytes(const Plan& p, int32_t M, int32_t N) {
  return p.splits == 1 ? 0 : aligned((size_t)p.splits * M * N * 4);
}

template <typename T, typename TO, bool AKC, bool BKC>
hipError_t launch_product(ProductArgs a, const Plan& p, void* partial, hipStream_t s) {
  a.tiles_m = p.tiles_m;
  a.tiles_n = p.tiles_n;
  a.splits = p.splits;
  a.tiles_per_split = p.tiles_per_split;
  a.partial = p.splits > 1 ? (float*)partial : nullptr;
  const int grid = p.tiles_m * p.tiles_n * p.splits;
  if (p.large)
    k_product<T, TO, AKC, BKC, 2, 2><<<grid, kThreads, 0, s>>>(a);
  else
    k_product<T, TO, AKC, BKC, 1, 1><<<grid, kThreads, 0, s>>>(a);
  if (p.splits > 1) {
    const int64_t units = (int64_t)a.M * ((a.N + 3) / 4);
    const int64_t blocks = ceil_div(units, kThreads);
    k_join<T, TO><<<(int)(blocks < 8192 ? blocks : 8192), kThreads, 0, s>>>(a);
  }
  return hipGetLastError();
}

// Rows of x up to which W is streamed past them (k_few_rows).
constexpr int kFewRows = 32;

bool few_rows(int32_t M, int32_t K) { return M <= kFewRows && K <= 8192; }

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
    if (l.M <= 16)
      k_few_rows<T, TO, 1><<<grid, kThreads, 0, s>>>(a);
    else
      k_few_rows<T, TO, 2><<<grid, kThreads, 0, s>>>(a);
    return hipGetLastError();
  }
  return launch_product<T, TO, true, true>(a, plan_product(l.M, l.N, l.K, l.dtype), workspace,
                                           s);
}

// The backward pass's parts of its workspace.
struct BackwardPlan {
  Plan dx, dw;
  size_t dz, partial, sums;  // bytes
};

BackwardPlan plan_backward(int32_t M, int32_t N, int32_t K, int32_t dtype,
                           int32_t activation) {
  BackwardPlan b;
  b.dx = plan_product(M, K, N, dtype);
  b.dw = plan_product(N, K, M, dtype);
  b.dz = activation == W2V_ACTIVATION_NONE
             ? 0
             : aligned((size_t)M * N * element_size(dtype));
  const size_t px = partial_bytes(b.dx, M, K), pw = partial_bytes(b.dw, N, K);
  b.partial = px > pw ? px : pw;
  b.sums = b.dw.splits == 1 ? 0 : aligned((size_t)b.dw.splits * N * 4);
  return b;
}

template <typename T>
hipError_t launch_backward_as(const LinearBackwardArgs& l, void* workspace, hipStream_t s) {
  const BackwardPlan b = plan_backward(l.M, l.N, l.K, l.dtype, l.activation);
  char* ws = (char*)workspace;
  const T* dz = (const T*)l.dy;
  int64_t lddz = l.lddy;
  if (l.activation != W2V_ACTIVATION_NONE && l.M > 0) {
    const int64_t units = (int64_t)l.M * ceil_div(l.N, 16 / (int)sizeof(T));
    const int64_t blocks = ceil_div(units, kThreads);
    k_slope<T><<<(int)(blocks < 16384 ? blocks : 16384), kThreads, 0, s>>>(
        (const T*)l.dy, l.lddy, (const T*)l.pre, l.ldp, (T*)ws, l.M, l.N, l.activation);
    dz = (const T*)ws;
    lddz = l.N;
  }
  ws += b.dz;
  void* partial = ws;
  float* sums = (float*)(ws + b.partial);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (l.dx != nullptr && l.M > 0) {
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
    e = launch_product<T, T, true, false>(a, b.dx, partial, s);
    if (e != hipSuccess) return e;
  }
  if (l.dw != nullptr || l.db != nullptr) {
    ProductArgs a{};
    a.a = dz;
    a.lda = lddz;
    a.b = l.x;
    a.ldb = l.ldx;
    a.M = l.N;
    a.N = l.K;
    a.K = l.M;
    a.y = l.dw;
    a.ldy = l.lddw;
    a.row_sums = l.db == nullptr ? nullptr : b.dw.splits > 1 ? sums : l.db;
    e = launch_product<T, T, false, false>(a, b.dw, partial, s);
    if (e != hipSuccess) return e;
    if (l.db != nullptr && b.dw.splits > 1) {
      k_join_sums<<<(int)ceil_div(l.N, kThreads), kThreads, 0, s>>>(sums, l.db, b.dw.splits,
                                                                    l.N);
      e = hipGetLastError();
    }
  }
  return e;
}

}  // namespace

size_t linear_workspace_bytes(int32_t M, int32_t N, int32_t K, int32_t dtype) {
  if (few_rows(M, K)) return 0;
  return partial_bytes(plan_product(M, N, K, dtype), M, N);
}

size_t linear_backward_workspace_bytes(int32_t M, int32_t N, int32_t K, int32_t dtype,
                                       int32_t activation) {
  const BackwardPlan b = plan_backward(M, N, K, dtype, activation);
  return b.dz + b.partial + b.sums;
}

hipError_t launch_linear(const LinearArgs& a, void* workspace, hipStream_t s) {
  switch (a.dtype) {
    case W2V_DTYPE_F32:
      return launch_linear_as<float, float>(a, workspace, s);
    case W2V_DTYPE_BF16:
      return a.out_dtype == W2V_DTYPE_F32 ? launch_linear_as<bf16_t, float>(a, workspace, s)
                                          : launch_linear_as<bf16_t, bf16_t>(a, workspace, s);
    default:
      return a.out_dtype == W2V_DTYPE_F32 ? launch_linear_as<f16_t, float>(a, workspace, s)
                                          : launch_linear_as<f16_t, f16_t>(a, workspace, s);
  }
}

hipError_t launch_linear_backward(const LinearBackwardArgs& a, void* workspace,
                                  hipStream_t s) {
  switch (a.dtype) {
    case W2V_DTYPE_F32:
      return launch_backward_as<float>(a, workspace, s);
    case W2V_DTYPE_BF16:
      return launch_backward_as<bf16_t>(a, workspace, s);
    default:
      return launch_backward_as<f16_t>(a, workspace, s);
  }
}

}  // namespace w2v
