// How the vocabulary head's matrix products are cut into tiles, splits and
// workspace (host only).
#pragma once

#include <cmath>

#include "linear.h"
#include "w2v.h"

namespace w2v {

// Output tiles, and 16-byte granules of k per tile row in LDS.
struct Tile {
  int rows, cols, granules;
};
constexpr Tile kTiles[3] = {{64, 64, 8}, {128, 64, 4}, {128, 128, 4}};

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline size_t aligned(size_t bytes) { return (bytes + 255) / 256 * 256; }
inline int element_size(int32_t dtype) { return dtype == W2V_DTYPE_F32 ? 4 : 2; }

// Tile and split of a product.
struct Plan {
  int32_t tile;  // of kTiles
  int32_t tiles_m, tiles_n, splits, k_per_split;
};

// Blocks that the GPU holds at once, 4 on each of 256 CUs.
constexpr int kSlots = 1024;

// Share of the GPU's rate that so many blocks reach: one block a CU is half of
// it, four are all. (fp32 4,096 x 600 x 600 with 160, 320 and 640 blocks took
// 65, 54 and 43 us.)
inline double filled(double blocks) {
  if (blocks >= kSlots) return 1.0;
  const double cus = kSlots / 4.0;
  return blocks >= cus ? std::sqrt(blocks / kSlots) : 0.5 * blocks / cus;
}

// The tile and the split of k with the least time. What a tile's element costs
// beside one of a 128 x 128 tile, by products that fill the GPU (8192 x 8192
// outputs, k 2048): fp32, bound by MFMA, 1.10 for 64 x 64 and 1.07 for 128 x 64;
// 16 bits, bound by LDS reads, 1.8 and 1.45, but 1.35 and 1.15 where both
// operands are turned (dW). bf16 65,536 x 300 x 300 takes 42 us with 128 x 128
// tiles and 51 with 64 x 64 ones.
// A k may be split into as many parts as the GPU has room for, of at least 8
// tiles of k each. Partial sums are written and read at 4 TB/s, and one more
// launch takes 3 us: bf16 4,096 x 600 x 600 takes 26 us in two parts, 14.5 in
// one, fp32 4,096 x 300 x 300 23 and 18; but dW of 4,096 x 600 x 600 fp32 (600 x
// 600 outputs) takes 116 in one, 46 in ten.
inline Plan plan_product(int32_t M, int32_t N, int32_t K, int32_t dtype, bool both_turned) {
  static const double kCost[3][3] = {{1.10, 1.07, 1.0}, {1.8, 1.45, 1.0}, {1.35, 1.15, 1.0}};
  const double* cost = kCost[dtype == W2V_DTYPE_F32 ? 0 : both_turned ? 2 : 1];
  const double rate = dtype == W2V_DTYPE_F32 ? 115e6 : 420e6;  // operations a us
  Plan best{};
  double least = 0.0;
  for (int i = 2; i >= 0; i--) {
    const Tile& t = kTiles[i];
    Plan p;
    p.tile = i;
    p.tiles_m = (int32_t)ceil_div(M, t.rows);
    p.tiles_n = (int32_t)ceil_div(N, t.cols);
    const int64_t k_tiles = ceil_div(K, t.granules * 16 / element_size(dtype));
    const int64_t tiles = (int64_t)p.tiles_m * p.tiles_n;
    int64_t most = kSlots / tiles;
    if (most > k_tiles / 8) most = k_tiles / 8;
    if (most > 64) most = 64;
    if (most < 1) most = 1;
    const double work = cost[i] * (double)tiles * t.rows * t.cols * 2.0 * K / rate;
    for (int64_t splits = 1; splits <= most; splits++) {
      p.k_per_split = (int32_t)ceil_div(k_tiles, splits);
      p.splits = (int32_t)ceil_div(k_tiles, p.k_per_split);
      double us = work / filled((double)tiles * p.splits);
      if (p.splits > 1) us += 3.0 + 2.0 * p.splits * (double)M * N * 4.0 / 4e6;
      if ((i == 2 && splits == 1) || us < least) {
        best = p;
        least = us;
      }
    }
  }
  return best;
}

inline size_t partial_bytes(const Plan& p, int32_t M, int32_t N) {
  return p.splits == 1 ? 0 : aligned((size_t)p.splits * M * N * 4);
}

// Whether x and W are worth a copy with rows on 64-byte lines where theirs are
// not. Tiles read 64 bytes of k of each row, so every read of a 600-byte row
// meets one line too many: bf16 4,096 x 71,290 x 300 takes 550 us as it is, 450
// with aligned rows. The copies are (M + N) K elements against a product that
// reads x N / 128 times and W M / 128 times: they cost a tenth of it where
// M N / (M + N) is 1600.
inline bool worth_aligning(int32_t M, int32_t N, int32_t dtype) {
  return dtype != W2V_DTYPE_F32 && (double)M * N > 1600.0 * ((double)M + N);
}
inline int64_t aligned_columns(int32_t K) { return ceil_div(K, 32) * 32; }
// Bytes of such a copy of `rows` rows, where it may be made.
inline size_t copy_bytes(int32_t rows, int32_t M, int32_t N, int32_t K, int32_t dtype) {
  return worth_aligning(M, N, dtype) ? aligned((size_t)rows * aligned_columns(K) * 2) : 0;
}

// Whether W is streamed past x (k_few_rows): at most 16 rows, one MFMA operand,
// and a k that one wave goes through before tiles split along k would end.
// Streamed and by tiles (us, in a graph): 1 x 71,290 x 300 fp32 17.5 and 38.5,
// 16 rows 20.6 and 39.8; 1 x 10^6 x 300 bf16 122 and 152, 16 rows 187 and 172
// (the one of these where streaming loses);
// 1 x 4,096 x 2,000 fp32 28 and 33, bf16 9.7 and 11.5; 1 x 4,096 x 4,000 fp32
// 55 and 34; 32 x 71,290 x 300 bf16 with two operands 17.9 and 14.9.
inline bool few_rows(int32_t M, int32_t K) { return M <= 16 && K <= 2048; }

// Blocks of k_slope_sums: stripes of up to 32 packs of 16 bytes, as even as they
// come, by chunks of rows, about 2048 blocks in all and at most 1024 chunks, whose
// sums are added up afterwards.
struct SlopePlan {
  int32_t stripes, chunks, across, rows;
};

inline SlopePlan plan_slope(int32_t M, int32_t N, int32_t dtype) {
  SlopePlan p;
  const int64_t packs = ceil_div(N, 16 / element_size(dtype));
  p.stripes = (int32_t)ceil_div(packs, 32);
  p.across = (int32_t)ceil_div(packs, p.stripes);
  const int64_t down = 256 / p.across;  // rows that a block has at once
  int64_t chunks = ceil_div(2048, p.stripes);
  if (chunks > 1024) chunks = 1024;
  p.rows = (int32_t)(ceil_div(ceil_div(M, chunks), down) * down);
  p.chunks = (int32_t)ceil_div(M, p.rows);
  return p;
}

// The backward pass's parts of its workspace.
struct BackwardPlan {
  Plan dx, dw;
  bool apart;  // db is summed beside dz; otherwise within dW's product
  SlopePlan slope;  // where it is
  size_t dz, partial, sums, x;  // bytes
};

inline BackwardPlan plan_backward(int32_t M, int32_t N, int32_t K, int32_t dtype,
                                  int32_t activation) {
  BackwardPlan b{};
  if (M == 0) return b;
  b.dx = plan_product(M, K, N, dtype, false);
  b.dw = plan_product(N, K, M, dtype, true);
  b.dz = activation == W2V_ACTIVATION_NONE
             ? 0
             : aligned((size_t)M * N * element_size(dtype));
  b.apart = b.dz != 0 && dtype != W2V_DTYPE_F32;  // dz is rounded to 16 bits
  if (b.apart) b.slope = plan_slope(M, N, dtype);
  const size_t px = partial_bytes(b.dx, M, K), pw = partial_bytes(b.dw, N, K);
  b.partial = px > pw ? px : pw;
  const int32_t parts = b.apart ? b.slope.chunks : b.dw.splits;
  b.sums = parts == 1 ? 0 : aligned((size_t)parts * N * 4);
  b.x = copy_bytes(M, M, N, K, dtype);
  return b;
}

// One element type's launches (linear_<type>.hip).
hipError_t launch_linear_f32(const LinearArgs& l, void* workspace, hipStream_t s);
hipError_t launch_linear_bf16(const LinearArgs& l, void* workspace, hipStream_t s);
hipError_t launch_linear_f16(const LinearArgs& l, void* workspace, hipStream_t s);
hipError_t launch_backward_f32(const LinearBackwardArgs& l, void* workspace, hipStream_t s);
hipError_t launch_backward_bf16(const LinearBackwardArgs& l, void* workspace, hipStream_t s);
hipError_t launch_backward_f16(const LinearBackwardArgs& l, void* workspace, hipStream_t s);

}  // namespace w2v
