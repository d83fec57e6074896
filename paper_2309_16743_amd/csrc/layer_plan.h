// Tiles, splits and workspace of a dense layer's products (dense.hip) and of the column
// sums, free of HIP, so that the workspace bound and the choice of every kernel can be
// checked on the CPU.
#pragma once

#include <algorithm>
#include <cstdint>

#include "adapt_plan.h"
#include "intmath.h"

namespace ot {

// Block tiles (rows x columns): of gemm_bf16.h (k tiles of 32, 64 and eight wavefronts where said), then of
// gemm_f32x3.h.
enum DenseTile : int {
  kT64x64, kT64x128, kT128k32, kT128k64, kT128w8, kT256,
  kF64x64, kF64x128, kF32x256, kF64x256, kF128x64, kF128x128
};
constexpr int kDenseTileRows[] = {64, 64, 128, 128, 128, 256, 64, 64, 32, 64, 128, 128};
constexpr int kDenseTileCols[] = {64, 128, 128, 128, 128, 256, 64, 128, 256, 256, 64, 128};

inline int64_t dense_tiles(int tile, int64_t M, int64_t N) {
  return ceil_div(M, kDenseTileRows[tile]) * ceil_div(N, kDenseTileCols[tile]);
}

enum class Product : int { Forward, InputGrad, WeightGrad };

struct DensePlan {
  int tile;
  int64_t want;             // splits of K asked for
};

// Tile and splits of a product of M x N results over K with A as the sum of `planes` matrices, by the number of
// blocks that a tile gives (256 CUs; us of the product, with its join where it is split):
// bf16 layers (two or three blocks of 128 x 128 with k tile 32 share a CU, so that one's epilogue runs under
//   another's products; 256 x 256 holds a CU alone and wants a long k): 160000 x 256 x 256 on 64 x 128, 128 x 128,
//   256 x 256: 59, 47, 62; 512 x 200000 x 1024: 411, 336, 303; 20000 x 1024 x 512: 61, 53, 78.  Small ones:
//   1024 x 2048 x 2048 on 64 x 64, 128 x 128: 22, 40.  100000 x 64 x 64 on 64 x 64, 128 x 128: 21, 30.
//   Few rows of a long output (4 x 1000000 x 1024) on 64 x 64, 64 x 128, 128 x 128: 371, 357, 411.
// bf16 input gradients: 4096 x 2048 x 2048 on 64 x 128, 128 x 128 with k tiles 32, 64, 256 x 256: 57, 51, 43, 64;
//   160000 x 256 x 256 with k tiles 32, 64 (eight wavefronts): 47, 64.  1024 x 2048 x 2048 of one plane on 64 x 128
//   20, on 128 x 128 in 2 splits 24; of three planes 56, and 43 with eight wavefronts in 2 splits.
//   512 x 1024, k 1000000 on 256 x 256, 128 x 128 in 32 splits 1140, 1220; 64 x 1024, k 100000 on 64 x 128, 128 x
//   128 in 32: 40, 42.
// bf16 weight gradients: 1000000 x 1024 over 512 rows on 128 x 128, 256 x 256: 2030, 1860; 100000 x 1024 over 64
//   rows 79, 101; 2048 x 2048 over 1024 rows on 128 x 128 with k tiles 32, 64 (eight wavefronts): 24, 18;
//   512 x 512 over 4096 rows in 4, 8, 16 splits of the latter: 16.5, 16.0, 19.4.
// fp32 input gradients: 1024 x 2048 x 2048 on 128 x 128 in 1, 2, 4 splits, 64 x 64 in 2: 99, 61, 58, 71; 1024 x 256
//   x 256 on 64 x 64 in 1, 4 splits 11.3, 10.2, on 128 x 128 in 4 12.6.
// fp32 weight gradients: 6561 x 437 over 331 rows on 64 x 64, 128 x 128, 128 x 64 in 2: 38.6, 41.9, 35.5; 10000 x
//   256 over 1024 rows on 128 x 128 in 4, 128 x 64 in 1, 2, 4: 62, 98, 67, 59; 2048 x 2048 over 1024 on 128 x 128,
//   128 x 64: 56, 62; 256 x 256 over 1024 on 64 x 64, 128 x 64 in 4: 13.9, 17.8.
constexpr int64_t kLongRows = 768;
constexpr int64_t kMostTiles = (1LL << 24) - 1;           // a launch has fewer than 2^32 threads, 256 a block
inline DensePlan plan_dense(bool bf16, Product product, int64_t M, int64_t N, int64_t K, int planes) {
  constexpr int64_t kCUs = 256;
  auto tiles = [&](int t) { return dense_tiles(t, M, N); };
  auto splits = [](int64_t most, int64_t by_k) { return std::max<int64_t>(1, std::min(most, by_k)); };
  const int64_t k = K * planes;
  if (bf16) {
    switch (product) {
      case Product::Forward:
        if (N <= 64) return {kT64x64, 1};
        if (M <= 64 && tiles(kT64x128) >= kCUs - 16) return {kT64x128, 1};
        if (M > 128 && K >= 1024 && tiles(kT256) >= kCUs - 16) return {kT256, 1};
        if (tiles(kT128k32) >= 2 * kCUs - 32) return {kT128k32, 1};
        if (tiles(kT64x128) >= 2 * kCUs - 32) return {kT64x128, 1};
        return {kT64x64, 1};
      case Product::InputGrad:
        if (M > 64 && tiles(kT128k32) >= 2 * kCUs - 32) return {K < 512 ? kT128k32 : kT128k64, 1};
        // (where 256 x 256 would fill the card unsplit, the line above has taken all but up to 128 columns, which leave
        // half of it empty)
        if (M > 128 && k >= 65536 && tiles(kT256) < kCUs - 16) return {kT256, ceil_div(kCUs - 16, tiles(kT256))};
        if (M > 64 && k >= 4096) return {kT128w8, splits(ceil_div(kCUs - 16, tiles(kT128w8)), k / 1024)};
        return {kT64x128, splits(ceil_div(kCUs - 16, tiles(kT64x128)), k / 512)};
      default:
        if (tiles(kT256) >= kCUs - 16) return {k < 256 ? kT128k32 : kT256, 1};
        return {kT128w8, splits(kCUs / tiles(kT128w8), k / 512)};
    }
  }
  switch (product) {
    case Product::Forward:
      if (M <= 32 && tiles(kF32x256) >= kCUs) return {kF32x256, 1};
      if (M <= 64 && tiles(kF64x256) >= kCUs) return {kF64x256, 1};
      return {tiles(kF64x128) >= 2 * kCUs ? kF64x128 : kF64x64, 1};
    case Product::InputGrad:
      if (M <= 32 && N > 128) return {kF32x256, splits(2 * kCUs / tiles(kF32x256), K / 128)};
      if (M <= 64 && N > 128) return {kF64x256, splits(2 * kCUs / tiles(kF64x256), K / 128)};
      if (M > 64 && N > 64 && (K >= 1024 || tiles(kF64x64) > kMostTiles)) return {kF128x128, splits(2 * kCUs / tiles(kF128x128), K / 128)};
      return {kF64x64, splits(2 * kCUs / tiles(kF64x64), K / 64)};
    default:
      if (N > 64 && K >= kLongRows && tiles(kF128x128) >= 200) return {kF128x128, 1};
      if (tiles(kF64x64) > 256) return {kF128x64, splits(5 * kCUs / tiles(kF128x64), K / 160)};
      return {kF64x64, splits(2 * kCUs / tiles(kF64x64), K / 128)};
  }
}
// The splits that are not empty, in whole k tiles.
inline AdaptPlan split_dense(const DensePlan& d, int64_t K) { return split_plan(d.tile, K, d.want); }

// Whether the layer runs on dense_rows.h: few rows or few outputs, where the tiles are too few or walk k in too many
// steps one after the other, and so little in all that the loads of x and W, once per 32 rows and 16 outputs,
// do not count.  us there and tiled (rows, inputs, outputs):
// fp32 107, 516, 1512 9.3, 21.8; 1024, 256, 256 8.2, 14.6; 256, 2048, 2048 49, 70; 1024, 2048, 16 14, 59; but 512, 516,
//   1512 20.7, 22.7; 128, 64, 10000 10.1, 10.4; 256, 64, 10000 17.9, 12.9; 1024, 516, 1512 36, 30; and 8, 16 rows of
//   1024, 200000 175, 200 and 212, 204;
// bf16 32, 2048, 2048 9, 17; 64, 2048, 2048 9.8, 16.4; 128, 2048, 2048 14.9, 16.3; 1024, 2048, 16 9.6, 15.9; but 256, 2048,
//   2048 26, 16; 256, 256, 256 9.3, 9.1; 512, 516, 1512 11.8, 9.7; 32, 2048, 16384 24, 16.
inline bool direct_layer(bool bf16, int64_t M, int64_t N, int64_t K) {
  if (bf16) {
    if (M == 1 || (M <= 32 && M * N * K <= (1LL << 28))) return true;
    return K >= 512 && M * N <= (1LL << 18) && M * N * K <= (1LL << 29);
  }
  return M <= 8 || (M * N <= (1LL << 19) && M * N * K <= (1LL << 30));
}

// Sums over the rows of n x cols values: a thread holds 8 columns, a block of 256 threads
// col_threads x 8 columns and `rows` rows; `chunks` partial sums per column (1: the sum itself).
struct ColumnPlan {
  int32_t col_threads;
  int64_t blocks_x, chunks, rows;
};
constexpr int64_t kColumnBlocks = 1024;
inline ColumnPlan plan_columns(int64_t n, int64_t cols) {
  ColumnPlan p{};
  const int64_t groups = ceil_div(cols, 8);
  p.col_threads = 1;
  while (p.col_threads < 256 && p.col_threads < groups) p.col_threads *= 2;
  p.blocks_x = ceil_div(groups, p.col_threads);
  const int64_t lanes = 256 / p.col_threads;             // rows side by side
  const int64_t most = std::max<int64_t>(1, ceil_div(n, 4 * lanes));
  p.chunks = p.blocks_x >= 256 ? 1 : std::max<int64_t>(1, std::min(most, kColumnBlocks / p.blocks_x));
  p.rows = ceil_div(ceil_div(std::max<int64_t>(n, 1), p.chunks), lanes) * lanes;
  p.chunks = std::max<int64_t>(1, ceil_div(n, p.rows));
  return p;
}
inline int64_t column_values(int64_t n, int64_t cols) {
  const int64_t c = plan_columns(n, cols).chunks;
  return c > 1 ? c * round_up(cols, 4) : 0;
}

// Sizes of a dense layer and what its backward keeps.
struct DenseSizes {
  int64_t in, out;
  bool bf16;
  int32_t planes;           // bf16 terms of dz (0: dz is dy)
};
inline int64_t dz_ld(const DenseSizes& d) { return round_up(d.out, 8); }
inline int64_t dz_bytes(const DenseSizes& d, int64_t n) { return d.planes * n * dz_ld(d) * (d.bf16 ? 2 : 4); }

// Partial sums (fp32 values) of a product whose splits are `want`, at most.
inline int64_t product_values(bool bf16, Product p, int64_t M, int64_t N, int64_t K, int planes) {
  const DensePlan d = plan_dense(bf16, p, M, N, K, planes);
  return d.want > 1 ? d.want * M * ((N + 3) / 4 * 4) : 0;
}
// A backward's products, as dense_backward takes them: both every term of dz.
inline int dx_planes(const DenseSizes& d) { return std::max(1, d.planes); }
inline int64_t dx_values(const DenseSizes& d, int64_t n) {
  return product_values(d.bf16, Product::InputGrad, n, d.in, d.out, dx_planes(d));
}
inline int64_t dw_values(const DenseSizes& d, int64_t n) {
  return product_values(d.bf16, Product::WeightGrad, d.out, d.in, n, std::max(1, d.planes));
}
// Partial sums that calls of up to n rows need: of the weight gradient, of the input gradient and of the columns.
inline int64_t dense_values(const DenseSizes& d, int64_t n) {
  if (n < 1) return 0;
  // columns: chunks * blocks_x <= kColumnBlocks, and a chunk has at least 4 rows
  const int64_t db = std::min(kColumnBlocks * 256 * 8, ceil_div(n, 4) * round_up(d.out, 4));
  // the weight gradient: the tile changes at kLongRows only, and the splits asked for grow with the rows
  const int64_t dw = std::max(dw_values(d, n), dw_values(d, std::min(n, kLongRows - 1)));
  // the input gradient: a plan depends on the rows only through whole groups of 32, and past 65536 of them
  // there are so many tiles that nothing is split
  int64_t dx = 0;
  for (int64_t m = 32; m < std::min<int64_t>(n, 65536) + 32; m += 32) dx = std::max(dx, dx_values(d, m));
  return round_up(dw, 4) + round_up(dx, 4) + db;
}

}  // namespace ot
