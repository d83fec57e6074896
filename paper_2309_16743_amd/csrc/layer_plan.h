// Tiles, splits and workspace of a dense layer's products (dense.hip) and of the column
// sums, free of HIP, so that the workspace bound and the choice of every kernel can be
// checked on the CPU.
#pragma once

#include <algorithm>
#include <cstdint>

#include "adapt_plan.h"
#include "intmath.h"

namespace ot {

// The layer y = x W^T (kmajor) and its input gradient dx = dz W take the tiles and splits of the
// adapters' products of the same layouts (plan_expand); the weight gradient dW = dz^T x, both operands
// MNMajor:
inline int wgrad_tile(bool bf16, int64_t M, int64_t N) {
  if (bf16) return adapt_tiles(kB256x256, M, N) >= 240 ? kB256x256 : kB128x128;
  return N <= 64 ? kX64x64 : kX128x128;
}
// Splits asked for: two blocks per CU, each with at least 512 (fp32: 128) rows.
inline int64_t wgrad_splits(bool bf16, int64_t M, int64_t N, int64_t K) {
  const int64_t tiles = adapt_tiles(wgrad_tile(bf16, M, N), M, N);
  return std::max<int64_t>(1, std::min(512 / tiles, K / (bf16 ? 512 : 128)));
}
inline AdaptPlan plan_wgrad(bool bf16, int64_t M, int64_t N, int64_t K) {
  return split_plan(wgrad_tile(bf16, M, N), K, wgrad_splits(bf16, M, N, K));
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
  p.chunks = std::max<int64_t>(1, std::min(most, kColumnBlocks / p.blocks_x));
  p.rows = ceil_div(ceil_div(std::max<int64_t>(n, 1), p.chunks), lanes) * lanes;
  p.chunks = std::max<int64_t>(1, ceil_div(n, p.rows));
  return p;
}
inline int64_t column_values(int64_t n, int64_t cols) {
  const int64_t c = plan_columns(n, cols).chunks;
  return c > 1 ? c * cols : 0;
}

// Sizes of a dense layer and what its backward keeps.
struct DenseSizes {
  int64_t in, out;
  bool bf16;
  int32_t planes;           // bf16 terms of dz (0: dz is dy)
};
inline int64_t dz_ld(const DenseSizes& d) { return round_up(d.out, 8); }
inline int64_t dz_bytes(const DenseSizes& d, int64_t n) { return d.planes * n * dz_ld(d) * (d.bf16 ? 2 : 4); }

inline int64_t dx_values(const DenseSizes& d, int64_t n) {
  return plan_values(plan_expand(d.bf16, false, n, d.in, d.out), n, d.in);
}
inline int64_t dw_values(const DenseSizes& d, int64_t n) {
  return plan_values(plan_wgrad(d.bf16, d.out, d.in, n), d.out, d.in);
}
// Partial sums that calls of up to n rows need (the products run one after the other and share them).
inline int64_t dense_values(const DenseSizes& d, int64_t n) {
  if (n < 1) return 0;
  // column sums: chunks * blocks_x <= kColumnBlocks
  int64_t most = std::min(kColumnBlocks * 256 * 8, ceil_div(n, 4) * d.out);
  // the weight gradient: the splits asked for grow with the rows
  const int64_t splits = wgrad_splits(d.bf16, d.out, d.in, n);
  if (splits > 1) most = std::max(most, splits * d.out * ((d.in + 3) / 4 * 4));
  // the input gradient: a plan depends on the rows only through whole groups of 32, and from 240 tiles
  // on nothing is split
  for (int64_t m = 32; m < std::min<int64_t>(n, 240 * 256) + 32; m += 32) most = std::max(most, dx_values(d, m));
  return most;
}

}  // namespace ot
