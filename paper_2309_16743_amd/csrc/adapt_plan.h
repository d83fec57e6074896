// Splits, tiles and workspace of the adapters' products (adapters.hip), free of HIP, so
// that the workspace bound and the choice of every kernel can be checked on the CPU.
#pragma once

#include <algorithm>
#include <cstdint>

#include "intmath.h"

namespace ot {

constexpr int kSlotRows = 32;       // sorted rows of one adapter that a shrink block takes together, at most
constexpr int kPassThreads = 512;   // of the one launch over a long dy

// What the plans of a bank depend on.
struct AdaptSizes {
  int64_t in, out;
  int32_t RP, G;                    // rank rounded up to 16, adapters
  bool bf16;
};

// Splits of the shrink's k range (length L) for n rows: enough blocks to fill the
// card, each with at least 512 values (331 rows of 6561: 8.5 us, 15.6 with 2048); one when the range is short,
// since the join costs a launch.  Blocks of unused slots (a large bank, few rows) are
// not multiplied without bound.
constexpr int64_t kShrinkBlocks = 1024;
inline int64_t shrink_splits(int64_t n, int64_t L, int32_t G) {
  if (L <= 4096) return 1;
  const int64_t slots = ceil_div(n, kSlotRows) + std::min<int64_t>(G, n) / 2;
  return std::max<int64_t>(1, std::min(std::min(ceil_div(kShrinkBlocks, slots), L / 512),
                                       32768 / (n / kSlotRows + G + 1)));
}

// Block tiles (rows x columns): of gemm_bf16.h, then of gemm_f32x3.h.
enum AdaptTileShape : int {
  kB64x64, kB64x128, kB128x128, kB256x256,
  kX128x128, kX64x64, kX64x128, kX32x256, kX64x256
};
constexpr int kAdaptTileRows[] = {64, 64, 128, 256, 128, 64, 64, 32, 64};
constexpr int kAdaptTileCols[] = {64, 128, 128, 256, 128, 64, 128, 256, 256};

struct AdaptPlan {
  int tile;
  int64_t splits, k_chunk;
};

inline int64_t adapt_tiles(int tile, int64_t M, int64_t N) {
  return ceil_div(M, kAdaptTileRows[tile]) * ceil_div(N, kAdaptTileCols[tile]);
}

// `want` splits of K, in k tiles of 64, as many as are not empty.
inline AdaptPlan split_plan(int tile, int64_t K, int64_t want) {
  AdaptPlan p{tile, 1, K};
  if (want > 1) {
    p.k_chunk = ceil_div(ceil_div(K, want), 64) * 64;
    p.splits = ceil_div(K, p.k_chunk);
    if (p.splits == 1) p.k_chunk = K;
  }
  return p;
}

// Tile and splits by the number of blocks that each choice gives (us of the whole call, as measured with each
// tile for all products of the kind):
// bf16 layers: 1024 x 1000000 x 2048 on 64 x 64, 64 x 128, 128 x 128, 256 x 256 tiles 8529, 7111, 6277, 4700: the
//   largest tile that still gives about a block per CU.  16 x 1000000 x 1024 on the same 678, 538, 638, 755: few
//   rows stream the weights and want the blocks' loads, not their products.  1024 x 2048 x 2048 37.5, 38.9,
//   51.9, 82.7: small tiles until every CU has blocks.
// bf16 input gradients: 512 x 1024, k 1000000 on 256 x 256 tiles in 16, 32, 64 splits 2207, 1677, 1708, on
//   128 x 128 2216, 2104, 2214: about a block per CU.  1024 x 2048, k 2048 on 64 x 128 tiles whole 51, in
//   2 splits 55 (the join is a launch).
// fp32 layers: 1024 x 10000 x 256 on 64 x 64, 64 x 128, 128 x 128 tiles 71, 66, 74.
// fp32 input gradients (the product alone): 331 x 437, k 6561 on 128 x 128 tiles in 12, 28, 42, 60 splits 64, 41,
//   35, 38; on 64 x 64 in 28, 60 41, 37.
// A plan depends on the rows only through whole groups of 32 (part_values).
inline AdaptPlan plan_expand(bool bf16, bool kmajor, int64_t M, int64_t N, int64_t K) {
  constexpr int64_t kCUs = 256;
  if (bf16) {
    if (kmajor) {
      if (M > 128 && adapt_tiles(kB256x256, M, N) >= kCUs - 16) return split_plan(kB256x256, K, 1);
      if (M <= 64 && adapt_tiles(kB64x128, M, N) >= kCUs - 16) return split_plan(kB64x128, K, 1);
      if (adapt_tiles(kB128x128, M, N) >= 2 * kCUs - 32) return split_plan(kB128x128, K, 1);
      if (adapt_tiles(kB64x128, M, N) >= 2 * kCUs - 32) return split_plan(kB64x128, K, 1);
      return split_plan(kB64x64, K, 1);
    }
    const int big = M > 128 ? kB256x256 : M > 64 ? kB128x128 : kB64x128;
    const int64_t t = adapt_tiles(big, M, N), sp = ceil_div(kCUs - 16, t);
    if (K / sp >= 2048) return split_plan(big, K, sp);
    const int64_t t2 = adapt_tiles(kB64x128, M, N);
    return split_plan(kB64x128, K, std::max<int64_t>(1, std::min(ceil_div(kCUs - 16, t2), K / 512)));
  }
  if (kmajor) {
    if (M <= 32 && adapt_tiles(kX32x256, M, N) >= kCUs) return split_plan(kX32x256, K, 1);
    if (M <= 64 && adapt_tiles(kX64x256, M, N) >= kCUs) return split_plan(kX64x256, K, 1);
    return split_plan(adapt_tiles(kX64x128, M, N) >= 2 * kCUs ? kX64x128 : kX64x64, K, 1);
  }
  const int tile = M <= 32 && N > 128 ? kX32x256 : M <= 64 && N > 128 ? kX64x256 : M <= 64 || N <= 64 ? kX64x64 : kX128x128;
  return split_plan(tile, K, std::max<int64_t>(1, std::min(2 * kCUs / adapt_tiles(tile, M, N), K / 128)));
}

// Partial sums of the plan (fp32 values; 0: not split).
inline int64_t plan_values(const AdaptPlan& p, int64_t M, int64_t N) { return p.splits > 1 ? p.splits * M * ((N + 3) / 4 * 4) : 0; }

// The one launch over a long dy keeps a partial of every row and column range: it takes
// batches of up to this many rows, and ranges so long that the partials stay within
// kPassBytes (at that many rows of rank 64 still 512 ranges of two blocks each and adapter).  One adapter, 1000000
// columns, no dx, with ranges for the number of blocks alone and so held: 4096 rows of rank 64 11.8 ms with 1.95 GB of
// partials, 8.4 with 0.51; 2048 rows 5.7 and 4.6; of rank 16, 4096 rows need 0.49 GB (3.2; held to 0.26 GB 3.7).
constexpr int64_t kPassMaxRows = 4096;
constexpr int64_t kPassBytes = 512 << 20;

// Pieces of 64 columns per wavefront in that launch (0: dy is short, or the rows too many, and
// the two products run apart).  512 rows, 8 adapters of rank 16, all launches but the input gradient, in it and
// apart: 8192 columns 27.2 and 26.4 us, 16384 31.0 and 32.7 (fp32 41.2 and 40.7), 65536 56 and 67
// (fp32 98 and 110; rank 64 147 and 322), 131072 88 and 123.
inline int pass_chunks(const AdaptSizes& a, int64_t n) {
  if (a.out < 16384 || n > kPassMaxRows) return 0;
  const int64_t few = std::max<int64_t>(1, std::min<int64_t>(4, a.out / 512 * a.G / 1024));
  const int64_t most = kPassBytes / (4 * std::max<int64_t>(n, 1) * a.RP);
  return (int)std::max(few, ceil_div(ceil_div(a.out, kPassThreads), most));
}
inline int64_t pass_ranges(const AdaptSizes& a, int64_t n) {
  return ceil_div(a.out, (int64_t)pass_chunks(a, n) * kPassThreads);
}

// Partial sums that a call of n rows asks for, product by product.
inline int64_t shrink_values(const AdaptSizes& a, int64_t n, int64_t L) {
  const int64_t splits = shrink_splits(n, L, a.G);
  return splits > 1 ? splits * n * a.RP : 0;
}
inline int64_t pass_values(const AdaptSizes& a, int64_t n) {
  return pass_chunks(a, n) ? pass_ranges(a, n) * n * a.RP : 0;
}
inline int64_t gradient_values(const AdaptSizes& a, int64_t n) {
  return plan_values(plan_expand(a.bf16, false, n, a.in, a.out), n, a.in);
}

// Partial sums that calls of up to n rows need.
inline int64_t part_values(const AdaptSizes& a, int64_t n) {
  // shrinks: splits * rows, with splits <= kShrinkBlocks / (rows / 32) + 1
  int64_t most = std::max(a.in, a.out) > 4096 ? (kShrinkBlocks * kSlotRows + n) * a.RP : 0;
  // the pass: the fewest pieces give the most ranges, up to the byte bound
  if (pass_chunks(a, 1))
    most = std::max(most, std::min(kPassBytes / 4, pass_ranges(a, 1) * std::min(n, kPassMaxRows) * a.RP));
  // the input gradient: a plan depends on the rows only through whole groups of 32
  for (int64_t m = 32; m < n + 32; m += 32) most = std::max(most, gradient_values(a, m));
  return most;
}

}  // namespace ot
