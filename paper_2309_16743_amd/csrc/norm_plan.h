// Launch shapes and workspaces of group norm (norm.hip), free of HIP, so that they can be checked on the
// CPU.
#pragma once

#include <algorithm>
#include <cstdint>

#include "intmath.h"

namespace ot {

struct NormSizes {
  int64_t channels, positions;
  int32_t groups;
  int64_t per() const { return channels / groups; }     // channels of a group
};

// Over slabs (few positions): groups of a sample are kept in LDS as fp32, so that they are read once.  A slab holds
// kSlabAim values where it can, for several blocks on a CU (364 samples of 2408 channels in 56 groups, fp32 backward: 15
// us, 27 with one slab of 2408), and a group of up to kSlab.  From kSlabPositions positions on the
// split passes are faster (247 x 308 x 217 bf16, 31 groups, silu, backward: 84 us,
// 511 over slabs).
constexpr int64_t kSlab = 8192, kSlabAim = 2048;
constexpr int64_t kSlabPositions = 16;

// Groups of one block (0: the passes are split): whole vectors of 8 channels where that can be had.
inline int32_t slab_groups(const NormSizes& s) {
  const int64_t one = s.per() * s.positions;
  if (s.positions >= kSlabPositions || one > kSlab) return 0;
  const int64_t aim = std::max<int64_t>(1, kSlabAim / one), fit = kSlab / one;
  if (aim >= s.groups) return s.groups;
  for (int64_t g = aim; g >= 1; --g)
    if (g * s.per() % 8 == 0) return (int32_t)g;
  for (int64_t g = aim + 1; g <= fit && g < s.groups; ++g)
    if (g * s.per() % 8 == 0) return (int32_t)g;
  return (int32_t)(fit >= s.groups ? s.groups : aim);
}
// LDS of a block, in fp32 values.
inline int64_t slab_values(const NormSizes& s, bool back) {
  const int64_t gb = slab_groups(s), width = gb * s.per();
  return back ? 2 * width * s.positions + 2 * width + 2 * gb : width * s.positions + 2 * gb;
}

// Lanes that keep a sample's group in registers (0: it has no whole vectors of 8 channels, or more than 4
// of them a lane), and how many vectors each holds.
inline int32_t team_lanes(const NormSizes& s) {
  const int64_t vecs = s.per() / 8 * s.positions;
  if (s.per() % 8 != 0 || s.positions > 4 || vecs > 4 * 64) return 0;   // (a group's rows are short pieces)
  int32_t lanes = 1;
  while (lanes < 64 && lanes < vecs) lanes *= 2;
  return lanes;
}
inline int32_t team_vectors(const NormSizes& s) {
  const int64_t v = ceil_div(s.per() / 8 * s.positions, team_lanes(s));
  return v > 2 ? 4 : (int32_t)v;
}

// The backward over teams (one position): a block takes `groups` groups, tiles of them cover a sample, in
// `ranges` of the samples.
struct TeamPlan {
  int32_t lanes, groups;
  int64_t tiles, ranges;
};
constexpr int64_t kTeamBlocks = 256;
inline TeamPlan plan_team_back(const NormSizes& s, int64_t n) {
  TeamPlan t{team_lanes(s), 1, 0, 0};
  while (t.groups * 2 <= s.groups && t.groups * 2 * t.lanes <= 256) t.groups *= 2;
  t.tiles = ceil_div(s.groups, t.groups);
  t.ranges = std::max<int64_t>(1, std::min(ceil_div(n, 256 / t.lanes / t.groups), kTeamBlocks / t.tiles));
  return t;
}

// Split passes: a block holds col_threads x 8 channels (tiles of them cover the row) and a chunk of `rows`
// positions of one sample.
struct NormPlan {
  int32_t col_threads;
  int64_t tiles, chunks, rows;
};
constexpr int64_t kNormBlocks = 1024;
inline NormPlan plan_norm(const NormSizes& s, int64_t n) {
  NormPlan p{};
  const int64_t vecs = ceil_div(s.channels, 8);
  p.col_threads = 1;
  while (p.col_threads < 256 && p.col_threads < vecs) p.col_threads *= 2;
  p.tiles = ceil_div(vecs, p.col_threads);
  const int64_t lanes = 256 / p.col_threads;
  // 16 rows a thread, 64 a block at least; fewer while the card is not filled
  int64_t chunks = ceil_div(s.positions, std::max<int64_t>(16 * lanes, 64));
  if (n * p.tiles * chunks < kNormBlocks)
    chunks = std::max(chunks, std::min(ceil_div(kNormBlocks, n * p.tiles), ceil_div(s.positions, 2 * lanes)));
  p.rows = ceil_div(ceil_div(s.positions, chunks), lanes) * lanes;
  p.chunks = ceil_div(s.positions, p.rows);
  return p;
}

// Whether a block joins a group's partial sums, and not a wavefront (many small ones: 7657 groups of 14 values 12
// us by blocks, 5 by wavefronts).
inline bool long_join(const NormSizes& s, const NormPlan& p) { return p.chunks * s.per() > 512; }

// Sample ranges that the backward over slabs keeps sums of.
inline int64_t slab_ranges(const NormSizes& s, int64_t n) {
  const int64_t parts = ceil_div(s.groups, slab_groups(s));
  return std::max<int64_t>(1, std::min(n, kNormBlocks / parts));
}

// fp32 values that calls of up to n samples need: split passes keep two sums per channel and chunk, and
// two values per sample and group.  Over slabs the backward keeps two sums per range and channel.
inline int64_t norm_values(const NormSizes& s, int64_t n) {
  if (n < 1) return 0;
  if (slab_groups(s) > 0) return 2 * s.channels * std::min(n, kNormBlocks);
  const NormPlan most = plan_norm(s, n);
  const int64_t lanes = 256 / most.col_threads;
  const int64_t all = n * ceil_div(s.positions, std::max<int64_t>(16 * lanes, 64));
  const int64_t chunks = std::max(all, std::min(ceil_div(kNormBlocks, most.tiles) + n, n * ceil_div(s.positions, 2 * lanes)));
  return 2 * (chunks * s.channels + n * s.groups);
}

}  // namespace ot
