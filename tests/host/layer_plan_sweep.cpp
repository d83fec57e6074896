// A seeded sweep of the layers' plans (csrc/layer_plan.h, norm_plan.h) over sizes spread over their whole range and
// close to multiples of the tiles:
//   kernels COUNT SEED      every kernel that a dense layer takes, one a line, each with a size that takes it
//   bound COUNT SEED        workspaces sized for n rows hold what calls of n and fewer rows need; dz and the partial
//                           sums keep to what include/layers.h says
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <random>
#include <string>

#include "layer_plan.h"
#include "norm_plan.h"

using namespace ot;

static std::mt19937_64 rng;

static int64_t below(int64_t n) { return (int64_t)(rng() % (uint64_t)n); }

// From 1 to `most`, uniform over the logarithm; half of them moved next to a multiple of a tile's edge.
static int64_t size(int64_t most) {
  const double f = (double)(rng() >> 11) * 0x1p-53;
  int64_t v = (int64_t)std::exp(f * std::log((double)most));
  if (below(2)) {
    const int64_t edge = 32LL << below(4);
    v = (v + edge / 2) / edge * edge + below(5) - 2;
  }
  return std::max<int64_t>(1, std::min(v, most));
}

// A row count whose tiles of `rows` rows, `cols` of them side by side, come close to `want`.
static int64_t near(int64_t rows, int64_t cols, int64_t want) {
  return std::max<int64_t>(1, rows * std::max<int64_t>(1, want / std::max<int64_t>(1, cols) + below(5) - 2) + below(5) - 2);
}

struct Size {
  int64_t n, in, out;
};

static Size draw() {
  for (;;) {
    Size s{size(1 << 26), size(1 << 26), size(1 << 26)};
    if (below(2)) {                      // around a number of blocks where a plan changes
      const int64_t tile[] = {32, 64, 128, 256}, count[] = {200, 240, 256, 480, 512};
      const int64_t t = tile[below(4)], u = tile[below(4)], c = count[below(5)];
      switch (below(3)) {
        case 0: s.n = near(t, ceil_div(s.out, u), c); break;
        case 1: s.n = near(t, ceil_div(s.in, u), c); break;
        default: s.out = near(t, ceil_div(s.in, u), c); break;
      }
    }
    const int64_t most = 1LL << 36, side = 1LL << 26;
    if (s.n <= side && s.in <= side && s.out <= side && s.n * std::max(s.in, s.out) <= most && s.in * s.out <= most) return s;
  }
}

static std::map<std::string, Size> found;

static void kernels(const Size& z) {
  char b[128];
  for (int bf = 0; bf < 2; ++bf)
    for (int planes : {0, 1, 3}) {
      if (planes == 3 && !bf) continue;
      const DenseSizes d{z.in, z.out, bf != 0, planes};
      auto add = [&](const char* what, Product p, int64_t M, int64_t N, int64_t K, int pl) {
        const AdaptPlan a = split_dense(plan_dense(bf, p, M, N, K, pl), K);
        snprintf(b, sizeof b, "%s bf16=%d tile=%d split=%d", what, bf, a.tile, a.splits > 1);
        found.emplace(b, z);
      };
      if (direct_layer(bf, z.n, z.out, z.in)) {
        snprintf(b, sizeof b, "forward bf16=%d direct=%d", bf, z.n > 32 ? 3 : z.n > 16 ? 2 : 1);
        found.emplace(b, z);
      } else {
        add("forward", Product::Forward, z.n, z.out, z.in, 1);
      }
      add("dx", Product::InputGrad, z.n, z.in, z.out, dx_planes(d));
      add("dw", Product::WeightGrad, z.out, z.in, z.n, std::max(1, planes));
      snprintf(b, sizeof b, "columns chunks=%d", plan_columns(z.n, z.out).chunks > 1);
      found.emplace(b, z);
    }
}

static int64_t used(const DenseSizes& d, int64_t n) {
  auto values = [&](Product p, int64_t M, int64_t N, int64_t K, int pl) {
    return plan_values(split_dense(plan_dense(d.bf16, p, M, N, K, pl), K), M, N);
  };
  const int64_t dw = dw_values(d, n), dx = dx_values(d, n);
  if (values(Product::InputGrad, n, d.in, d.out, dx_planes(d)) > dx ||
      values(Product::WeightGrad, d.out, d.in, n, std::max(1, d.planes)) > dw)
    return 1LL << 60;
  return round_up(dw, 4) + round_up(dx, 4) + column_values(n, d.out);
}

static bool bounds(const Size& z) {
  bool ok = true;
  for (int bf = 0; bf < 2; ++bf)
    for (int planes : {0, 1, 3}) {
      if (planes == 3 && !bf) continue;
      const DenseSizes d{z.in, z.out, bf != 0, planes};
      const int64_t have = dense_values(d, z.n), fewer = 1 + below(z.n);
      const char* bad = nullptr;
      if (used(d, z.n) > have || used(d, fewer) > have) bad = "partial sums past their place";
      // include/layers.h: dz takes its terms of dy's size, rows padded to 8 values; partial sums 0.3 GB
      const int64_t row = ceil_div(z.out, 8) * 8 * (bf ? 2 : 4);
      if (dz_bytes(d, z.n) != planes * z.n * row || dz_bytes(d, fewer) > dz_bytes(d, z.n)) bad = "dz";
      if (4 * have > 300000000) bad = "partial sums past 0.3 GB";
      if (bad) {
        printf("%s: rows %lld (%lld) in %lld out %lld bf16 %d terms %d: %lld values\n", bad, (long long)z.n,
               (long long)fewer, (long long)z.in, (long long)z.out, bf, planes, (long long)have);
        ok = false;
      }
    }
  return ok;
}

int main(int argc, char** argv) {
  if (argc != 4) return 2;
  rng.seed((uint64_t)atoll(argv[3]));
  const int64_t count = atoll(argv[2]);
  if (!strcmp(argv[1], "kernels")) {
    for (int64_t i = 0; i < count; ++i) kernels(draw());
    for (const auto& k : found)
      printf("%s\t%lld %lld %lld\n", k.first.c_str(), (long long)k.second.n, (long long)k.second.in, (long long)k.second.out);
    return 0;
  }
  if (!strcmp(argv[1], "bound")) {
    bool ok = true;
    for (int64_t i = 0; i < count; ++i) ok = bounds(draw()) && ok;
    if (ok) puts("ok");
    return ok ? 0 : 1;
  }
  return 2;
}
