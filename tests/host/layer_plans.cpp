// Checks of the layers' plans (csrc/layer_plan.h, norm_plan.h) on the host.
//   bound            workspaces sized for n rows (samples) hold what every call of fewer needs
//   dense            every kernel that some call takes, one a line
//   dense-of R I O   those of the calls of a tested size (both precisions, activations with 0, 1 and 3 terms)
//   launches         no launch of the largest calls has 2^32 threads
//   norm, norm-of N P C G   the same for group norm
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <set>
#include <string>

#include "layer_plan.h"
#include "norm_plan.h"

using namespace ot;

static void dense_kernels(int64_t n, int64_t in, int64_t out, std::set<std::string>& s) {
  char b[128];
  for (int bf = 0; bf < 2; ++bf)
    for (int planes : {0, 1, 3}) {
      if (planes == 3 && !bf) continue;
      const DenseSizes d{in, out, bf != 0, planes};
      auto add = [&](const char* what, Product p, int64_t M, int64_t N, int64_t K, int pl) {
        const AdaptPlan a = split_dense(plan_dense(bf, p, M, N, K, pl), K);
        snprintf(b, sizeof b, "%s bf16=%d tile=%d split=%d", what, bf, a.tile, a.splits > 1);
        s.insert(b);
      };
      if (direct_layer(bf, n, out, in)) {
        snprintf(b, sizeof b, "forward bf16=%d direct=%d", bf, n > 32 ? 3 : n > 16 ? 2 : 1);
        s.insert(b);
      } else {
        add("forward", Product::Forward, n, out, in, 1);
      }
      add("dx", Product::InputGrad, n, in, out, dx_planes(d));
      add("dw", Product::WeightGrad, out, in, n, std::max(1, planes));
      snprintf(b, sizeof b, "columns chunks=%d", plan_columns(n, out).chunks > 1);
      s.insert(b);
    }
}

static void norm_kernels(int64_t n, int64_t p, int64_t c, int32_t g, std::set<std::string>& s) {
  const NormSizes z{c, p, g};
  char b[128];
  const int lanes = team_lanes(z);
  if (lanes) {
    snprintf(b, sizeof b, "forward team vectors=%d", team_vectors(z));
    s.insert(b);
  } else if (slab_groups(z)) {
    snprintf(b, sizeof b, "forward slab whole=%d", slab_groups(z) == g);
    s.insert(b);
  } else {
    snprintf(b, sizeof b, "forward split long=%d", long_join(z, plan_norm(z, n)));
    s.insert(b);
  }
  if (lanes && p == 1) {
    snprintf(b, sizeof b, "backward team vectors=%d rows=%d", team_vectors(z), 256 / lanes / plan_team_back(z, n).groups > 1);
    s.insert(b);
  } else if (slab_groups(z)) {
    snprintf(b, sizeof b, "backward slab whole=%d", slab_groups(z) == g);
    s.insert(b);
  } else {
    snprintf(b, sizeof b, "backward split long=%d", long_join(z, plan_norm(z, n)));
    s.insert(b);
  }
}

static bool fail(const char* what, int64_t a, int64_t b, int64_t c, int64_t d) {
  printf("%s: %lld %lld %lld %lld\n", what, (long long)a, (long long)b, (long long)c, (long long)d);
  return false;
}

// How far a dense_backward of n rows reaches into its partial sums; 0 if one of them is larger than its place.
static int64_t dense_used(const DenseSizes& d, int64_t n) {
  auto used = [&](Product p, int64_t M, int64_t N, int64_t K, int pl) {
    const AdaptPlan a = split_dense(plan_dense(d.bf16, p, M, N, K, pl), K);
    return plan_values(a, M, N);
  };
  const int64_t dw = dw_values(d, n), dx = dx_values(d, n);
  if (used(Product::InputGrad, n, d.in, d.out, dx_planes(d)) > dx ||
      used(Product::WeightGrad, d.out, d.in, n, std::max(1, d.planes)) > dw)
    return 1LL << 60;
  return round_up(dw, 4) + round_up(dx, 4) + column_values(n, d.out);
}

static int64_t norm_used(const NormSizes& s, int64_t n) {
  if (slab_groups(s) > 0) {
    int64_t r = 2 * slab_ranges(s, n) * s.channels;
    if (team_lanes(s) && s.positions == 1) r = std::max(r, 2 * plan_team_back(s, n).ranges * s.channels);
    return r;
  }
  const NormPlan p = plan_norm(s, n);
  return 2 * n * s.groups + 2 * n * p.chunks * s.channels;
}

static bool bounds() {
  bool ok = true;
  const int64_t wide[] = {1, 3, 6, 31, 64, 65, 128, 200, 437, 1024, 2048, 5000, 10000, 65537, 1000000, 1 << 26};
  for (int64_t in : wide)
    for (int64_t out : wide) {
      if (in * out > (1LL << 36)) continue;
      for (int bf = 0; bf < 2; ++bf)
        for (int planes : {0, 1, 3}) {
          if (planes == 3 && !bf) continue;
          const DenseSizes d{in, out, bf != 0, planes};
          for (int64_t most : {1LL, 20LL, 100LL, 1000LL, 4096LL, 70000LL}) {
            const int64_t have = dense_values(d, most);
            if (have * 4 > 300LL << 20) ok = fail("dense partial sums", in, out, most, have);
            for (int64_t n = 1; n <= most; n += 1 + n / 37)
              if (dense_used(d, n) > have) ok = fail("dense", in, out, n, most);
            if (dense_used(d, most) > have) ok = fail("dense", in, out, most, most);
          }
        }
    }
  for (int64_t c : {1, 2, 8, 30, 64, 435, 2048, 5000, 65536})
    for (int64_t p : {1, 2, 9, 15, 16, 100, 1000, 10000, 1000000})
      for (int32_t g : {1, 2, 3, 5, 8, 64, 435, 2048, 65536}) {
        if (g > c || c % g) continue;
        const NormSizes s{c, p, g};
        for (int64_t most : {1LL, 7LL, 64LL, 3000LL}) {
          const int64_t have = norm_values(s, most);
          for (int64_t n = 1; n <= most; n += 1 + n / 23)
            if (norm_used(s, n) > have) ok = fail("norm", c, p, g, n);
          if (norm_used(s, most) > have) ok = fail("norm", c, p, g, most);
          if (slab_groups(s) > 0 && 4 * std::max(slab_values(s, false), slab_values(s, true)) > 159 * 1024)
            ok = fail("norm slab", c, p, g, slab_values(s, true));
          const NormPlan q = plan_norm(s, most);
          if (q.chunks * q.rows < p || (q.chunks - 1) * q.rows >= p || q.tiles * q.col_threads * 8 < c)
            ok = fail("norm plan", c, p, g, most);
        }
      }
  return ok;
}

static bool launches() {
  bool ok = true;
  const int64_t most = 1LL << 36, row[] = {1, 8, 9, 31, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 513, 1000, 1023,
                                           1024, 1025, 1029, 2047, 2049, 65535, 65537, 1 << 20, 1 << 26};
  for (int64_t N : row)
    for (int64_t K : {1, 40, 300, 767, 1023, 1024, 5000, 100000}) {
      const int64_t M = std::min<int64_t>(1LL << 26, most / N);
      for (int bf = 0; bf < 2; ++bf)
        for (Product p : {Product::Forward, Product::InputGrad, Product::WeightGrad})
          for (bool turn : {false, true})
            for (int planes : {1, 2, 3}) {
              const int64_t m = turn ? N : M, n = turn ? M : N;
              if (p == Product::Forward && direct_layer(bf, m, n, K)) continue;
              const DensePlan d = plan_dense(bf, p, m, n, K, planes);
              const int64_t threads = d.tile == kT128w8 || d.tile == kT64x128 || d.tile == kT256 ? 512 : 256;
              if (dense_tiles(d.tile, m, n) * threads >= 1LL << 32) ok = fail("dense launch", m, n, K, d.tile);
            }
    }
  return ok;
}

int main(int argc, char** argv) {
  std::set<std::string> s;
  if (argc == 2 && !strcmp(argv[1], "bound")) {
    const bool ok = bounds();
    if (ok) puts("ok");
    return ok ? 0 : 1;
  }
  if (argc == 2 && !strcmp(argv[1], "launches")) {
    const bool ok = launches();
    if (ok) puts("ok");
    return ok ? 0 : 1;
  }
  if (argc == 2 && !strcmp(argv[1], "dense")) {
    const int64_t sizes[] = {1, 6, 20, 30, 64, 65, 100, 128, 129, 200, 300, 512, 600, 1024, 2048, 5000, 10000, 40000, 100000, 1000000};
    for (int64_t n : sizes)
      for (int64_t in : sizes)
        for (int64_t out : sizes) dense_kernels(n, in, out, s);
  } else if (argc == 5 && !strcmp(argv[1], "dense-of")) {
    dense_kernels(atoll(argv[2]), atoll(argv[3]), atoll(argv[4]), s);
  } else if (argc == 2 && !strcmp(argv[1], "norm")) {
    for (int64_t n : {1, 3, 64, 1024})
      for (int64_t p : {1, 2, 9, 100, 1000, 10000})
        for (int64_t c : {1, 8, 16, 24, 64, 96, 435, 700, 1024, 2048, 4096, 8192, 20000, 65536})
          for (int32_t g : {1, 2, 3, 4, 5, 8, 16, 32, 64, 128, 512, 4096})
            if (g <= c && c % g == 0) norm_kernels(n, p, c, g, s);
  } else if (argc == 6 && !strcmp(argv[1], "norm-of")) {
    norm_kernels(atoll(argv[2]), atoll(argv[3]), atoll(argv[4]), (int32_t)atoll(argv[5]), s);
  } else {
    return 2;
  }
  for (const std::string& k : s) puts(k.c_str());
  return 0;
}
