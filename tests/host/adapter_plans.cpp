// Checks the adapters' plans (csrc/adapt_plan.h) on the CPU; see ../test_adapter_plans.py.
//   bound     every call's partial sums fit the workspace of any larger call, whose size is bounded
//   kernels   the kernels that calls of any size can take, one a line
//   of T N I O  the kernels that a forward and a backward with dx of N rows take (T: fp32 or bf16)
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <set>
#include <string>
#include <vector>

#include "adapt_plan.h"

using namespace ot;

// Partial sums that a bank may hold: 512 MB of fp32 values.
constexpr int64_t kMost = 128LL << 20;

int64_t workspace(const AdaptSizes& a, int64_t n) {
#ifdef ROWS_ONLY
  // the pass bounded by its rows alone
  if (a.out >= 16384) {
    const int64_t chunks = std::max<int64_t>(1, std::min<int64_t>(4, a.out / 512 * a.G / 1024));
    return std::max(part_values(a, n), ceil_div(a.out, chunks * kPassThreads) * std::min(n, kPassMaxRows) * a.RP);
  }
#endif
  return part_values(a, n);
}

int bound() {
  int64_t checked = 0;
  std::vector<int64_t> rows;
  for (int64_t n = 1; n <= 300; ++n) rows.push_back(n);
  for (int64_t n = 310; n <= (1 << 20); n += n / 12) rows.push_back(n);
  for (int64_t n : {512, 1024, 4095, 4096, 4097, 1 << 20}) rows.push_back(n);
  for (int64_t in : {1, 16, 437, 1024, 2048, 20500, 131072})
    for (int64_t out : {1, 256, 6561, 16383, 16384, 70001, 1000000, 1 << 26})
      for (int32_t rp : {16, 64})
        for (int32_t g : {1, 8, 300, 4096})
          for (bool bf16 : {false, true}) {
            const AdaptSizes a{in, out, rp, g, bf16};
            for (int64_t most : {1, 33, 300, 1024, 4096, 5000, 1 << 20}) {
              const int64_t ws = workspace(a, most);
              if (ws > kMost) {
                printf("in %lld out %lld rank %d adapters %d: %lld values for %lld rows\n", (long long)in, (long long)out,
                       rp, g, (long long)ws, (long long)most);
                return 1;
              }
              for (int64_t n : rows) {
                if (n > most) continue;
                const int64_t ask = std::max(std::max(shrink_values(a, n, in), shrink_values(a, n, out)),
                                             std::max(pass_values(a, n), gradient_values(a, n)));
                ++checked;
                if (ask > ws) {
                  printf("in %lld out %lld rank %d adapters %d: %lld rows of at most %lld ask for %lld of %lld values\n",
                         (long long)in, (long long)out, rp, g, (long long)n, (long long)most, (long long)ask,
                         (long long)ws);
                  return 1;
                }
              }
            }
          }
  printf("%lld calls ok\n", (long long)checked);
  return 0;
}

std::string kernel(bool bf16, bool forward, int64_t n, int64_t in, int64_t out) {
  const AdaptPlan p = forward ? plan_expand(bf16, true, n, out, in) : plan_expand(bf16, false, n, in, out);
  char s[80];
  snprintf(s, sizeof s, "%s %s %dx%d%s", bf16 ? "bf16" : "fp32", forward ? "forward" : "gradient", kAdaptTileRows[p.tile],
           kAdaptTileCols[p.tile], p.splits > 1 ? " split" : "");
  return s;
}

// How the rows are sorted and which launches take dy's two low-rank products.
std::string low_rank(const AdaptSizes& a, int64_t n) {
  return pass_chunks(a, n) ? "pass" : shrink_splits(n, a.out, a.G) > 1 ? "split shrink" : "shrink";
}

int main(int argc, char** argv) {
  if (argc == 2 && !strcmp(argv[1], "bound")) return bound();
  if (argc == 2 && !strcmp(argv[1], "kernels")) {
    std::set<std::string> all;
    for (bool bf16 : {false, true})
      for (int64_t n = 1; n <= 1 << 20; n += 1 + n / 9)
        for (int64_t in = 1; in <= 1 << 26; in += 1 + in / 3)
          for (int64_t out = 1; out <= 1 << 26; out += 1 + out / 3) {
            all.insert(kernel(bf16, true, n, in, out));
            all.insert(kernel(bf16, false, n, in, out));
            all.insert(std::string(bf16 ? "bf16 " : "fp32 ") + low_rank(AdaptSizes{in, out, 16, 8, bf16}, n));
          }
    for (const std::string& s : all) puts(s.c_str());
    return 0;
  }
  if (argc == 6 && !strcmp(argv[1], "of")) {
    const bool bf16 = !strcmp(argv[2], "bf16");
    const int64_t n = atoll(argv[3]), in = atoll(argv[4]), out = atoll(argv[5]);
    puts(kernel(bf16, true, n, in, out).c_str());
    puts(kernel(bf16, false, n, in, out).c_str());
    puts((std::string(bf16 ? "bf16 " : "fp32 ") + low_rank(AdaptSizes{in, out, 16, 8, bf16}, n)).c_str());
    return 0;
  }
  return 2;
}
