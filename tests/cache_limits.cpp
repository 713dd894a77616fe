// The launches of kvp_cache_attend against the limits that include/kvp.h states: every size within them fits a grid, and no launch is counted
// that does not happen.  Prints the number of sizes walked; with a shape and whether weights are asked for as arguments, the blocks of every launch and
// whether they fit.
#include <stdio.h>
#include <stdlib.h>

#include <random>

#include "cache_attend_plan.h"

using namespace kvp;

static AttendBlocks blocks(int64_t B, int64_t H, int64_t G, int64_t W, int64_t T, bool weights, AttendPlan* plan) {
  *plan = make_attend_plan(B, H, G * H, W, T, weights);
  return attend_blocks(*plan, B * H, G * W, T, weights);
}

int main(int argc, char** argv) {
  AttendPlan p;
  if (argc == 7) {
    int64_t x[6];
    for (int i = 0; i < 6; ++i) x[i] = atoll(argv[i + 1]);
    const AttendBlocks n = blocks(x[0], x[1], x[2], x[3], x[4], x[5] != 0, &p);
    printf("%lld %lld %lld %lld %d\n", (long long)n.attend, (long long)n.join_rows, (long long)n.join_sums, (long long)n.sums, attend_fits(n));
    return 0;
  }
  std::mt19937_64 rng(11);
  auto upto = [&](int bits) { return (int64_t)(1 + rng() % (1ull << (rng() % (bits + 1)))); };
  int64_t walked = 0;
  for (int i = 0; i < 2000000; ++i) {
    const int64_t B = upto(23), H = upto(8), G = upto(8), W = upto(16), T = upto(31) - 1 > 0 ? upto(30) : 1, M = G * W;
    const bool weights = i & 1;
    if (M >= 1 << 24 || B * H * ceil_div(M, M > 128 ? 256 : 16) >= (1 << 23) - 7 || (weights && B * H * ceil_div(T, 128) >= 1 << 24)) continue;
    const AttendBlocks n = blocks(B, H, G, W, T, weights, &p);
    const bool keep = weights && M <= kTileRows;
    if (!attend_fits(n) || n.attend < p.cells * p.chunks || n.attend % 8 || (n.join_rows != 0) != (p.chunks > 1) || (n.join_sums != 0) != keep ||
        (n.sums != 0) != (weights && !keep) || (p.chunks > 1 && n.join_rows < p.cells * std::min(M, p.tile_rows))) {
      printf("B %lld H %lld G %lld W %lld T %lld weights %d\n", (long long)B, (long long)H, (long long)G, (long long)W, (long long)T, weights);
      return 1;
    }
    ++walked;
  }
  printf("%lld\n", (long long)walked);
  return 0;
}
