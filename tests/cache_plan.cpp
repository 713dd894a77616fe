// Checks the sharing-out of kvp_cache_attend over its range: the chunks cover every token once and none is empty, what the kernels write
// lies inside the scratch memory, and the parts of the scratch do not overlap.  Prints the number of plans walked; with a shape as
// arguments, the rows of a tile and the number of chunks.
#include <stdio.h>
#include <stdlib.h>

#include <random>

#include "cache_attend_plan.h"

using namespace kvp;

static void fail(const char* what, int64_t B, int64_t H, int64_t G, int64_t W, int64_t T) {
  printf("%s: B %lld H %lld G %lld W %lld T %lld\n", what, (long long)B, (long long)H, (long long)G, (long long)W, (long long)T);
  exit(1);
}

static void check(int64_t B, int64_t H, int64_t G, int64_t W, int64_t T, bool weights) {
  const AttendPlan p = make_attend_plan(B, H, G * H, W, T, weights);
  const int64_t M = G * W;
  if (p.tile_rows != kTileRows && p.tile_rows != 2 * kTileRows && p.tile_rows != kManyRows) fail("rows of a tile", B, H, G, W, T);
  if (p.row_tiles * p.tile_rows < M || (p.row_tiles - 1) * p.tile_rows >= M) fail("row tiles", B, H, G, W, T);
  if (p.cells != B * H * p.row_tiles) fail("cells", B, H, G, W, T);
  if (p.chunk <= 0 || p.chunk % (kTileTokens * kAttendWaves)) fail("chunk", B, H, G, W, T);
  if (p.chunks * p.chunk < T || (p.chunks - 1) * p.chunk >= T) fail("chunks do not cover the tokens", B, H, G, W, T);
  // partial results: a row of 128 floats and a pair of statistics per (cell, chunk, tile row)
  const size_t parts = (size_t)p.cells * p.chunks * p.tile_rows;
  const bool keep = weights && M <= kTileRows;
  if (p.chunks > 1 ? p.out_bytes < parts * 512 : p.out_bytes != 0) fail("partial outputs", B, H, G, W, T);
  if ((p.chunks > 1 || keep) && p.stat_bytes < parts * 8) fail("statistics", B, H, G, W, T);
  // kept logits: whole tiles of 64 tokens of every row; several row tiles never keep them
  if (keep != (p.logit_bytes != 0)) fail("kept logits", B, H, G, W, T);
  if (keep && (p.row_tiles != 1 || p.logit_stride % kTileTokens || p.logit_stride < T || p.logit_bytes < (size_t)(B * H * M * p.logit_stride) * 4))
    fail("logits", B, H, G, W, T);
  if (weights && !keep && p.row_bytes < (size_t)p.cells * p.tile_rows * 4) fail("row statistics", B, H, G, W, T);
  if (p.out_bytes % 256 || p.stat_bytes % 256 || p.row_bytes % 256 || p.bytes < p.out_bytes + p.stat_bytes + p.row_bytes + p.logit_bytes)
    fail("layout", B, H, G, W, T);
}

int main(int argc, char** argv) {
  if (argc == 6) {
    int64_t x[5];
    for (int i = 0; i < 5; ++i) x[i] = atoll(argv[i + 1]);
    const AttendPlan p = make_attend_plan(x[0], x[1], x[1] * x[2], x[3], x[4], false);
    printf("%lld %lld\n", (long long)p.tile_rows, (long long)p.chunks);
    return 0;
  }
  std::mt19937_64 rng(7);
  auto upto = [&](int bits) { return (int64_t)(1 + rng() % (1ull << (rng() % (bits + 1)))); };
  int64_t plans = 0;
  for (int64_t T : {1, 63, 64, 65, 255, 256, 257, 511, 512, 513, 1024, 1025, 131072, 131073, 1 << 20})
    for (int64_t M : {1, 15, 16, 17, 31, 32, 33, 96, 97, 128, 129, 255, 256, 257, 4096})
      for (int64_t cells : {1, 2, 255, 256, 257, 511, 512, 513, 4096})
        for (int weights = 0; weights < 2; ++weights, ++plans) check(cells, 1, 1, M, T, weights != 0);
  for (int i = 0; i < 200000; ++i, ++plans) check(upto(9), upto(6), upto(6), upto(12), upto(20), i & 1);
  printf("%lld\n", (long long)plans);
  return 0;
}
