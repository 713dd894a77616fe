// How kvp_cache_attend is shared out, and its scratch (host arithmetic; compiles without the HIP headers).
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <algorithm>

#include "kvp_math.h"

namespace kvp {

constexpr int kTileTokens = 64;   // tokens a wave works on at a time
constexpr int kTileRows = 16;     // query rows of a block that reads operands straight from memory
constexpr int kFewRows = 32;      // rows up to which tiles of 16 are taken, see make_attend_plan
constexpr int kManyRows = 256;    // ... of a block that shares its tiles by way of LDS
constexpr int kAttendWaves = 4;

struct AttendPlan {
  int64_t tile_rows, row_tiles;   // rows of a tile; tiles of the G * W rows of a (sequence, head)
  int64_t cells;                  // (sequence, head, row tile)
  int64_t chunk, chunks;          // tokens per block, blocks per cell
  int64_t logit_stride;           // tokens per row of kept logits
  size_t out_bytes, stat_bytes, row_bytes, logit_bytes, bytes;   // partial outputs and statistics, row statistics, logits
};

inline size_t align256_bytes(size_t n) { return (n + 255) / 256 * 256; }

inline AttendPlan make_attend_plan(int64_t B, int64_t H, int64_t Hq, int64_t W, int64_t T, bool weights) {
  AttendPlan p{};
  const int64_t M = Hq / H * W, stride = ceil_div(T, kTileTokens) * kTileTokens;
  // Tiles of 16 rows read every key and value once per tile, the wide ones once, but a wave has 32 rows and few rows leave most waves
  // without.  Wide over 16-row time at 16 x 8 x 8192 keys: 1.42 (32 rows), 0.95 (40, 48), 0.83 (64), 0.63 (80), 0.46 (128); at 1 x 8 x 8192 1.35
  // (32), 1.18 (40, 48), 1.16 (64), 0.87 (80): 33 to 64 rows are even on the whole, and few keys cost little either way.
  p.tile_rows = M <= kFewRows ? kTileRows : kManyRows;
  p.row_tiles = ceil_div(M, p.tile_rows);
  p.cells = B * H * p.row_tiles;
  const int64_t step = kTileTokens * kAttendWaves;
  const int64_t n = std::min(std::max<int64_t>(1, 512 / p.cells), ceil_div(T, step));
  p.chunk = ceil_div(ceil_div(T, n), step) * step;
  p.chunks = ceil_div(T, p.chunk);
  // sized for n chunks, which grow with T where the rounded ones need not: scratch for a T serves every smaller one
  const size_t stats = align256_bytes(static_cast<size_t>(p.cells) * n * p.tile_rows * 2 * sizeof(float));
  if (p.chunks > 1) {
    p.out_bytes = align256_bytes(static_cast<size_t>(p.cells) * n * p.tile_rows * 128 * sizeof(float));
    p.stat_bytes = stats;
  }
  // Weights need the final statistics of their rows, and then the logits once more.  Up to 16 rows they are kept (4 bytes a row and token,
  // against 128 bytes of keys); for more they are formed again.
  if (weights && M <= kTileRows) {
    p.stat_bytes = stats;
    p.logit_stride = stride;
    p.logit_bytes = align256_bytes(static_cast<size_t>(p.cells) * M * p.logit_stride * sizeof(float));
  } else if (weights) {
    p.row_bytes = align256_bytes(static_cast<size_t>(p.cells) * p.tile_rows * sizeof(float));
  }
  p.bytes = p.out_bytes + p.stat_bytes + p.row_bytes + p.logit_bytes;
  return p;
}

}  // namespace kvp
