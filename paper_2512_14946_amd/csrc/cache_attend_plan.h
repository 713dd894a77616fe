// How kvp_cache_attend is shared out, and its scratch (host arithmetic; compiles without the HIP headers).
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <algorithm>

#include "kvp_math.h"

namespace kvp {

constexpr int kTileTokens = 64;   // tokens a wave works on at a time
constexpr int kTileRows = 16;     // query rows of a block
constexpr int kAttendWaves = 4;

struct AttendPlan {
  int64_t row_tiles;              // 16-row tiles of the G * W rows of a (sequence, head)
  int64_t cells;                  // (sequence, head, row tile)
  int64_t chunk, chunks;          // tokens per block, blocks per cell
  int64_t logit_stride;           // tokens per row of kept logits
  size_t out_bytes, stat_bytes, row_bytes, logit_bytes, bytes;   // partial outputs and statistics, row statistics, logits
};

inline size_t align256_bytes(size_t n) { return (n + 255) / 256 * 256; }

inline AttendPlan make_attend_plan(int64_t B, int64_t H, int64_t Hq, int64_t W, int64_t T, bool weights) {
  AttendPlan p{};
  p.row_tiles = ceil_div(Hq / H * W, kTileRows);
  p.cells = B * H * p.row_tiles;
  const int64_t step = kTileTokens * kAttendWaves;
  int64_t n = std::min(std::max<int64_t>(1, 512 / p.cells), ceil_div(T, step));
  p.chunk = ceil_div(ceil_div(T, n), step) * step;
  p.chunks = ceil_div(T, p.chunk);
  const size_t stats = align256_bytes(static_cast<size_t>(p.cells) * p.chunks * kTileRows * 2 * sizeof(float));
  if (p.chunks > 1) {
    p.out_bytes = align256_bytes(static_cast<size_t>(p.cells) * p.chunks * kTileRows * 128 * sizeof(float));
    p.stat_bytes = stats;
  }
  // Weights need the final statistics of their rows, and then the logits once more.  Up to 16 rows they are kept (4 bytes a row and token,
  // against 128 bytes of keys); for more they are formed again.
  const int64_t M = Hq / H * W, stride = ceil_div(T, kTileTokens) * kTileTokens;
  if (weights && p.row_tiles == 1 && M * stride < (1ll << 31)) {
    p.stat_bytes = stats;
    p.logit_stride = stride;
    p.logit_bytes = align256_bytes(static_cast<size_t>(p.cells) * M * p.logit_stride * sizeof(float));
  } else if (weights) {
    p.row_bytes = align256_bytes(static_cast<size_t>(p.cells) * kTileRows * 2 * sizeof(float));
  }
  p.bytes = p.out_bytes + p.stat_bytes + p.row_bytes + p.logit_bytes;
  return p;
}

}  // namespace kvp
