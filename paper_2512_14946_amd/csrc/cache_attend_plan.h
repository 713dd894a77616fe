// How kvp_cache_attend is shared out, and its scratch (host arithmetic; compiles without the HIP headers).
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <algorithm>

#include "kvp_math.h"

namespace kvp {

constexpr int kTileTokens = 64;   // tokens a wave works on at a time
constexpr int kTileRows = 16;     // query rows of a block that reads operands straight from memory, or twice that, see attend_tile_rows
constexpr int kFewRows = 128;     // rows up to which those blocks are taken
constexpr int kManyRows = 256;    // ... of a block that shares its tiles by way of LDS
constexpr int kAttendWaves = 4;
constexpr int kSumTokens = 128;   // tokens of a block that sums the weights of many rows
constexpr int kJoinTokens = 1024; // ... of a block of the joining kernel that sums weights from logits
constexpr int kUnits = 256;       // CUs

struct AttendPlan {
  int64_t tile_rows, row_tiles;   // rows of a tile; tiles of the G * W rows of a (sequence, head)
  int64_t cells;                  // (sequence, head, row tile)
  int64_t chunk, chunks;          // tokens per block, blocks per cell
  int64_t logit_stride;           // tokens per row of kept logits
  size_t out_bytes, stat_bytes, row_bytes, logit_bytes, bytes;   // partial outputs and statistics, row statistics, logits
};

inline size_t align256_bytes(size_t n) { return (n + 255) / 256 * 256; }

// Tokens from which M rows (17 .. 96) of n_bh (sequence, head)s take tiles of 32.
inline int64_t wide_tiles_from(int64_t n_bh, int64_t M) { return std::max<int64_t>(1024, ceil_div(3 << 18, n_bh * ceil_div(M, kTileRows))); }

// Rows of a tile.  Small tiles read and decode every code once per tile (by way of the L2 after the first), those of 256 once, but a wave
// has 32 rows of them and few rows leave most waves without.  Tiles of 32 decode half as often as tiles of 16 and take longer to begin and end.  us,
// tiles of 16 / 32 / 256:
//   16 x 8 x 8192 keys   60 / 54 / 132 (20 rows), 99 / 71 / 139 (64), 138 / 118 / 146 (96), 175 / 126 / 154 (128), 171 (32) / 159 (160)
//   4 x 4 x 30000        34 / 30 / 68,  52 / 40 / 69,  76 / 52 / 72,  90 / 63 / 75,  78 / 79
//   1 x 8 x 32768        20 / 21 / -,   29 / 25 / -,   40 / 32 / - (88)
//   1 x 8 x 8192         12 / 14 / 20,  14 / 15 / 21,  18 / 18 / 23,  21 / 18 / 25,  22 / 27
//   64 x 8 x 512         19 / 22 / -,   35 / 40 / -,   50 / 59 / - (88)
inline int64_t attend_tile_rows(int64_t n_bh, int64_t M, int64_t T) {
  if (M <= kTileRows) return kTileRows;
  if (M > kFewRows) return kManyRows;
  return M > 96 || T >= wide_tiles_from(n_bh, M) ? 2 * kTileRows : kTileRows;
}

inline AttendPlan make_attend_plan_of(int64_t tile_rows, int64_t B, int64_t H, int64_t M, int64_t T, bool weights) {
  AttendPlan p{};
  const int64_t stride = ceil_div(T, kTileTokens) * kTileTokens;
  p.tile_rows = tile_rows;
  p.row_tiles = ceil_div(M, p.tile_rows);
  p.cells = B * H * p.row_tiles;
  const int64_t step = kTileTokens * kAttendWaves;
  // Chunks: the fewest of a cell that leave CUs idle for less than a fifth of the time, in rounds of a block per CU (a second block per CU adds
  // partial results, and little that four loads in flight per lane do not do).  256 against 512 blocks, us: 61, 71 (16 x 8 x 8192 keys, 32 rows),
  // 34, 40 (4 x 4 x 30000), 89, 90 (4 x 4 x 131072, 7 rows), 49, 62 (8 x 2048, 2048 rows); 480 against 192: 76, 87 (4 x 4 x 30000, 96 rows).
  // More than a round only for chunks that outweigh their partial results: 1056 blocks in 5 rounds against 264 in 2: 146, 200 (33 x 8 x 12000, 4
  // rows); but 45, 38 with chunks of 768 (130 x 2 x 2100), and 84, 78 with 2000 for 528 cells (33 x 8 x 4000, 28 rows).
  // Those are times of tiles of 16 and 256.  Tiles of 32, us with 1, 2, 3, 4, 5, 8 chunks, and with what the rule takes: 73, 89, 95, 101, 109, 124, 73 (16 x 8 x
  // 8192 keys, 64 rows); 190, 104, 76, 60, 53, 66, 53 (4 x 4 x 30000, 96); 212, 191, 183, 189, 184, 207, 189 (33 x 8 x 12000, 20); 71, 48, 63, 54, 51, 57, 51
  // (12 x 8 x 8192, 20); 131, 78, 98, 82, 74, 77, 73 (3 x 8 x 20000, 128); 203, 110, 78, 61, 52, 37, 33 (1 x 8 x 32768, 96).
  const int64_t first = std::max<int64_t>(1, kUnits / p.cells);
  const int64_t last = std::min(first + 8, std::max(first, T / (p.tile_rows == kManyRows ? 4096 : p.cells < kUnits ? 1024 : 2048)));
  int64_t n = first;
  for (int64_t i = first, best = 0; i <= last && best < 52; ++i) {
    const int64_t full = i * p.cells * 64 / (ceil_div(i * p.cells, kUnits) * kUnits);   // how full the CUs are, of 64
    if (full > best) best = full, n = i;
  }
  n = std::min(n, ceil_div(T, step));
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

inline AttendPlan make_attend_plan(int64_t B, int64_t H, int64_t Hq, int64_t W, int64_t T, bool weights) {
  const int64_t M = Hq / H * W, rows = attend_tile_rows(B * H, M, T);
  AttendPlan p = make_attend_plan_of(rows, B, H, M, T, weights);
  // scratch that serves every smaller T: the smaller tiles of fewer tokens too
  if (rows == 2 * kTileRows && M <= 96)
    p.bytes = std::max(p.bytes, make_attend_plan_of(kTileRows, B, H, M, wide_tiles_from(B * H, M) - 1, weights).bytes);
  return p;
}

// Blocks of the launches that a plan takes (0: none): the attention's (512 threads at most), the joining kernel's (rows of chunks, and weights
// from kept logits; 256) and those that sum the weights of many rows (256).
struct AttendBlocks {
  int64_t attend, join_rows, join_sums, sums;
};

inline AttendBlocks attend_blocks(const AttendPlan& p, int64_t n_bh, int64_t M, int64_t T, bool weights) {
  AttendBlocks n{};
  n.attend = ceil_div(p.cells * p.chunks, 8) * 8;   // a whole number of blocks for each of the 8 XCDs
  if (p.chunks > 1) n.join_rows = p.cells * std::min(M, p.tile_rows);
  if (p.logit_bytes) n.join_sums = p.cells * ceil_div(T, kJoinTokens);
  if (weights && !p.logit_bytes) n.sums = n_bh * ceil_div(T, kSumTokens);
  return n;
}

inline bool attend_fits(const AttendBlocks& n) {
  return fits_grid(n.attend, 512) && fits_grid(n.join_rows + n.join_sums, 256) && fits_grid(n.sums, 256);
}

}  // namespace kvp
