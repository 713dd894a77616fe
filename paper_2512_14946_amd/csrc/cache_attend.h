// kvp_cache_attend: what its kernels share.
#pragma once

#include "cache_attend_plan.h"
#include "cache_common.h"

namespace kvp {

constexpr float kLog2e = 1.4426950408889634f;
// How far (base 2) the reference of a row is set below its largest logit.  A probability times its page's share of the reference scale is rounded to
// a half, which has 11 bits down to 2^-14 and steps of 2^-24 below.  With the reference AT the largest logit, rows that give 0.9 to 0.995 of their
// weight to a token of no value, over 131072 tokens, came out 10 % (tiles of 16 rows) to 44 % (256) wrong, as all others were a step or two; 2^10
// below it they keep their bits, at no cost: 987 us and 983 (4 x 8 x 16384 keys, 4096 rows), 88.8 and 89.0 (4 x 4 x 131072, 7 rows).
constexpr float kBelow = 10.0f;
constexpr float kLeastScale = 0x1p-100f;    // value scales below this count as this one's fractions
constexpr float kLeast = -3.402823466e38f;

struct AttendArgs {
  CacheArgs c;
  const uint16_t* q;
  uint16_t* out;
  int64_t q_sb, q_sw, q_sh, o_sb, o_sw, o_sh;
  const int32_t* q_lens;
  uint32_t W, G, M, tile_rows, row_tiles, max_len, chunk, chunks;
  uint32_t blocks, per_xcd;                 // blocks of the attention launch; of an XCD
  FastDiv div_tiles, div_h, div_g, div_bh;  // div_bh: by the blocks of a (sequence, head)
  float scale2;                             // scale * log2(e)
  int32_t causal;
  float* part_out;                          // [cell][chunk][tile row][128] divided by the chunk's sum, or null (one chunk)
  float2* part_stat;                        // [cell][chunk][tile row] (reference, sum)
  float* row_bias;                          // [cell][tile row]: reference + log2(sum), +inf for an empty row: weights of more than 16 rows
  float* logits;                            // [cell][tile of 64 tokens][i][M][g][4], see the kernel: weights of a single row tile
  int64_t logit_stride;
  const float* acc_in;
  float* acc_out;
  int64_t acc_stride;
};

// What a row tile of a (sequence, head) sees.
struct Rows {
  uint32_t b, h, tile, n;                   // n: tokens of the sequence
  int32_t m;                                // query tokens of the sequence
  uint32_t least, most;                     // tokens seen by the tile's first and last row (most: by any)
};

// Block of an attention launch -> its number in the order (sequence, head; chunk; row tile), its cell and its chunk.  Blocks reach the 8
// XCDs in turn, so an XCD takes a run of them: the row tiles of a chunk share its keys and values in one L2.
__device__ __forceinline__ bool block_of(const AttendArgs& a, uint32_t& cell, uint32_t& chunk) {
  const uint32_t id = (blockIdx.x & 7) * a.per_xcd + (blockIdx.x >> 3);
  const uint32_t bh = a.div_bh.quot(id), in_bh = id - bh * a.chunks * a.row_tiles;
  chunk = a.div_tiles.quot(in_bh);
  cell = bh * a.row_tiles + (in_bh - chunk * a.row_tiles);
  return id < a.blocks;
}

__device__ __forceinline__ uint32_t seen_by(const AttendArgs& a, uint32_t n, int32_t m, uint32_t w) {
  if (!a.causal) return n;
  const int64_t p = static_cast<int64_t>(n) - m + w + 1;
  return p < 0 ? 0u : static_cast<uint32_t>(p);   // w < m: at most n
}

__device__ __forceinline__ Rows rows_of(const AttendArgs& a, uint32_t cell) {
  Rows r;
  const uint32_t bh = a.div_tiles.quot(cell);
  r.tile = a.row_tiles - 1 - (cell - bh * a.row_tiles);   // the tiles that see most begin first
  r.b = a.div_h.quot(bh);
  r.h = bh - r.b * a.c.H;
  r.n = min(cache_len(a.c, r.b), a.max_len);
  r.m = static_cast<int32_t>(a.W);
  if (a.q_lens) r.m = min(max(a.q_lens[r.b], 0), r.m);
  const uint32_t w0 = a.div_g.quot(r.tile * a.tile_rows), w1 = a.div_g.quot(min(r.tile * a.tile_rows + a.tile_rows, a.M) - 1);
  r.least = r.most = 0;
  if (static_cast<int32_t>(w0) < r.m) {
    r.least = seen_by(a, r.n, r.m, w0);
    r.most = seen_by(a, r.n, r.m, min(w1, static_cast<uint32_t>(r.m) - 1));
  }
  return r;
}

// reference + log2(sum) of a row, from the mantissa of the sum (the instruction is best below 1)
__device__ __forceinline__ float bias_of(float m, float z) {
  return z > 0.0f ? m + static_cast<float>(__builtin_amdgcn_frexp_expf(z)) + __builtin_amdgcn_logf(__builtin_amdgcn_frexp_mantf(z)) : INFINITY;
}

// Table entry of the 16-token run that starts at token t, and the pool cell that it names; runs behind the last token take its page.
__device__ __forceinline__ int32_t run_entry(const AttendArgs& a, uint32_t b, uint32_t t, uint32_t n) {
  return a.c.table[static_cast<int64_t>(b) * a.c.table_stride + (min(t, n - 1) >> a.c.bs_log2)];
}
__device__ __forceinline__ int64_t entry_cell(const AttendArgs& a, uint32_t h, int32_t entry) {
  return static_cast<int64_t>(clamp_page(a.c, entry)) * a.c.H + h;
}
__device__ __forceinline__ int64_t run_cell(const AttendArgs& a, uint32_t b, uint32_t h, uint32_t t, uint32_t n) {
  return entry_cell(a, h, run_entry(a, b, t, n));
}

// Tiles of kManyRows: attention of all chunks (to a.out, or partial results).  More than 16 query rows: the weights of the tokens.
void attend_rows_launch(const AttendArgs& a, int format, hipStream_t st);
void weights_rows_launch(const AttendArgs& a, int format, hipStream_t st);

}  // namespace kvp
