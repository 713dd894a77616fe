// How kvp_rotary is shared out (host arithmetic; compiles without the HIP headers).
#pragma once

#include <stdint.h>

#include <algorithm>

#include "kvp_math.h"

namespace kvp {

constexpr int kRotaryThreads = 256;
constexpr int kRotaryRows = 4;        // rows per lane whose loads are all ahead of the arithmetic
constexpr int kRotaryTokens = 64;     // tokens of a block, at most

// Tokens of a block whose heads share positions: 64 rows; more where a launch would not hold the blocks otherwise.
inline int64_t rotary_tokens_block(int64_t T, int64_t H) {
  const int64_t most_blocks = (1ll << 32) / kRotaryThreads - 1;
  return std::min<int64_t>(kRotaryTokens, std::max(std::max<int64_t>(1, 64 / H), ceil_div(T, most_blocks)));
}

// Blocks per layer: any (half layout, rotary_dim no multiple of 16): 16 lanes a row; per_head: 8 lanes a row; otherwise by tokens.
inline int64_t rotary_blocks(int64_t T, int64_t H, bool any, bool per_head) {
  if (any) return ceil_div(T * H, kRotaryRows * kRotaryThreads / 16);
  if (per_head) return ceil_div(T * H, kRotaryRows * kRotaryThreads / 8);
  return ceil_div(T, rotary_tokens_block(T, H));
}

}  // namespace kvp
