// The sharing-out of kvp_rotary: with the sizes that include/kvp.h allows every launch fits a grid, and blocks of tokens cover T.  Prints the number of
// sizes walked.
#include <stdio.h>
#include <stdlib.h>

#include <random>

#include "rotary_plan.h"

using namespace kvp;

static void check(int64_t T, int64_t H) {
  if (T * H >= 1ll << 31) return;
  const int64_t tokens = rotary_tokens_block(T, H), blocks = rotary_blocks(T, H, false, false);
  const bool bad = tokens < 1 || tokens > kRotaryTokens || blocks * tokens < T || (blocks - 1) * tokens >= T || (T < 1 << 24 && tokens != std::max<int64_t>(1, 64 / H)) ||
                   fits_grid(blocks, kRotaryThreads) != (T <= (1ll << 30) - 64) ||
                   fits_grid(rotary_blocks(T, H, false, true), kRotaryThreads) != (T * H <= (1ll << 31) - 128) ||
                   fits_grid(rotary_blocks(T, H, true, true), kRotaryThreads) != (T * H <= (1ll << 30) - 64);
  if (bad) {
    printf("T %lld H %lld\n", (long long)T, (long long)H);
    exit(1);
  }
}

int main() {
  std::mt19937_64 rng(5);
  auto upto = [&](int bits) { return (int64_t)(1 + rng() % (1ull << (rng() % (bits + 1)))); };
  int64_t walked = 0;
  for (int64_t H : {1, 2, 3, 31, 32, 33, 64, 65, 127, 128, 200})
    for (int64_t edge : {1ll << 24, 1ll << 25, 1ll << 29, 1ll << 30, (1ll << 30) / H, (1ll << 31) / H, 65ll, 1ll << 12})
      for (int64_t d = -140; d <= 140; ++d)
        if (edge + d > 0) check(edge + d, H), ++walked;
  for (int i = 0; i < 1000000; ++i, ++walked) check(upto(31), upto(8));
  printf("%lld\n", (long long)walked);
  return 0;
}
