// Integer arithmetic of host code that also has to compile without the HIP headers.
#pragma once

#include <stdint.h>

namespace kvp {

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// A launch takes fewer than 2^32 threads.
inline bool fits_grid(int64_t blocks, int64_t threads) { return blocks < (1ll << 32) / threads; }

}  // namespace kvp
