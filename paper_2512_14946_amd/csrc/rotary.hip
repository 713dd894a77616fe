// kvp_rotary: rotary positions.  Every pair (a, b) of a row turns by t = position * freq[i]:
//   y_a = m (a cos t - b sin t),  y_b = m (b cos t + a sin t)
// The angle of a far position has too many bits for fp32 (131072 radians leave an error of 0.004), so position * freq / 2 pi and its
// fraction are formed in double; the fraction of a turn in [-1/2, 1/2] goes to v_sin_f32 / v_cos_f32, which take turns and are
// off by at most 1.25e-7 there (all 2^24 multiples of 2^-24 compared with double; the results are rounded to bf16, 2^-9).
//
// Bound by HBM (x is read and written once): eight lanes share a row, each owns two 16-byte pieces, which hold both channels of
// its eight pairs (half layout: pieces rotary_dim / 2 apart).  Where heads share a position a block takes some tokens with all
// their heads, and one sine and cosine per (token, pair) go to LDS once and serve every head: 4 x 8192 x 8 rows 23.7 us, 5.7 TB/s.  With a position
// per head a lane forms those of its own eight pairs: 80 x 4916 x 8 rows 273 us, 6.0 TB/s (580 us by way of
// LDS with a library sincospi of 25 instructions).  Pairs that do not fall on such pieces (half layout, rotary_dim not a multiple of 16) take a
// kernel whose lanes find the other channel in LDS: 63 x 1944 x 8 rows, 2 of 128 channels, 85 us, 5.9 TB/s (a wave per row, two bytes a
// lane: 276); 34 channels 107.

#include <math.h>

#include "kvp_common.h"
#include "quant_device.h"
#include "rotary_plan.h"

namespace kvp {
namespace {

constexpr int kThreads = kRotaryThreads;
constexpr int kRows = kRotaryRows;

struct RotaryArgs {
  const uint16_t* x;
  uint16_t* out;
  int64_t x_sl, x_st, x_sh, o_sl, o_st, o_sh;  // elements
  const int32_t* pos;
  int64_t p_sl, p_st, p_sh;
  const double* freq;
  uint32_t T, H, pairs;                        // pairs = rotary_dim / 2
  uint32_t tokens_block;                       // tokens of a block, heads sharing a position
  FastDiv div_h, div_pairs;
  float mscale, sign;
  bool copy;                                   // out is not x: channels behind rotary_dim are copied
};

constexpr double kTurn = 0.15915494309189535;   // 1 / (2 pi)

// cosine and sine (times mscale, the sine with the direction's sign) of a position's pair; freq in turns
__device__ __forceinline__ float2 turn_of(const RotaryArgs& a, int32_t pos, double freq) {
  double r = static_cast<double>(pos) * freq;
  r -= __builtin_rint(r);
  const float f = static_cast<float>(r);
  return make_float2(__builtin_amdgcn_cosf(f) * a.mscale, __builtin_amdgcn_sinf(f) * (a.mscale * a.sign));
}

__device__ __forceinline__ void rotate(float& x, float& y, float2 cs) {
  const float p = fmaf(x, cs.x, -(y * cs.y)), q = fmaf(y, cs.x, x * cs.y);
  x = p;
  y = q;
}

__device__ __forceinline__ uint4 rotate_pair8(uint4& lo, uint4 hi, const float2* cs) {   // half layout: 8 pairs over two pieces
  uint32_t* l = reinterpret_cast<uint32_t*>(&lo);
  uint32_t* h = reinterpret_cast<uint32_t*>(&hi);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float a0 = bf16lo(l[i]), a1 = bf16hi(l[i]), b0 = bf16lo(h[i]), b1 = bf16hi(h[i]);
    rotate(a0, b0, cs[2 * i]);
    rotate(a1, b1, cs[2 * i + 1]);
    l[i] = pack_bf16x2(a0, a1);
    h[i] = pack_bf16x2(b0, b1);
  }
  return hi;
}

__device__ __forceinline__ uint4 rotate_piece(uint4 v, const float2* cs, uint32_t first, uint32_t pairs) {   // interleaved: 4 pairs of a piece, the first of them `first`
  uint32_t* w = reinterpret_cast<uint32_t*>(&v);
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i) {
    if (first + i < pairs) {
      float a = bf16lo(w[i]), b = bf16hi(w[i]);
      rotate(a, b, cs[i]);
      w[i] = pack_bf16x2(a, b);
    }
  }
  return v;
}

// The pieces of lane j of a row: half layout (rotary_dim a multiple of 16) 8 j and 8 j + rotary_dim / 2 while there are pairs, then
// two of the rest each.
template <int LAYOUT>
__device__ __forceinline__ bool pieces_of(const RotaryArgs& a, uint32_t j, uint32_t& c0, uint32_t& c1) {
  if (LAYOUT == KVP_ROTARY_INTERLEAVED) {
    c0 = 8 * j;
    c1 = 64 + 8 * j;
    return true;
  }
  const bool turns = 8 * j < a.pairs;
  c0 = turns ? 8 * j : 2 * a.pairs + 16 * (j - a.pairs / 8);
  c1 = turns ? c0 + a.pairs : c0 + 8;
  return turns;
}

// One position for all heads of a token.
template <int LAYOUT>
__global__ __launch_bounds__(kThreads) void rotary_kernel(const RotaryArgs a) {
  __shared__ float2 cs_s[kRotaryTokens * 64];
  const uint32_t l = blockIdx.y, token0 = blockIdx.x * a.tokens_block, tokens = min(a.tokens_block, a.T - token0);
  for (uint32_t i = threadIdx.x; i < tokens * a.pairs; i += kThreads) {
    const uint32_t u = a.div_pairs.quot(i), p = i - u * a.pairs;
    const int32_t pos = a.pos[static_cast<int64_t>(l) * a.p_sl + static_cast<int64_t>(token0 + u) * a.p_st];
    cs_s[u * 64 + p] = turn_of(a, pos, a.freq[p] * kTurn);
  }
  __syncthreads();
  const uint32_t rows = tokens * a.H;
  const uint16_t* x_l = a.x + static_cast<int64_t>(l) * a.x_sl;
  uint16_t* o_l = a.out + static_cast<int64_t>(l) * a.o_sl;
  uint32_t c0, c1;
  const bool turns = pieces_of<LAYOUT>(a, threadIdx.x & 7, c0, c1);
  if (!turns && !a.copy) return;
  for (uint32_t r0 = threadIdx.x >> 3; r0 < rows; r0 += kRows * kThreads / 8) {
    uint4 v[kRows][2];
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
      const uint32_t r = r0 + k * (kThreads / 8), u = a.div_h.quot(r), t = token0 + u, h = r - u * a.H;
      if (r >= rows) continue;
      const uint16_t* src = x_l + static_cast<int64_t>(t) * a.x_st + static_cast<int64_t>(h) * a.x_sh;
      v[k][0] = load_stream16(src + c0);
      v[k][1] = load_stream16(src + c1);
    }
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
      const uint32_t r = r0 + k * (kThreads / 8), u = a.div_h.quot(r), t = token0 + u, h = r - u * a.H;
      if (r >= rows) continue;
      if (LAYOUT == KVP_ROTARY_HALF) {
        if (turns) v[k][1] = rotate_pair8(v[k][0], v[k][1], cs_s + u * 64 + c0);
      } else {
        v[k][0] = rotate_piece(v[k][0], cs_s + u * 64 + c0 / 2, c0 / 2, a.pairs);
        v[k][1] = rotate_piece(v[k][1], cs_s + u * 64 + c1 / 2, c1 / 2, a.pairs);
      }
      uint16_t* dst = o_l + static_cast<int64_t>(t) * a.o_st + static_cast<int64_t>(h) * a.o_sh;
      store_stream16(dst + c0, v[k][0]);
      store_stream16(dst + c1, v[k][1]);
    }
  }
}

// A position for every row.

template <int LAYOUT>
__global__ __launch_bounds__(kThreads) void rotary_rows_kernel(const RotaryArgs a) {
  const uint32_t l = blockIdx.y, j = threadIdx.x & 7, n_rows = a.T * a.H;
  uint32_t c0, c1;
  const bool turns = pieces_of<LAYOUT>(a, j, c0, c1);
  if (!turns && !a.copy) return;
  double f[8];   // of this lane's pairs, in turns
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t p = LAYOUT == KVP_ROTARY_HALF ? c0 + i : (i < 4 ? c0 / 2 + i : c1 / 2 + i - 4);
    f[i] = turns && p < a.pairs ? a.freq[p] * kTurn : 0.0;
  }
  const uint32_t row0 = blockIdx.x * (kRows * kThreads / 8) + (threadIdx.x >> 3);
  uint4 v[kRows][2];
  int32_t pos[kRows];
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    const uint32_t row = row0 + k * (kThreads / 8), t = a.div_h.quot(row), h = row - t * a.H;
    if (row >= n_rows) continue;
    const uint16_t* src = a.x + static_cast<int64_t>(l) * a.x_sl + static_cast<int64_t>(t) * a.x_st + static_cast<int64_t>(h) * a.x_sh;
    pos[k] = a.pos[static_cast<int64_t>(l) * a.p_sl + static_cast<int64_t>(t) * a.p_st + static_cast<int64_t>(h) * a.p_sh];
    v[k][0] = load_stream16(src + c0);
    v[k][1] = load_stream16(src + c1);
  }
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    const uint32_t row = row0 + k * (kThreads / 8), t = a.div_h.quot(row), h = row - t * a.H;
    if (row >= n_rows) continue;
    if (turns) {
      float2 cs[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) cs[i] = turn_of(a, pos[k], f[i]);
      if (LAYOUT == KVP_ROTARY_HALF) {
        v[k][1] = rotate_pair8(v[k][0], v[k][1], cs);
      } else {
        v[k][0] = rotate_piece(v[k][0], cs, c0 / 2, a.pairs);
        v[k][1] = rotate_piece(v[k][1], cs + 4, c1 / 2, a.pairs);
      }
    }
    uint16_t* dst = a.out + static_cast<int64_t>(l) * a.o_sl + static_cast<int64_t>(t) * a.o_st + static_cast<int64_t>(h) * a.o_sh;
    store_stream16(dst + c0, v[k][0]);
    store_stream16(dst + c1, v[k][1]);
  }
}

// Half layout with any even rotary_dim: 16 lanes share a row, a 16-byte piece each; the other channel of a pair lies anywhere in the row and
// comes by way of LDS.  Both lanes of a pair work out its turn.  A row may be turned in place: it is in LDS before any of it is written.
constexpr int kRowPitch = kHeadDim + 8;
__global__ __launch_bounds__(kThreads) void rotary_any_kernel(const RotaryArgs a) {
  __shared__ __attribute__((aligned(16))) uint16_t row_s[kRows * kThreads / 16][kRowPitch];
  const uint32_t l = blockIdx.y, j = threadIdx.x & 15, n_rows = a.T * a.H, row0 = blockIdx.x * (kRows * kThreads / 16) + (threadIdx.x >> 4);
  const bool turns = 8 * j < 2 * a.pairs, works = turns || a.copy;
  double f[8];   // of this lane's channels, in turns
#pragma unroll
  for (uint32_t e = 0; e < 8; ++e) {
    const uint32_t c = 8 * j + e;
    f[e] = c < 2 * a.pairs ? a.freq[c < a.pairs ? c : c - a.pairs] * kTurn : 0.0;
  }
  uint4 v[kRows];
  int32_t pos[kRows];
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    const uint32_t row = row0 + k * (kThreads / 16), t = a.div_h.quot(row), h = row - t * a.H;
    if (row >= n_rows || !works) continue;
    if (turns) pos[k] = a.pos[static_cast<int64_t>(l) * a.p_sl + static_cast<int64_t>(t) * a.p_st + static_cast<int64_t>(h) * a.p_sh];
    v[k] = load_stream16(a.x + static_cast<int64_t>(l) * a.x_sl + static_cast<int64_t>(t) * a.x_st + static_cast<int64_t>(h) * a.x_sh + 8 * j);
  }
#pragma unroll
  for (int k = 0; k < kRows; ++k)
    if (turns && row0 + k * (kThreads / 16) < n_rows) *reinterpret_cast<uint4*>(&row_s[k * (kThreads / 16) + (threadIdx.x >> 4)][8 * j]) = v[k];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    const uint32_t row = row0 + k * (kThreads / 16), t = a.div_h.quot(row), h = row - t * a.H;
    if (row >= n_rows || !works) continue;
    if (turns) {
      const uint16_t* x = row_s[k * (kThreads / 16) + (threadIdx.x >> 4)];
      uint32_t* w = reinterpret_cast<uint32_t*>(&v[k]);
      float y[8];
      unpack_bf16x8(v[k], y);
#pragma unroll
      for (uint32_t e = 0; e < 8; ++e) {
        const uint32_t c = 8 * j + e;
        if (c >= 2 * a.pairs) continue;
        const float2 cs = turn_of(a, pos[k], f[e]);
        float p = y[e], q = __uint_as_float(static_cast<uint32_t>(x[c < a.pairs ? c + a.pairs : c - a.pairs]) << 16);
        if (c < a.pairs) {
          rotate(p, q, cs);
        } else {
          rotate(q, p, cs);
        }
        y[e] = p;
      }
#pragma unroll
      for (uint32_t i = 0; i < 4; ++i)
        if (8 * j + 2 * i < 2 * a.pairs) w[i] = pack_bf16x2(y[2 * i], y[2 * i + 1]);
    }
    store_stream16(a.out + static_cast<int64_t>(l) * a.o_sl + static_cast<int64_t>(t) * a.o_st + static_cast<int64_t>(h) * a.o_sh + 8 * j, v[k]);
  }
}

}  // namespace
}  // namespace kvp

extern "C" int32_t kvp_rotary(const kvp_view* x, const kvp_view* out, const int32_t* positions, int64_t pos_stride_l,
                              int64_t pos_stride_t, int64_t pos_stride_h, const double* freq, int32_t rotary_dim, int32_t layout,
                              int32_t inverse, float mscale, void* stream) {
  using namespace kvp;
  int32_t rc = check_view(x);
  if (rc == KVP_OK) rc = check_view(out);
  if (rc != KVP_OK) return rc;
  if (!positions || !freq) return KVP_ERR_NULL;
  if (layout != KVP_ROTARY_HALF && layout != KVP_ROTARY_INTERLEAVED) return KVP_ERR_UNSUPPORTED;
  if (rotary_dim < 2 || rotary_dim > kHeadDim || rotary_dim % 2) return KVP_ERR_UNSUPPORTED;
  if (out->L != x->L || out->T != x->T || out->H != x->H) return KVP_ERR_SHAPE;
  if (out->ptr == x->ptr && (out->stride_l != x->stride_l || out->stride_t != x->stride_t || out->stride_h != x->stride_h)) return KVP_ERR_SHAPE;
  if (x->L > 65535 || x->T >= (1ll << 31) || x->H >= (1ll << 31) || x->T * x->H >= (1ll << 31)) return KVP_ERR_SHAPE;
  if (pos_stride_l < 0 || pos_stride_t < 0 || pos_stride_h < 0) return KVP_ERR_SHAPE;
  if ((reinterpret_cast<uintptr_t>(positions) & 3u) || (reinterpret_cast<uintptr_t>(freq) & 7u)) return KVP_ERR_ALIGN;
  const bool any = layout == KVP_ROTARY_HALF && rotary_dim % 16, per_head = pos_stride_h != 0;
  const int64_t blocks = rotary_blocks(x->T, x->H, any, per_head);
  if (!fits_grid(blocks, kThreads)) return KVP_ERR_SHAPE;
  RotaryArgs a{};
  a.x = static_cast<const uint16_t*>(x->ptr);
  a.out = static_cast<uint16_t*>(const_cast<void*>(out->ptr));
  a.x_sl = x->stride_l; a.x_st = x->stride_t; a.x_sh = x->stride_h;
  a.o_sl = out->stride_l; a.o_st = out->stride_t; a.o_sh = out->stride_h;
  a.pos = positions;
  a.p_sl = pos_stride_l; a.p_st = pos_stride_t; a.p_sh = pos_stride_h;
  a.freq = freq;
  a.T = static_cast<uint32_t>(x->T);
  a.H = static_cast<uint32_t>(x->H);
  a.pairs = static_cast<uint32_t>(rotary_dim / 2);
  a.div_h = FastDiv(a.H);
  a.div_pairs = FastDiv(a.pairs);
  a.mscale = mscale;
  a.sign = inverse ? -1.0f : 1.0f;
  a.copy = x->ptr != out->ptr;
  const hipStream_t st = as_stream(stream);
  const dim3 grid(static_cast<unsigned>(blocks), static_cast<unsigned>(x->L));
  if (any) {
    rotary_any_kernel<<<grid, kThreads, 0, st>>>(a);
  } else if (per_head) {
    if (layout == KVP_ROTARY_HALF)
      rotary_rows_kernel<KVP_ROTARY_HALF><<<grid, kThreads, 0, st>>>(a);
    else
      rotary_rows_kernel<KVP_ROTARY_INTERLEAVED><<<grid, kThreads, 0, st>>>(a);
  } else {
    a.tokens_block = static_cast<uint32_t>(rotary_tokens_block(x->T, x->H));
    if (layout == KVP_ROTARY_HALF)
      rotary_kernel<KVP_ROTARY_HALF><<<grid, kThreads, 0, st>>>(a);
    else
      rotary_kernel<KVP_ROTARY_INTERLEAVED><<<grid, kThreads, 0, st>>>(a);
  }
  return launch_status();
}

extern "C" int32_t kvp_rotary_frequencies(double base, int32_t rotary_dim, int32_t scaling, double factor, double original, double low,
                                          double high, double* freq, float* mscale) {
  using namespace kvp;
  if (rotary_dim < 2 || rotary_dim > kHeadDim || rotary_dim % 2) return KVP_ERR_UNSUPPORTED;
  if (scaling < KVP_ROTARY_PLAIN || scaling > KVP_ROTARY_BANDED) return KVP_ERR_UNSUPPORTED;
  if (!(base > 1.0) || !isfinite(base)) return KVP_ERR_SHAPE;
  if (scaling != KVP_ROTARY_PLAIN && !(factor >= 1.0 && isfinite(factor))) return KVP_ERR_SHAPE;
  if (scaling == KVP_ROTARY_NTK && rotary_dim == 2) return KVP_ERR_SHAPE;
  if (scaling >= KVP_ROTARY_YARN && !(original > 0.0 && isfinite(original) && low > 0.0 && high > low && isfinite(high))) return KVP_ERR_SHAPE;
  if (mscale) *mscale = scaling == KVP_ROTARY_YARN ? static_cast<float>(0.1 * log(factor) + 1.0) : 1.0f;
  if (!freq) return KVP_OK;
  const double dim = rotary_dim, two_pi = 6.283185307179586;
  if (scaling == KVP_ROTARY_NTK) base *= pow(factor, dim / (dim - 2.0));
  const int32_t n = rotary_dim / 2;
  // pair index at which the original context holds r turns: f = base^(-2 i / dim) = 2 pi r / original
  auto index_of = [&](double r) { return dim * log(original / (two_pi * r)) / (2.0 * log(base)); };
  double from = 0.0, to = 1.0;
  if (scaling == KVP_ROTARY_YARN) {
    from = fmin(fmax(floor(index_of(high)), 0.0), dim - 1.0);
    to = fmin(fmax(ceil(index_of(low)), 0.0), dim - 1.0);
  }
  for (int32_t i = 0; i < n; ++i) {
    const double f = pow(base, -2.0 * i / dim);
    double keep = 1.0;   // share of the unscaled frequency
    if (scaling == KVP_ROTARY_LINEAR) {
      keep = 0.0;
    } else if (scaling == KVP_ROTARY_YARN) {
      keep = to > from ? 1.0 - fmin(fmax((i - from) / (to - from), 0.0), 1.0) : (i <= from ? 1.0 : 0.0);
    } else if (scaling == KVP_ROTARY_BANDED) {
      keep = fmin(fmax((original * f / two_pi - low) / (high - low), 0.0), 1.0);
    }
    freq[i] = scaling == KVP_ROTARY_PLAIN || scaling == KVP_ROTARY_NTK ? f : keep * f + (1.0 - keep) * f / factor;
  }
  return KVP_OK;
}
