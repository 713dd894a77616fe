// The 8-bit paged cache (kvp_cache): what its kernels share.
#pragma once

#include "kvp_internal.h"
#include "quant_device.h"

namespace kvp {

typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));

// A cache as the kernels take it.  Page sizes are powers of two (16 .. 128).
struct CacheArgs {
  uint8_t* k_codes;
  uint8_t* v_codes;
  float* k_scales;
  float* v_scales;
  const int32_t* table;
  const int32_t* lens;
  int64_t table_stride;
  uint32_t B, H, bs_log2, num_blocks, max_blocks;
};

// lens and table entries are clamped where they are read: nothing in them can take an access out of the pool
__device__ __forceinline__ uint32_t cache_len(const CacheArgs& c, uint32_t b) {
  const int32_t n = c.lens[b];
  return n < 0 ? 0u : min(static_cast<uint32_t>(n), c.max_blocks << c.bs_log2);
}
__device__ __forceinline__ uint32_t clamp_page(const CacheArgs& c, int32_t entry) {
  return entry < 0 ? 0u : min(static_cast<uint32_t>(entry), c.num_blocks - 1);
}
// page index below max_blocks -> pool page
__device__ __forceinline__ uint32_t cache_page(const CacheArgs& c, uint32_t b, uint32_t page) {
  return clamp_page(c, c.table[static_cast<int64_t>(b) * c.table_stride + page]);
}

// Validation of the fields that every call uses.
inline int32_t check_cache(const kvp_cache* c, bool need_lens) {
  if (!c || !c->k_codes || !c->v_codes || !c->k_scales || !c->v_scales || !c->block_table || (need_lens && !c->lens)) return KVP_ERR_NULL;
  if (c->D != kHeadDim) return KVP_ERR_UNSUPPORTED;
  if (c->bs != 16 && c->bs != 32 && c->bs != 64 && c->bs != 128) return KVP_ERR_UNSUPPORTED;
  if (c->format != KVP_CACHE_INT8 && c->format != KVP_CACHE_E4M3) return KVP_ERR_UNSUPPORTED;
  constexpr int64_t kMost = 1ll << 31;
  if (c->B <= 0 || c->H <= 0 || c->num_blocks <= 0 || c->max_blocks <= 0 || c->table_stride < c->max_blocks) return KVP_ERR_SHAPE;
  if (c->B >= kMost || c->H >= kMost || c->num_blocks >= kMost || c->max_blocks >= kMost) return KVP_ERR_SHAPE;
  if (c->B * c->H >= kMost || c->num_blocks * c->H >= kMost || c->max_blocks * c->bs >= kMost || c->B * c->H >= ceil_div(kMost, c->max_blocks))
    return KVP_ERR_SHAPE;
  if (!aligned16(c->k_codes) || !aligned16(c->v_codes)) return KVP_ERR_ALIGN;
  if ((reinterpret_cast<uintptr_t>(c->k_scales) | reinterpret_cast<uintptr_t>(c->v_scales) | reinterpret_cast<uintptr_t>(c->block_table) |
       reinterpret_cast<uintptr_t>(c->lens)) & 3u)
    return KVP_ERR_ALIGN;
  return KVP_OK;
}

inline CacheArgs cache_args(const kvp_cache* c) {
  CacheArgs a{};
  a.k_codes = c->k_codes; a.v_codes = c->v_codes;
  a.k_scales = c->k_scales; a.v_scales = c->v_scales;
  a.table = c->block_table; a.lens = c->lens;
  a.table_stride = c->table_stride;
  a.B = static_cast<uint32_t>(c->B);
  a.H = static_cast<uint32_t>(c->H);
  a.num_blocks = static_cast<uint32_t>(c->num_blocks);
  a.max_blocks = static_cast<uint32_t>(c->max_blocks);
  a.bs_log2 = c->bs == 16 ? 4 : c->bs == 32 ? 5 : c->bs == 64 ? 6 : 7;
  return a;
}

// ---- codes <-> values ----

template <int FMT> constexpr float kCodeMax = FMT == KVP_CACHE_INT8 ? 127.0f : 448.0f;

// four codes of a word -> floats (exact)
template <int FMT>
__device__ __forceinline__ void decode4(uint32_t w, float x[4]) {
  if constexpr (FMT == KVP_CACHE_INT8) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = static_cast<float>(static_cast<int>(__builtin_amdgcn_sbfe(static_cast<int>(w), 8 * i, 8)));
  } else {
    typedef float f2 __attribute__((ext_vector_type(2)));
    const f2 a = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), false), b = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), true);
    x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y;
  }
}

// Eight codes -> halves (exact: an int8 code has 7 bits and a sign, an e4m3 value 4 significant bits of at least 2^-9).
// int8: with the sign bit flipped a byte u is code + 128, and the half with bytes (u, 0x64) is 1024 + u.
template <int FMT>
__device__ __forceinline__ half8_t decode8_half(uint32_t w0, uint32_t w1) {
  union { half2_t h[4]; half8_t v; uint32_t u[4]; } r;
  if constexpr (FMT == KVP_CACHE_INT8) {
    const half2_t off = {static_cast<_Float16>(-1152.0f), static_cast<_Float16>(-1152.0f)};
    const uint32_t x0 = w0 ^ 0x80808080u, x1 = w1 ^ 0x80808080u;
    r.u[0] = __builtin_amdgcn_perm(0x64646464u, x0, 0x04010400u);
    r.u[1] = __builtin_amdgcn_perm(0x64646464u, x0, 0x04030402u);
    r.u[2] = __builtin_amdgcn_perm(0x64646464u, x1, 0x04010400u);
    r.u[3] = __builtin_amdgcn_perm(0x64646464u, x1, 0x04030402u);
#pragma unroll
    for (int i = 0; i < 4; ++i) r.h[i] = r.h[i] + off;
  } else {
    r.h[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(static_cast<int>(w0), 1.0f, false);
    r.h[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(static_cast<int>(w0), 1.0f, true);
    r.h[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(static_cast<int>(w1), 1.0f, false);
    r.h[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(static_cast<int>(w1), 1.0f, true);
  }
  return r.v;
}

// Codes of values on a given scale: rnd(fl32(x / scale)).  The quotient without a division per element, as in quant_device.h: the correctly
// rounded reciprocal, a product and one remainder step.  Scales outside [2^-60, 2^60] divide; a subnormal one may be off by up to a third (a
// largest value of 1.49 qmax units of 2^-149 has a scale of one), and quotients beyond the largest code become that code.
struct PageQuantizer {
  float scale, inv;
  bool unsafe;
  __device__ __forceinline__ explicit PageQuantizer(float s) : scale(s) {
    unsafe = !(s >= 0x1p-60f && s <= 0x1p60f) && s != 0.0f;
    inv = s == 0.0f ? 0.0f : reciprocal_in_range(s);
  }
  __device__ __forceinline__ float quotient(float x) const {
    if (unsafe) return x / scale;   // the scale is uniform over the block: no divergence
    const float q0 = x * inv;
    return fmaf(fmaf(-scale, q0, x), inv, q0);
  }
  // four values -> a word of codes
  template <int FMT>
  __device__ __forceinline__ uint32_t codes4(const float x[4]) const {
    float q[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = quotient(x[i]);
    if (unsafe) {
#pragma unroll
      for (int i = 0; i < 4; ++i) q[i] = fminf(fmaxf(q[i], -kCodeMax<FMT>), kCodeMax<FMT>);
    }
    if constexpr (FMT == KVP_CACHE_INT8) {
#pragma unroll
      for (int i = 0; i < 4; ++i) q[i] = rintf(q[i]);
      return pack_int8x4(q);
    } else {
      int w = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
      return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], w, true));
    }
  }
};

// four codes of an old scale on a new one
template <int FMT>
__device__ __forceinline__ uint32_t recode4(uint32_t w, float old, const PageQuantizer& q) {
  float x[4];
  decode4<FMT>(w, x);
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] *= old;
  return q.codes4<FMT>(x);
}

// largest value over the wave of a non-negative number per lane
__device__ __forceinline__ float wave_max(float v) {
  uint32_t u = __float_as_uint(group_max(v, 16));
  u = max(u, static_cast<uint32_t>(__shfl_xor(static_cast<int>(u), 16)));
  u = max(u, static_cast<uint32_t>(__shfl_xor(static_cast<int>(u), 32)));
  return __uint_as_float(u);
}
// ... over a 256-thread block; every thread gets it.  sh: 4 floats
__device__ __forceinline__ float block_max256(float v, float* sh) {
  v = wave_max(v);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  return fmaxf(fmaxf(sh[0], sh[1]), fmaxf(sh[2], sh[3]));
}

}  // namespace kvp
