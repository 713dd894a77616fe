// kvp_cache_append and kvp_cache_read: bf16 K/V rows into the 8-bit paged cache and back.
//
// Append: a block owns one page of one head, keys or values: it reads the page's new rows (kept in registers), reduces
// their largest magnitude, settles the page's scale, recodes what the page held where that scale grew, and stores the codes.
// Values are stored channel-major: a row's codes are turned in LDS, and whole runs of 16 slots of a channel go out as 16 bytes.
// Read: the same blocks the other way.
// Both move 2 + 1 bytes per element and are bound by HBM; a decode step (one row per sequence) is bound by latency.

#include "cache_common.h"

namespace kvp {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxItems = 8;      // 16-byte pieces of a page's rows per thread: bs / 16

struct AppendArgs {
  CacheArgs c;
  const uint16_t* src[2];         // keys, values
  int64_t sb[2], sw[2], sh[2];    // element strides
  const int32_t* counts;
  uint32_t W, pages;              // pages a call may touch per sequence
  FastDiv div_h, div_pages;
};

struct ReadArgs {
  CacheArgs c;
  uint16_t* dst[2];               // keys, values; null: not asked for
  int64_t sb[2], sr[2], sh[2];
  const int32_t* first;
  uint32_t R, pages;
  FastDiv div_h, div_pages;
};

// 16 bytes of which bytes [lo, hi) are ones
__device__ __forceinline__ uint4 byte_mask(int lo, int hi) {
  uint32_t m[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int a = min(max(lo - 4 * i, 0), 4), b = min(max(hi - 4 * i, 0), 4);
    m[i] = static_cast<uint32_t>(((1ull << (8 * b)) - 1) & ~((1ull << (8 * a)) - 1));
  }
  return make_uint4(m[0], m[1], m[2], m[3]);
}
__device__ __forceinline__ uint4 blend(uint4 m, uint4 a, uint4 b) {   // a where m is set
  return make_uint4((a.x & m.x) | (b.x & ~m.x), (a.y & m.y) | (b.y & ~m.y), (a.z & m.z) | (b.z & ~m.z), (a.w & m.w) | (b.w & ~m.w));
}

template <int FMT>
__device__ __forceinline__ uint32_t recode4(uint32_t w, float old, const PageQuantizer& q) {
  float x[4];
  decode4<FMT>(w, x);
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] *= old;
  return q.codes4<FMT>(x);
}

template <int FMT>
__global__ __launch_bounds__(kThreads) void cache_append_kernel(const AppendArgs a) {
  __shared__ __attribute__((aligned(16))) uint8_t turn_s[kHeadDim * (128 + 16)];   // values: [channel][slot], pitch bs + 16
  __shared__ float max_s[4];
  const CacheArgs& c = a.c;
  // block -> (sequence, plane, page of the call, head)
  const uint32_t rest = a.div_h.quot(blockIdx.x), h = blockIdx.x - rest * c.H;
  const uint32_t bp = a.div_pages.quot(rest), p = rest - bp * a.pages, b = bp >> 1, plane = bp & 1;
  const uint32_t bs = 1u << c.bs_log2, len = cache_len(c, b);
  uint32_t count = a.W;
  if (a.counts) count = static_cast<uint32_t>(min(max(a.counts[b], 0), static_cast<int32_t>(a.W)));
  const uint32_t end = min(len + count, c.max_blocks << c.bs_log2);
  const uint32_t page = (len >> c.bs_log2) + p, t0 = page << c.bs_log2;
  if (max(t0, len) >= end) return;
  const int s0 = static_cast<int>(max(len, t0) - t0), s1 = static_cast<int>(min(end - t0, bs));   // new slots
  const int64_t cell = static_cast<int64_t>(cache_page(c, b, page)) * c.H + h;
  const uint16_t* src = a.src[plane] + static_cast<int64_t>(b) * a.sb[plane] + static_cast<int64_t>(h) * a.sh[plane];
  const int64_t sw = a.sw[plane];
  const int64_t w0 = static_cast<int64_t>(t0) - len;                        // row of slot 0
  const int items = static_cast<int>(bs >> 4);

  uint4 raw[kMaxItems];
  float amax = 0.0f;
#pragma unroll
  for (int i = 0; i < kMaxItems; ++i) {
    if (i >= items) break;
    const int slot = static_cast<int>((threadIdx.x + i * kThreads) >> 4);
    raw[i] = make_uint4(0, 0, 0, 0);
    if (slot >= s0 && slot < s1) raw[i] = load_stream16(src + (w0 + slot) * sw + (threadIdx.x & 15) * 8);
  }
  float* scale_at = (plane ? c.v_scales : c.k_scales) + cell;
  const float old = s0 > 0 ? *scale_at : 0.0f;
#pragma unroll
  for (int i = 0; i < kMaxItems; ++i) {
    if (i >= items) break;
    float x[8];
    unpack_bf16x8(raw[i], x);
    amax = fmaxf(amax, abs_max8(x));
  }
  amax = block_max256(amax, max_s);
  const float fresh = amax / kCodeMax<FMT>, scale = s0 > 0 ? fmaxf(old, fresh) : fresh;
  const bool recode = s0 > 0 && scale != old;
  const PageQuantizer q(scale);
  if (threadIdx.x == 0 && (s0 == 0 || recode)) *scale_at = scale;

  uint8_t* codes = (plane ? c.v_codes : c.k_codes) + (cell << (c.bs_log2 + 7));
  const int pitch = static_cast<int>(bs) + 16;
#pragma unroll
  for (int i = 0; i < kMaxItems; ++i) {
    if (i >= items) break;
    const int slot = static_cast<int>((threadIdx.x + i * kThreads) >> 4), ch = static_cast<int>(threadIdx.x & 15) * 8;
    const bool is_new = slot >= s0 && slot < s1;
    uint2 w;
    if (is_new) {
      float x[8];
      unpack_bf16x8(raw[i], x);
      w = make_uint2(q.codes4<FMT>(x), q.codes4<FMT>(x + 4));
    }
    if (plane == 0) {
      uint2* at = reinterpret_cast<uint2*>(codes + slot * kHeadDim + ch);
      if (is_new) {
        *at = w;
      } else if (recode && slot < s0) {
        const uint2 v = *at;
        *at = make_uint2(recode4<FMT>(v.x, old, q), recode4<FMT>(v.y, old, q));
      }
    } else if (is_new) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        turn_s[(ch + k) * pitch + slot] = static_cast<uint8_t>(w.x >> (8 * k));
        turn_s[(ch + 4 + k) * pitch + slot] = static_cast<uint8_t>(w.y >> (8 * k));
      }
    }
  }
  if (plane == 0) return;
  __syncthreads();
  // values: every run of 16 slots of a channel that changes
  for (int i = static_cast<int>(threadIdx.x); i < kHeadDim * items; i += kThreads) {
    const int ch = i >> (c.bs_log2 - 4), run = i & (items - 1), lo = s0 - run * 16, hi = s1 - run * 16;   // new bytes of the run
    const bool changes = hi > 0 && lo < 16;
    if (!changes && !(recode && lo > 0)) continue;
    uint4* at = reinterpret_cast<uint4*>(codes + (ch << c.bs_log2) + run * 16);
    const uint4 fresh16 = *reinterpret_cast<const uint4*>(turn_s + ch * pitch + run * 16);
    if (lo <= 0 && hi >= 16) {
      *at = fresh16;
      continue;
    }
    uint4 v = *at;
    if (recode && lo > 0) {
      const uint4 again = make_uint4(recode4<FMT>(v.x, old, q), recode4<FMT>(v.y, old, q), recode4<FMT>(v.z, old, q), recode4<FMT>(v.w, old, q));
      v = blend(byte_mask(0, lo), again, v);
    }
    *at = changes ? blend(byte_mask(lo, hi), fresh16, v) : v;
  }
}

template <int FMT>
__global__ __launch_bounds__(kThreads) void cache_read_kernel(const ReadArgs a) {
  __shared__ __attribute__((aligned(16))) uint8_t turn_s[kHeadDim * (128 + 16)];
  const CacheArgs& c = a.c;
  const uint32_t rest = a.div_h.quot(blockIdx.x), h = blockIdx.x - rest * c.H;
  const uint32_t bp = a.div_pages.quot(rest), p = rest - bp * a.pages, b = bp >> 1, plane = bp & 1;
  if (!a.dst[plane]) return;
  const uint32_t bs = 1u << c.bs_log2;
  const uint32_t first = a.first ? static_cast<uint32_t>(max(a.first[b], 0)) : 0u;
  const uint32_t end = min(cache_len(c, b), first + a.R), page = (first >> c.bs_log2) + p;
  if (page >= c.max_blocks) return;
  const uint32_t t0 = page << c.bs_log2;
  if (max(t0, first) >= end) return;
  const int s0 = static_cast<int>(max(first, t0) - t0), s1 = static_cast<int>(min(end - t0, bs));
  const int64_t cell = static_cast<int64_t>(cache_page(c, b, page)) * c.H + h;
  const uint8_t* codes = (plane ? c.v_codes : c.k_codes) + (cell << (c.bs_log2 + 7));
  const float scale = (plane ? c.v_scales : c.k_scales)[cell];
  uint16_t* dst = a.dst[plane] + static_cast<int64_t>(b) * a.sb[plane] + static_cast<int64_t>(h) * a.sh[plane];
  const int64_t r0 = static_cast<int64_t>(t0) - first;                       // out row of slot 0
  const int items = static_cast<int>(bs >> 4), pitch = static_cast<int>(bs) + 16;
  if (plane) {
    for (int i = static_cast<int>(threadIdx.x); i < kHeadDim * items; i += kThreads) {
      const int ch = i >> (c.bs_log2 - 4), run = i & (items - 1);
      *reinterpret_cast<uint4*>(turn_s + ch * pitch + run * 16) = load_stream16(codes + (ch << c.bs_log2) + run * 16);
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < kMaxItems; ++i) {
    if (i >= items) break;
    const int slot = static_cast<int>((threadIdx.x + i * kThreads) >> 4), ch = static_cast<int>(threadIdx.x & 15) * 8;
    if (slot < s0 || slot >= s1) continue;
    uint32_t w[2];
    if (plane) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint8_t* at = turn_s + (ch + 4 * k) * pitch + slot;
        w[k] = at[0] | (at[pitch] << 8) | (at[2 * pitch] << 16) | (static_cast<uint32_t>(at[3 * pitch]) << 24);
      }
    } else {
      const uint2 v = load_stream8(codes + slot * kHeadDim + ch);
      w[0] = v.x;
      w[1] = v.y;
    }
    uint32_t o[4];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      float x[4];
      decode4<FMT>(w[k], x);
      o[2 * k] = pack_bf16x2(x[0] * scale, x[1] * scale);
      o[2 * k + 1] = pack_bf16x2(x[2] * scale, x[3] * scale);
    }
    store_stream16(dst + (r0 + slot) * a.sr[plane] + ch, make_uint4(o[0], o[1], o[2], o[3]));
  }
}

}  // namespace
}  // namespace kvp

extern "C" int32_t kvp_cache_append(const kvp_cache* cache, const kvp_view* k, const kvp_view* v, const int32_t* counts, void* stream) {
  using namespace kvp;
  int32_t rc = check_cache(cache, true);
  if (rc == KVP_OK) rc = check_view(k);
  if (rc == KVP_OK) rc = check_view(v);
  if (rc != KVP_OK) return rc;
  if (k->L != cache->B || v->L != cache->B || k->H != cache->H || v->H != cache->H || k->T != v->T || k->T >= (1ll << 31)) return KVP_ERR_SHAPE;
  if (reinterpret_cast<uintptr_t>(counts) & 3u) return KVP_ERR_ALIGN;
  AppendArgs a{};
  a.c = cache_args(cache);
  const kvp_view* views[2] = {k, v};
  for (int i = 0; i < 2; ++i) {
    a.src[i] = static_cast<const uint16_t*>(views[i]->ptr);
    a.sb[i] = views[i]->stride_l; a.sw[i] = views[i]->stride_t; a.sh[i] = views[i]->stride_h;
  }
  a.counts = counts;
  a.W = static_cast<uint32_t>(k->T);
  // W rows behind any number of older ones touch at most this many pages; never more than there are
  const int64_t pages = std::min<int64_t>(cache->max_blocks, ceil_div(k->T + cache->bs - 1, cache->bs));
  const int64_t blocks = cache->B * cache->H * 2 * pages;
  if (blocks >= (1ll << 31)) return KVP_ERR_SHAPE;
  a.pages = static_cast<uint32_t>(pages);
  a.div_h = FastDiv(a.c.H);
  a.div_pages = FastDiv(a.pages);
  const dim3 grid(static_cast<unsigned>(blocks));
  if (cache->format == KVP_CACHE_INT8)
    cache_append_kernel<KVP_CACHE_INT8><<<grid, kThreads, 0, as_stream(stream)>>>(a);
  else
    cache_append_kernel<KVP_CACHE_E4M3><<<grid, kThreads, 0, as_stream(stream)>>>(a);
  return launch_status();
}

extern "C" int32_t kvp_cache_read(const kvp_cache* cache, const int32_t* first, const kvp_view* k_out, const kvp_view* v_out, void* stream) {
  using namespace kvp;
  int32_t rc = check_cache(cache, true);
  if (rc != KVP_OK) return rc;
  if (!k_out && !v_out) return KVP_ERR_NULL;
  ReadArgs a{};
  const kvp_view* views[2] = {k_out, v_out};
  int64_t R = -1;
  for (int i = 0; i < 2; ++i) {
    if (!views[i]) continue;
    rc = check_view(views[i]);
    if (rc != KVP_OK) return rc;
    if (views[i]->L != cache->B || views[i]->H != cache->H || (R >= 0 && views[i]->T != R) || views[i]->T >= (1ll << 31)) return KVP_ERR_SHAPE;
    R = views[i]->T;
    a.dst[i] = static_cast<uint16_t*>(const_cast<void*>(views[i]->ptr));
    a.sb[i] = views[i]->stride_l; a.sr[i] = views[i]->stride_t; a.sh[i] = views[i]->stride_h;
  }
  if (reinterpret_cast<uintptr_t>(first) & 3u) return KVP_ERR_ALIGN;
  a.c = cache_args(cache);
  a.first = first;
  a.R = static_cast<uint32_t>(R);
  const int64_t pages = std::min<int64_t>(cache->max_blocks, ceil_div(R + cache->bs - 1, cache->bs));
  const int64_t blocks = cache->B * cache->H * 2 * pages;
  if (blocks >= (1ll << 31)) return KVP_ERR_SHAPE;
  a.pages = static_cast<uint32_t>(pages);
  a.div_h = FastDiv(a.c.H);
  a.div_pages = FastDiv(a.pages);
  const dim3 grid(static_cast<unsigned>(blocks));
  if (cache->format == KVP_CACHE_INT8)
    cache_read_kernel<KVP_CACHE_INT8><<<grid, kThreads, 0, as_stream(stream)>>>(a);
  else
    cache_read_kernel<KVP_CACHE_E4M3><<<grid, kThreads, 0, as_stream(stream)>>>(a);
  return launch_status();
}
