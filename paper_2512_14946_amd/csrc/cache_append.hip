// kvp_cache_append and kvp_cache_read: bf16 K/V rows into the 8-bit paged cache and back.
//
// Append: a block owns one page of one head, keys and values: it reads the page's new rows (kept in registers), reduces
// their largest magnitudes, settles the page's scales, recodes what the page held where a scale grew, and stores the codes.
// Values are stored channel-major: a row's codes are turned in LDS, and whole runs of 16 slots of a channel go out as 16 bytes.
// Read: the same blocks the other way.
// Both move 2 + 1 bytes per element and are bound by HBM; a decode step (one row per sequence) is bound by latency.
// 8 sequences x 8 heads, 4096 tokens at most, into 64-token pages and back: 57 us for both, 4.4 TB/s; 64 sequences x 8 heads, one token each: 5 us a call.
// Both planes in a block: 59 us against 72 with a block per plane; read by words of four slots: 57 (byte by byte LDS conflicts took half the read).

#include "cache_common.h"

namespace kvp {
namespace {

constexpr int kThreads = 256;

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

// What a page of a plane becomes: scale before and after, and whether its older codes are coded again.
struct PageScale {
  float old, scale;
  bool recode;
};

// Slot of a thread's item: consecutive ones, so that the codes of up to four slots of a channel leave as a word.
template <int ITEMS>
__device__ __forceinline__ int slot_of(int i) { return static_cast<int>(threadIdx.x >> 4) * ITEMS + i; }

// Bytes of four words turned: out[k] = bytes k of w[0 .. 3]
__device__ __forceinline__ void turn4(const uint32_t w[4], uint32_t out[4]) {
  const uint32_t a = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u), b = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u);
  const uint32_t c = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u), d = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);
  out[0] = __builtin_amdgcn_perm(b, a, 0x05040100u);
  out[1] = __builtin_amdgcn_perm(b, a, 0x07060302u);
  out[2] = __builtin_amdgcn_perm(d, c, 0x05040100u);
  out[3] = __builtin_amdgcn_perm(d, c, 0x07060302u);
}

// Keys of a page: new rows' codes, older ones again where the scale grew.
template <int FMT, int ITEMS>
__device__ __forceinline__ void store_keys(const uint4 (&raw)[ITEMS], const PageScale& ps, uint8_t* codes, int s0, int s1) {
  const PageQuantizer q(ps.scale);
  const int ch = static_cast<int>(threadIdx.x & 15) * 8;
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const int slot = slot_of<ITEMS>(i);
    uint2* at = reinterpret_cast<uint2*>(codes + slot * kHeadDim + ch);
    if (slot >= s0 && slot < s1) {
      float x[8];
      unpack_bf16x8(raw[i], x);
      *at = make_uint2(q.codes4<FMT>(x), q.codes4<FMT>(x + 4));
    } else if (ps.recode && slot < s0) {
      const uint2 v = *at;
      *at = make_uint2(recode4<FMT>(v.x, ps.old, q), recode4<FMT>(v.y, ps.old, q));
    }
  }
}

// Values of a page, turned in LDS: [channel][slot], 4 bytes more than a page's slots apart.
template <int FMT, int ITEMS>
__device__ __forceinline__ void store_values(const uint4 (&raw)[ITEMS], const PageScale& ps, uint8_t* codes, int s0, int s1, uint8_t* turn) {
  constexpr int bs = 16 * ITEMS, pitch = bs + 4;
  const PageQuantizer q(ps.scale);
  const int ch = static_cast<int>(threadIdx.x & 15) * 8;
  uint32_t w[ITEMS][2];
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {   // rows that are not new are zeros, and their codes are not used
    float x[8];
    unpack_bf16x8(raw[i], x);
    w[i][0] = q.codes4<FMT>(x);
    w[i][1] = q.codes4<FMT>(x + 4);
  }
  uint8_t* to = turn + ch * pitch + slot_of<ITEMS>(0);
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    if constexpr (ITEMS == 1)
      to[k * pitch] = static_cast<uint8_t>(w[0][k >> 2] >> (8 * (k & 3)));
    else if constexpr (ITEMS == 2)
      *reinterpret_cast<uint16_t*>(to + k * pitch) =
          static_cast<uint16_t>(((w[0][k >> 2] >> (8 * (k & 3))) & 0xffu) | (((w[1][k >> 2] >> (8 * (k & 3))) & 0xffu) << 8));
  }
  if constexpr (ITEMS >= 4) {
#pragma unroll
    for (int g = 0; g < ITEMS; g += 4)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint32_t in[4] = {w[g][j], w[g + 1][j], w[g + 2][j], w[g + 3][j]};
        uint32_t out[4];
        turn4(in, out);
#pragma unroll
        for (int k = 0; k < 4; ++k) *reinterpret_cast<uint32_t*>(to + (4 * j + k) * pitch + g) = out[k];
      }
  }
  __syncthreads();
  // every run of 16 slots of a channel that changes
#pragma unroll
  for (int i = 0; i < (ITEMS + 1) / 2; ++i) {
    const int n = static_cast<int>(threadIdx.x) + i * kThreads, c = n / ITEMS, run = n % ITEMS, lo = s0 - run * 16, hi = s1 - run * 16;   // new bytes of the run
    if (n >= kHeadDim * ITEMS) break;
    const bool changes = hi > 0 && lo < 16;
    if (!changes && !(ps.recode && lo > 0)) continue;
    uint4* at = reinterpret_cast<uint4*>(codes + c * bs + run * 16);
    const uint32_t* from = reinterpret_cast<const uint32_t*>(turn + c * pitch + run * 16);
    const uint4 fresh16 = make_uint4(from[0], from[1], from[2], from[3]);
    if (lo <= 0 && hi >= 16) {
      *at = fresh16;
      continue;
    }
    uint4 v = *at;
    if (ps.recode && lo > 0) {
      const uint4 again = make_uint4(recode4<FMT>(v.x, ps.old, q), recode4<FMT>(v.y, ps.old, q), recode4<FMT>(v.z, ps.old, q), recode4<FMT>(v.w, ps.old, q));
      v = blend(byte_mask(0, lo), again, v);
    }
    *at = changes ? blend(byte_mask(lo, hi), fresh16, v) : v;
  }
}

// ITEMS: 16-byte pieces of a page's rows per thread and plane, bs / 16
template <int FMT, int ITEMS>
__global__ __launch_bounds__(kThreads) void cache_append_kernel(const AppendArgs a) {
  __shared__ __attribute__((aligned(16))) uint8_t turn_s[kHeadDim * (16 * ITEMS + 4)];
  __shared__ float max_s[2][4];
  const CacheArgs& c = a.c;
  // block -> (sequence, page of the call, head)
  const uint32_t bp = a.div_h.quot(blockIdx.x), h = blockIdx.x - bp * c.H, b = a.div_pages.quot(bp), p = bp - b * a.pages;
  constexpr uint32_t bs = 16 * ITEMS;
  const uint32_t len = cache_len(c, b);
  uint32_t count = a.W;
  if (a.counts) count = static_cast<uint32_t>(min(max(a.counts[b], 0), static_cast<int32_t>(a.W)));
  const uint32_t end = min(len + count, c.max_blocks << c.bs_log2);
  const uint32_t page = (len >> c.bs_log2) + p, t0 = page << c.bs_log2;
  if (max(t0, len) >= end) return;
  const int s0 = static_cast<int>(max(len, t0) - t0), s1 = static_cast<int>(min(end - t0, bs));   // new slots
  const int64_t cell = static_cast<int64_t>(cache_page(c, b, page)) * c.H + h;
  const int64_t w0 = static_cast<int64_t>(t0) - len;                        // row of slot 0

  uint4 raw[2][ITEMS];
#pragma unroll
  for (int plane = 0; plane < 2; ++plane) {
    const uint16_t* src = a.src[plane] + static_cast<int64_t>(b) * a.sb[plane] + static_cast<int64_t>(h) * a.sh[plane] + (threadIdx.x & 15) * 8;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int slot = slot_of<ITEMS>(i);
      raw[plane][i] = make_uint4(0, 0, 0, 0);
      if (slot >= s0 && slot < s1) raw[plane][i] = load_stream16(src + (w0 + slot) * a.sw[plane]);
    }
  }
  PageScale ps[2];
  ps[0].old = s0 > 0 ? c.k_scales[cell] : 0.0f;
  ps[1].old = s0 > 0 ? c.v_scales[cell] : 0.0f;
  float amax[2];
#pragma unroll
  for (int plane = 0; plane < 2; ++plane) {
    amax[plane] = 0.0f;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      float x[8];
      unpack_bf16x8(raw[plane][i], x);
      amax[plane] = fmaxf(amax[plane], abs_max8(x));
    }
    amax[plane] = wave_max(amax[plane]);
    if ((threadIdx.x & 63) == 0) max_s[plane][threadIdx.x >> 6] = amax[plane];
  }
  __syncthreads();
#pragma unroll
  for (int plane = 0; plane < 2; ++plane) {
    const float fresh = fmaxf(fmaxf(max_s[plane][0], max_s[plane][1]), fmaxf(max_s[plane][2], max_s[plane][3])) / kCodeMax<FMT>;
    ps[plane].scale = s0 > 0 ? fmaxf(ps[plane].old, fresh) : fresh;
    ps[plane].recode = s0 > 0 && ps[plane].scale != ps[plane].old;
    if (threadIdx.x == 0 && (s0 == 0 || ps[plane].recode)) (plane ? c.v_scales : c.k_scales)[cell] = ps[plane].scale;
  }
  store_keys<FMT>(raw[0], ps[0], c.k_codes + (cell << (c.bs_log2 + 7)), s0, s1);
  store_values<FMT>(raw[1], ps[1], c.v_codes + (cell << (c.bs_log2 + 7)), s0, s1, turn_s);
}

// Eight codes on a scale as bf16 (one product and one rounding each)
template <int FMT>
__device__ __forceinline__ uint4 restore8(uint32_t w0, uint32_t w1, float scale) {
  float x[8];
  decode4<FMT>(w0, x);
  decode4<FMT>(w1, x + 4);
  return make_uint4(pack_bf16x2(x[0] * scale, x[1] * scale), pack_bf16x2(x[2] * scale, x[3] * scale), pack_bf16x2(x[4] * scale, x[5] * scale),
                    pack_bf16x2(x[6] * scale, x[7] * scale));
}

template <int FMT, int ITEMS>
__global__ __launch_bounds__(kThreads) void cache_read_kernel(const ReadArgs a) {
  __shared__ __attribute__((aligned(16))) uint8_t turn_s[kHeadDim * (16 * ITEMS + 4)];   // values: [channel][slot]
  const CacheArgs& c = a.c;
  const uint32_t bp = a.div_h.quot(blockIdx.x), h = blockIdx.x - bp * c.H, b = a.div_pages.quot(bp), p = bp - b * a.pages;
  constexpr uint32_t bs = 16 * ITEMS;
  constexpr int pitch = 16 * ITEMS + 4;
  const uint32_t first = a.first ? static_cast<uint32_t>(max(a.first[b], 0)) : 0u;
  const uint32_t end = min(cache_len(c, b), first + a.R), page = (first >> c.bs_log2) + p;
  if (page >= c.max_blocks) return;
  const uint32_t t0 = page << c.bs_log2;
  if (max(t0, first) >= end) return;
  const int s0 = static_cast<int>(max(first, t0) - t0), s1 = static_cast<int>(min(end - t0, bs));
  const int64_t cell = static_cast<int64_t>(cache_page(c, b, page)) * c.H + h;
  const int64_t r0 = static_cast<int64_t>(t0) - first;                       // out row of slot 0
  const uint8_t* k_codes = c.k_codes + (cell << (c.bs_log2 + 7));
  const uint8_t* v_codes = c.v_codes + (cell << (c.bs_log2 + 7));
  uint2 k[ITEMS];
  uint4 v[(ITEMS + 1) / 2];
  if (a.dst[1]) {
#pragma unroll
    for (int i = 0; i < (ITEMS + 1) / 2; ++i)
      if (threadIdx.x + i * kThreads < kHeadDim * ITEMS) v[i] = load_stream16(v_codes + (threadIdx.x + i * kThreads) * 16);   // the page as it lies
  }
  if (a.dst[0]) {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) k[i] = load_stream8(k_codes + (threadIdx.x + i * kThreads) * 8);
  }
  const float k_scale = c.k_scales[cell], v_scale = c.v_scales[cell];
  if (a.dst[1]) {
#pragma unroll
    for (int i = 0; i < (ITEMS + 1) / 2; ++i) {
      const int n = static_cast<int>(threadIdx.x + i * kThreads), ch = n / ITEMS, run = n % ITEMS;
      uint32_t* to = reinterpret_cast<uint32_t*>(turn_s + ch * pitch + run * 16);
      if (n < kHeadDim * ITEMS) to[0] = v[i].x, to[1] = v[i].y, to[2] = v[i].z, to[3] = v[i].w;
    }
  }
  const int ch = static_cast<int>(threadIdx.x & 15) * 8;
  if (a.dst[0]) {
    uint16_t* dst = a.dst[0] + static_cast<int64_t>(b) * a.sb[0] + static_cast<int64_t>(h) * a.sh[0] + ch;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int slot = static_cast<int>((threadIdx.x + i * kThreads) >> 4);
      if (slot >= s0 && slot < s1) store_stream16(dst + (r0 + slot) * a.sr[0], restore8<FMT>(k[i].x, k[i].y, k_scale));
    }
  }
  if (!a.dst[1]) return;
  __syncthreads();
  // values: four slots of eight channels as words, turned in registers
  uint16_t* dst = a.dst[1] + static_cast<int64_t>(b) * a.sb[1] + static_cast<int64_t>(h) * a.sh[1] + ch;
#pragma unroll
  for (int i = 0; i < (ITEMS + 3) / 4; ++i) {
    const int slot = static_cast<int>((threadIdx.x + i * kThreads) >> 4) * 4;
    if (slot >= s1 || slot + 4 <= s0) continue;   // s1: at most the page's slots
    uint32_t w[8], lo[4], hi[4];
#pragma unroll
    for (int c = 0; c < 8; ++c) w[c] = *reinterpret_cast<const uint32_t*>(turn_s + (ch + c) * pitch + slot);
    turn4(w, lo);
    turn4(w + 4, hi);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (slot + e >= s0 && slot + e < s1) store_stream16(dst + (r0 + slot + e) * a.sr[1], restore8<FMT>(lo[e], hi[e], v_scale));
  }
}

template <int FMT>
void append_launch(const AppendArgs& a, dim3 grid, hipStream_t st) {
  switch (a.c.bs_log2) {
    case 4: cache_append_kernel<FMT, 1><<<grid, kThreads, 0, st>>>(a); break;
    case 5: cache_append_kernel<FMT, 2><<<grid, kThreads, 0, st>>>(a); break;
    case 6: cache_append_kernel<FMT, 4><<<grid, kThreads, 0, st>>>(a); break;
    default: cache_append_kernel<FMT, 8><<<grid, kThreads, 0, st>>>(a); break;
  }
}

template <int FMT>
void read_launch(const ReadArgs& a, dim3 grid, hipStream_t st) {
  switch (a.c.bs_log2) {
    case 4: cache_read_kernel<FMT, 1><<<grid, kThreads, 0, st>>>(a); break;
    case 5: cache_read_kernel<FMT, 2><<<grid, kThreads, 0, st>>>(a); break;
    case 6: cache_read_kernel<FMT, 4><<<grid, kThreads, 0, st>>>(a); break;
    default: cache_read_kernel<FMT, 8><<<grid, kThreads, 0, st>>>(a); break;
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
  const int64_t blocks = cache->B * cache->H * pages;
  if (!fits_grid(blocks, kThreads)) return KVP_ERR_SHAPE;
  a.pages = static_cast<uint32_t>(pages);
  a.div_h = FastDiv(a.c.H);
  a.div_pages = FastDiv(a.pages);
  const dim3 grid(static_cast<unsigned>(blocks));
  if (cache->format == KVP_CACHE_INT8)
    append_launch<KVP_CACHE_INT8>(a, grid, as_stream(stream));
  else
    append_launch<KVP_CACHE_E4M3>(a, grid, as_stream(stream));
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
  const int64_t blocks = cache->B * cache->H * pages;
  if (!fits_grid(blocks, kThreads)) return KVP_ERR_SHAPE;
  a.pages = static_cast<uint32_t>(pages);
  a.div_h = FastDiv(a.c.H);
  a.div_pages = FastDiv(a.pages);
  const dim3 grid(static_cast<unsigned>(blocks));
  if (cache->format == KVP_CACHE_INT8)
    read_launch<KVP_CACHE_INT8>(a, grid, as_stream(stream));
  else
    read_launch<KVP_CACHE_E4M3>(a, grid, as_stream(stream));
  return launch_status();
}
