// kvp_cache_evict: of every (sequence, head) of an 8-bit paged cache the tokens that drew the most attention stay.
//
// Three steps: the weights become ranks (protected tokens +inf, what lies behind the last token -inf), kvp_select_topk's kernels take the
// `budget` largest, ascending, and a block per (page of the destination, head, plane) gathers its tokens, reduces their
// largest magnitude and codes them on the page's own scale.
// With ties toward the lowest index a sequence of n < budget tokens selects 0 .. budget - 1: its tokens, and then entries that the
// last step knows to be none.

#include "cache_common.h"

namespace kvp {
namespace {

constexpr int kThreads = 256;

struct EvictArgs {
  CacheArgs src, dst;
  const float* acc;
  int64_t acc_stride, acc_out_stride;
  float* rank;                  // [B * H][T]
  const int32_t* kept;          // [B * H][k]
  int32_t* keep_idx;
  float* acc_out;
  int32_t* lens_out;
  uint32_t T, k, budget, sink, recent, pages;   // T: max_len; k = min(budget, T); pages of the destination per sequence
  FastDiv div_h, div_pages;
};

__device__ __forceinline__ uint32_t evict_len(const EvictArgs& a, uint32_t b) { return min(cache_len(a.src, b), a.T); }

__global__ __launch_bounds__(kThreads) void evict_rank_kernel(const EvictArgs a, uint32_t groups, FastDiv div_groups) {
  const uint32_t bh = div_groups.quot(blockIdx.x), t0 = (blockIdx.x - bh * groups) * 1024 + threadIdx.x;
  const uint32_t n = evict_len(a, a.div_h.quot(bh));
  const float* acc = a.acc + static_cast<int64_t>(bh) * a.acc_stride;
  float* rank = a.rank + static_cast<int64_t>(bh) * a.T;
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i) {
    const uint32_t t = t0 + i * kThreads;
    if (t >= a.T) break;
    float x = -INFINITY;
    if (t < n) x = t < a.sink || t + a.recent >= n ? INFINITY : acc[t];
    rank[t] = x;
  }
}

template <int FMT>
__global__ __launch_bounds__(kThreads) void evict_move_kernel(const EvictArgs a) {
  __shared__ __attribute__((aligned(16))) uint8_t turn_s[kHeadDim * (128 + 16)];   // values: [channel][slot], pitch bs + 16
  __shared__ int64_t from_s[128];           // pool cell of a slot's old page
  __shared__ int32_t slot_s[128];           // its old slot, -1: none
  __shared__ float scale_s[128], max_s[4];
  const CacheArgs &s = a.src, &d = a.dst;
  const uint32_t rest = a.div_h.quot(blockIdx.x), h = blockIdx.x - rest * s.H;
  const uint32_t bp = a.div_pages.quot(rest), p = rest - bp * a.pages, b = bp >> 1, plane = bp & 1;
  const uint32_t bs = 1u << s.bs_log2, n = evict_len(a, b), m = min(n, a.budget), bh = b * s.H + h, t0 = p << s.bs_log2;
  if (threadIdx.x < bs) {
    const uint32_t i = t0 + threadIdx.x;
    int32_t t = -1;
    // entries below m are tokens of the sequence; clamped all the same
    if (i < m) t = static_cast<int32_t>(min(static_cast<uint32_t>(a.kept[static_cast<int64_t>(bh) * a.k + i]), n - 1));
    if (plane == 0 && i < a.budget) {
      if (a.keep_idx) a.keep_idx[static_cast<int64_t>(bh) * a.budget + i] = t;
      if (a.acc_out && t >= 0) a.acc_out[static_cast<int64_t>(bh) * a.acc_out_stride + i] = a.acc[static_cast<int64_t>(bh) * a.acc_stride + t];
    }
    if (i == 0 && h == 0 && plane == 0 && a.lens_out) a.lens_out[b] = static_cast<int32_t>(m);
    if (t >= 0) {
      const int64_t cell = static_cast<int64_t>(cache_page(s, b, static_cast<uint32_t>(t) >> s.bs_log2)) * s.H + h;
      from_s[threadIdx.x] = cell;
      scale_s[threadIdx.x] = (plane ? s.v_scales : s.k_scales)[cell];
      t &= static_cast<int32_t>(bs - 1);
    }
    slot_s[threadIdx.x] = t;
  }
  if (t0 >= m) return;
  __syncthreads();
  const int live = static_cast<int>(min(m - t0, bs)), items = static_cast<int>(bs >> 4);
  const uint8_t* codes = plane ? s.v_codes : s.k_codes;
  uint2 raw[8];
  float amax = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (i >= items) break;
    const int slot = static_cast<int>((threadIdx.x + i * kThreads) >> 4), ch = static_cast<int>(threadIdx.x & 15) * 8;
    raw[i] = make_uint2(0, 0);
    if (slot < live) {
      const uint8_t* at = codes + (from_s[slot] << (s.bs_log2 + 7));
      const int old = slot_s[slot];
      if (plane) {
        uint32_t w[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const uint8_t* c = at + ((ch + 4 * k) << s.bs_log2) + old;
          w[k] = c[0] | (c[bs] << 8) | (c[2 * bs] << 16) | (static_cast<uint32_t>(c[3 * bs]) << 24);
        }
        raw[i] = make_uint2(w[0], w[1]);
      } else {
        raw[i] = *reinterpret_cast<const uint2*>(at + old * kHeadDim + ch);
      }
      float x[8];
      decode4<FMT>(raw[i].x, x);
      decode4<FMT>(raw[i].y, x + 4);
      amax = fmaxf(amax, abs_max8(x) * scale_s[slot]);   // rounding is monotonic: the largest product is the product of the largest
    }
  }
  amax = block_max256(amax, max_s);
  const float scale = amax / kCodeMax<FMT>;
  const PageQuantizer q(scale);
  const int64_t cell = static_cast<int64_t>(cache_page(d, b, p)) * d.H + h;
  if (threadIdx.x == 0) (plane ? d.v_scales : d.k_scales)[cell] = scale;
  uint8_t* out = (plane ? d.v_codes : d.k_codes) + (cell << (d.bs_log2 + 7));
  const int pitch = static_cast<int>(bs) + 16;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (i >= items) break;
    const int slot = static_cast<int>((threadIdx.x + i * kThreads) >> 4), ch = static_cast<int>(threadIdx.x & 15) * 8;
    if (slot >= live) continue;
    float x[8];
    decode4<FMT>(raw[i].x, x);
    decode4<FMT>(raw[i].y, x + 4);
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] *= scale_s[slot];
    const uint2 w = make_uint2(q.codes4<FMT>(x), q.codes4<FMT>(x + 4));
    if (plane == 0) {
      *reinterpret_cast<uint2*>(out + slot * kHeadDim + ch) = w;
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        turn_s[(ch + k) * pitch + slot] = static_cast<uint8_t>(w.x >> (8 * k));
        turn_s[(ch + 4 + k) * pitch + slot] = static_cast<uint8_t>(w.y >> (8 * k));
      }
    }
  }
  if (plane == 0) return;
  __syncthreads();
  for (int i = static_cast<int>(threadIdx.x); i < kHeadDim * items; i += kThreads) {
    const int ch = i >> (s.bs_log2 - 4), run = i & (items - 1), n_run = min(live - run * 16, 16);
    if (n_run <= 0) continue;
    uint8_t* at = out + (ch << s.bs_log2) + run * 16;
    const uint8_t* from = turn_s + ch * pitch + run * 16;
    if (n_run == 16) {
      *reinterpret_cast<uint4*>(at) = *reinterpret_cast<const uint4*>(from);
    } else {
      for (int k = 0; k < n_run; ++k) at[k] = from[k];
    }
  }
}

struct EvictLayout {
  size_t rank, kept, select, total;
};

EvictLayout evict_layout(int64_t B, int64_t H, int64_t T, int64_t budget) {
  const auto up = [](size_t n) { return (n + 255) / 256 * 256; };
  EvictLayout w{};
  const int64_t rows = B * H;
  w.rank = up(static_cast<size_t>(rows) * T * sizeof(float));
  w.kept = up(static_cast<size_t>(rows) * std::min(budget, T) * sizeof(int32_t));
  w.select = up(select_workspace_bytes(rows, T));
  w.total = w.rank + w.kept + w.select;
  return w;
}

}  // namespace
}  // namespace kvp

extern "C" size_t kvp_cache_evict_workspace_bytes(int64_t B, int64_t H, int64_t T, int64_t budget) {
  if (B <= 0 || H <= 0 || T <= 0 || budget <= 0) return 0;
  return kvp::evict_layout(B, H, T, budget).total;
}

extern "C" int32_t kvp_cache_evict(const kvp_cache* src, const float* acc, int64_t acc_stride, int64_t budget, int64_t sink,
                                   int64_t recent, const kvp_cache* dst, int32_t* keep_idx, float* acc_out, int64_t acc_out_stride,
                                   int32_t* lens_out, int64_t max_len, void* ws, size_t ws_bytes, void* stream) {
  using namespace kvp;
  int32_t rc = check_cache(src, true);
  if (rc == KVP_OK) rc = check_cache(dst, false);
  if (rc != KVP_OK) return rc;
  if (!acc) return KVP_ERR_NULL;
  if (src->B != dst->B || src->H != dst->H || src->bs != dst->bs || src->format != dst->format) return KVP_ERR_SHAPE;
  const int64_t cap = src->max_blocks * src->bs;
  if (max_len < 0) return KVP_ERR_SHAPE;
  if (max_len == 0 || max_len > cap) max_len = cap;
  if (budget <= 0 || sink < 0 || recent < 0 || sink > budget || recent > budget || sink + recent > budget) return KVP_ERR_SHAPE;
  if (dst->max_blocks * dst->bs < budget || acc_stride < max_len || (acc_out && acc_out_stride < budget) || max_len >= (1ll << 30)) return KVP_ERR_SHAPE;
  if ((reinterpret_cast<uintptr_t>(acc) | reinterpret_cast<uintptr_t>(keep_idx) | reinterpret_cast<uintptr_t>(acc_out) |
       reinterpret_cast<uintptr_t>(lens_out)) & 3u)
    return KVP_ERR_ALIGN;
  if (lens_out == src->lens || dst->block_table == src->block_table) return KVP_ERR_SHAPE;
  const int64_t rows = src->B * src->H, pages = ceil_div(budget, src->bs), groups = ceil_div(max_len, 1024);
  if (rows * 2 * pages >= (1ll << 31) || rows * groups >= (1ll << 31)) return KVP_ERR_SHAPE;
  const EvictLayout w = evict_layout(src->B, src->H, max_len, budget);
  if (!ws || ws_bytes < w.total || !aligned16(ws)) return KVP_ERR_WORKSPACE;
  EvictArgs a{};
  a.src = cache_args(src);
  a.dst = cache_args(dst);
  a.acc = acc;
  a.acc_stride = acc_stride;
  a.acc_out_stride = acc_out_stride;
  char* base = static_cast<char*>(ws);
  a.rank = reinterpret_cast<float*>(base);
  int32_t* kept = reinterpret_cast<int32_t*>(base + w.rank);
  a.kept = kept;
  a.keep_idx = keep_idx;
  a.acc_out = acc_out;
  a.lens_out = lens_out;
  a.T = static_cast<uint32_t>(max_len);
  a.budget = static_cast<uint32_t>(budget);
  a.k = static_cast<uint32_t>(std::min(budget, max_len));
  a.sink = static_cast<uint32_t>(sink);
  a.recent = static_cast<uint32_t>(recent);
  a.pages = static_cast<uint32_t>(pages);
  a.div_h = FastDiv(a.src.H);
  a.div_pages = FastDiv(a.pages);
  const hipStream_t st = as_stream(stream);
  evict_rank_kernel<<<dim3(static_cast<unsigned>(rows * groups)), kThreads, 0, st>>>(a, static_cast<uint32_t>(groups),
                                                                                      FastDiv(static_cast<uint32_t>(groups)));
  select_topk_launch(a.rank, rows, max_len, max_len, a.k, kept, base + w.rank + w.kept, st);
  const dim3 grid(static_cast<unsigned>(rows * 2 * pages));
  if (src->format == KVP_CACHE_INT8)
    evict_move_kernel<KVP_CACHE_INT8><<<grid, kThreads, 0, st>>>(a);
  else
    evict_move_kernel<KVP_CACHE_E4M3><<<grid, kThreads, 0, st>>>(a);
  return launch_status();
}
