// kvp_cache_evict: of every (sequence, head) of an 8-bit paged cache the tokens that drew the most attention stay.
//
// Three steps: the weights become ranks (protected tokens +inf, what lies behind the last token -inf), kvp_select_topk's kernels take the
// `budget` largest, ascending, and a block per (page of the destination, head) gathers its tokens, reduces their
// largest magnitudes and codes them on the page's own scales.
// Bound by the select for short contexts (8 heads x 4096 -> 2048 tokens: ranks 3 us, selection 6.5, move 7); for a batch by the values, of which
// a token touches every 64 bytes of its page: 16 x 8 x 16384 (three quarters of that in the mean) -> 4916 tokens in 113 us, 4.6 TB/s of
// whole pages, key rows and what is written; ranks and selection 18.  The whole call and a read took 305 us when values were gathered
// byte by byte, and take 196.  A block per plane: 198, and 72 against 64 for 4 x 8 x 8192 -> 4096 tokens in 16-token pages.
// With ties toward the lowest index a sequence of n < budget tokens selects 0 .. budget - 1: its tokens, and then entries that the
// last step knows to be none.

#include "cache_common.h"

namespace kvp {
namespace {

constexpr int kThreads = 256;
constexpr int kRankTokens = 4 * kThreads;   // tokens of a block that ranks

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
  const uint32_t bh = div_groups.quot(blockIdx.x), t0 = (blockIdx.x - bh * groups) * kRankTokens + threadIdx.x;
  const uint32_t n = evict_len(a, a.div_h.quot(bh));
  const float* acc = a.acc + static_cast<int64_t>(bh) * a.acc_stride;
  float* rank = a.rank + static_cast<int64_t>(bh) * a.T;
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i) {
    const uint32_t t = t0 + i * kThreads;
    if (t >= a.T) break;
    float x = -INFINITY;
    if (t < n) x = t < a.sink || t + a.recent >= n ? INFINITY : fminf(acc[t], 3.402823466e38f);   // nothing above a protected token
    rank[t] = x;
  }
}

// What the slots of a destination page hold: pool cell, slot and scale of the token that moves there.
struct Origins {
  int64_t cell[128];
  float k_scale[128], v_scale[128];
  int32_t slot[128];
  int32_t start[129];     // first slot of every stretch of slots whose tokens lie in one page, and the number of live slots
  int32_t count[2];       // stretches that begin in each wave's slots
};

template <int FMT>
__device__ __forceinline__ float decode1(uint32_t code) {
  if constexpr (FMT == KVP_CACHE_INT8)
    return static_cast<float>(static_cast<int>(__builtin_amdgcn_sbfe(static_cast<int>(code), 0, 8)));
  else
    return __builtin_amdgcn_cvt_f32_fp8(static_cast<int>(code), 0);
}

template <int FMT, int ITEMS>
__global__ __launch_bounds__(kThreads) void evict_move_kernel(const EvictArgs a) {
  constexpr int bs = 16 * ITEMS, pitch = bs + 4;
  __shared__ __attribute__((aligned(16))) uint8_t in_s[kHeadDim * pitch], out_s[kHeadDim * pitch];   // values: a page, and what moves: [channel][slot]
  __shared__ Origins from;
  __shared__ float max_s[2][4];
  const CacheArgs &s = a.src, &d = a.dst;
  const uint32_t rest = a.div_h.quot(blockIdx.x), h = blockIdx.x - rest * s.H;
  const uint32_t b = a.div_pages.quot(rest), p = rest - b * a.pages;
  const uint32_t n = evict_len(a, b), m = min(n, a.budget), bh = b * s.H + h, t0 = p * bs;
  const int tid = static_cast<int>(threadIdx.x);
  bool begins = false;
  if (tid < bs) {
    const uint32_t i = t0 + tid;
    int32_t t = -1, before = -1;
    // entries below m are tokens of the sequence; clamped all the same
    if (i < m) {
      const int32_t* kept = a.kept + static_cast<int64_t>(bh) * a.k + i;
      t = static_cast<int32_t>(min(static_cast<uint32_t>(kept[0]), n - 1));
      if (tid > 0) before = static_cast<int32_t>(min(static_cast<uint32_t>(kept[-1]), n - 1));
    }
    if (i < a.budget) {
      if (a.keep_idx) a.keep_idx[static_cast<int64_t>(bh) * a.budget + i] = t;
      if (a.acc_out && t >= 0) a.acc_out[static_cast<int64_t>(bh) * a.acc_out_stride + i] = a.acc[static_cast<int64_t>(bh) * a.acc_stride + t];
    }
    if (i == 0 && h == 0 && a.lens_out) a.lens_out[b] = static_cast<int32_t>(m);
    if (t >= 0) {
      const int64_t cell = static_cast<int64_t>(cache_page(s, b, static_cast<uint32_t>(t) >> s.bs_log2)) * s.H + h;
      from.cell[tid] = cell;
      from.k_scale[tid] = s.k_scales[cell];
      from.v_scale[tid] = s.v_scales[cell];
      from.slot[tid] = t & (bs - 1);
      begins = before < 0 || (before >> s.bs_log2) != (t >> s.bs_log2);
    }
  }
  if (t0 >= m) return;
  const int live = static_cast<int>(min(m - t0, static_cast<uint32_t>(bs)));
  const uint64_t votes = __builtin_amdgcn_ballot_w64(begins);
  if (tid < 128 && (tid & 63) == 0) from.count[tid >> 6] = __popcll(votes);
  __syncthreads();
  const int stretches = from.count[0] + (bs > 64 ? from.count[1] : 0);
  if (begins) from.start[(tid >> 6 ? from.count[0] : 0) + __popcll(votes & ((1ull << (tid & 63)) - 1))] = tid;
  if (tid == 0) from.start[stretches] = live;

  const int64_t cell_out = static_cast<int64_t>(cache_page(d, b, p)) * d.H + h;
  const int ch8 = (tid & 15) * 8;
  uint2 raw[ITEMS];
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const int slot = (tid >> 4) + 16 * i;
    raw[i] = make_uint2(0, 0);
    if (slot < live) raw[i] = load_stream8(s.k_codes + (from.cell[slot] << (s.bs_log2 + 7)) + from.slot[slot] * kHeadDim + ch8);
  }
  __syncthreads();   // the stretches

  // Values lie channel by channel, so a token touches every 64 bytes of its page: pages are read whole, the next while this one's tokens
  // are picked.  More than four pages that average fewer than four tokens each: byte by byte, all at once.  Whole call and a read, us,
  // always by bytes, always by pages (8 x 8 x 16384, kept 8192, 4096, 2048, 1024, 512, 200):
  //   64-token pages   217 167, 124 109, 79 85, 63 67, 51 73, 35 85;    this rule 161, 106, 83, 69, 51, 39
  //   16-token pages   254 214, 140 128, 83 85, 53 58, 35 39, 28 34;    this rule 208, 138, 87, 54, 36, 28
  float amax = 0.0f;
  const bool bytes = stretches * 4 > live && stretches > 4;
  uint4 page[(ITEMS + 1) / 2];
  auto load = [&](int j) {
    const uint8_t* at = s.v_codes + (from.cell[from.start[j]] << (s.bs_log2 + 7));
#pragma unroll
    for (int i = 0; i < (ITEMS + 1) / 2; ++i)
      if (tid + i * kThreads < kHeadDim * ITEMS) page[i] = load_stream16(at + (tid + i * kThreads) * 16);
  };
  if (!bytes) load(0);

  // keys, while the first page is on its way
  {
    float k_max = 0.0f;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int slot = (tid >> 4) + 16 * i;
      if (slot >= live) continue;
      float x[8];
      decode4<FMT>(raw[i].x, x);
      decode4<FMT>(raw[i].y, x + 4);
      k_max = fmaxf(k_max, abs_max8(x) * from.k_scale[slot]);   // rounding is monotonic: the largest product is the product of the largest
    }
    k_max = block_max256(k_max, max_s[0]);
    const float scale = k_max / kCodeMax<FMT>;
    const PageQuantizer q(scale);
    if (tid == 0) d.k_scales[cell_out] = scale;
    uint8_t* out = d.k_codes + (cell_out << (d.bs_log2 + 7)) + ch8;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int slot = (tid >> 4) + 16 * i;
      if (slot < live)
        *reinterpret_cast<uint2*>(out + slot * kHeadDim) = make_uint2(recode4<FMT>(raw[i].x, from.k_scale[slot], q), recode4<FMT>(raw[i].y, from.k_scale[slot], q));
    }
  }

  if (bytes) {
    for (int i = tid; i < live * 16; i += kThreads) {
      const int slot = i >> 4, ch = (i & 15) * 8;
      const uint8_t* at = s.v_codes + (from.cell[slot] << (s.bs_log2 + 7)) + ch * bs + from.slot[slot];
      uint32_t w[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) w[k] = at[k * bs];
      float top = 0.0f;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        out_s[(ch + k) * pitch + slot] = static_cast<uint8_t>(w[k]);
        top = fmaxf(top, fabsf(decode1<FMT>(w[k])));
      }
      amax = fmaxf(amax, top * from.v_scale[slot]);
    }
  } else {
    const int c = tid & 127;
    for (int j = 0; j < stretches; ++j) {
#pragma unroll
      for (int i = 0; i < (ITEMS + 1) / 2; ++i) {
        const int k = tid + i * kThreads;
        if (k >= kHeadDim * ITEMS) break;
        uint32_t* to = reinterpret_cast<uint32_t*>(in_s + (k / ITEMS) * pitch + (k % ITEMS) * 16);
        to[0] = page[i].x; to[1] = page[i].y; to[2] = page[i].z; to[3] = page[i].w;
      }
      __syncthreads();
      if (j + 1 < stretches) load(j + 1);
      const int first = from.start[j], last = from.start[j + 1];
      float top = 0.0f;
      for (int slot = first + (tid >> 7); slot < last; slot += 2) {
        const uint32_t code = in_s[c * pitch + from.slot[slot]];
        out_s[c * pitch + slot] = static_cast<uint8_t>(code);
        top = fmaxf(top, fabsf(decode1<FMT>(code)));
      }
      amax = fmaxf(amax, top * from.v_scale[first]);   // one page, one scale
      __syncthreads();
    }
  }
  amax = block_max256(amax, max_s[1]);
  const float scale = amax / kCodeMax<FMT>;
  const PageQuantizer q(scale);
  if (tid == 0) d.v_scales[cell_out] = scale;
  uint8_t* out = d.v_codes + (cell_out << (d.bs_log2 + 7));
#pragma unroll
  for (int i = 0; i < (ITEMS + 1) / 2; ++i) {
    const int k = tid + i * kThreads, run = k % ITEMS, n_run = min(live - run * 16, 16);
    if (k >= kHeadDim * ITEMS || n_run <= 0) continue;
    const uint32_t* in = reinterpret_cast<const uint32_t*>(out_s + (k / ITEMS) * pitch + run * 16);
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float x[4];
      decode4<FMT>(in[j], x);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = 4 * j + e < n_run ? x[e] * from.v_scale[run * 16 + 4 * j + e] : 0.0f;
      w[j] = q.codes4<FMT>(x);
    }
    uint8_t* at = out + (k / ITEMS) * bs + run * 16;
    if (n_run == 16) {
      *reinterpret_cast<uint4*>(at) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (e < n_run) at[e] = static_cast<uint8_t>(w[e >> 2] >> (8 * (e & 3)));
    }
  }
}

template <int FMT>
void move_launch(const EvictArgs& a, dim3 grid, hipStream_t st) {
  switch (a.src.bs_log2) {
    case 4: evict_move_kernel<FMT, 1><<<grid, kThreads, 0, st>>>(a); break;
    case 5: evict_move_kernel<FMT, 2><<<grid, kThreads, 0, st>>>(a); break;
    case 6: evict_move_kernel<FMT, 4><<<grid, kThreads, 0, st>>>(a); break;
    default: evict_move_kernel<FMT, 8><<<grid, kThreads, 0, st>>>(a); break;
  }
}

// the launches that rank and select fit a grid
bool rows_fit(int64_t rows, int64_t T) { return fits_grid(rows * ceil_div(T, kRankTokens), kThreads) && select_fits(rows, T); }

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
  constexpr int64_t kMost = 1ll << 31;   // what a call accepts: nothing below overflows
  if (B <= 0 || H <= 0 || T <= 0 || budget <= 0) return 0;
  if (B >= kMost || H >= kMost || B * H >= kMost || T >= (1ll << 30) || budget >= kMost) return 0;
  if (!kvp::rows_fit(B * H, T)) return 0;
  // scratch that serves every smaller T: the selection's too, which rows beyond kMaxSplitT do without
  return std::max(kvp::evict_layout(B, H, T, budget).total, kvp::evict_layout(B, H, std::min(T, kvp::kMaxSplitT), budget).total);
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
  if (lens_out == src->lens || acc_out == acc || dst->block_table == src->block_table) return KVP_ERR_SHAPE;
  const int64_t rows = src->B * src->H, pages = ceil_div(budget, src->bs), groups = ceil_div(max_len, kRankTokens);
  if (!fits_grid(rows * pages, kThreads) || !rows_fit(rows, max_len)) return KVP_ERR_SHAPE;
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
  const dim3 grid(static_cast<unsigned>(rows * pages));
  if (src->format == KVP_CACHE_INT8)
    move_launch<KVP_CACHE_INT8>(a, grid, st);
  else
    move_launch<KVP_CACHE_E4M3>(a, grid, st);
  return launch_status();
}
