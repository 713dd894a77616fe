// kvp_cache_attend: attention over the 8-bit paged cache, read in place.
//
//   out[r] = sum_t p_rt v_t,  p_rt = softmax_t(scale q_r . k_t),  k_t = s_k(page) code,  v_t = s_v(page) code
//
// One pass over the keys and values with a running maximum and sum.  A wave works on 64 tokens and 16 query rows at a time, with both
// contractions on v_mfma_f32_16x16x32_f16 and nothing in LDS: S^T = K Q^T leaves a lane with one query row (lane mod 16)
// and 16 tokens, which, with the keys' rows dealt to the products accordingly, are 16 consecutive ones, and exactly those
// that the lane's operand of O^T = V^T P^T takes: the probabilities never leave the lane, and its operand of V^T is 16 consecutive
// bytes of a channel, which is why values are stored channel-major.  Codes become halves in registers (exact); the page
// scale of the keys multiplies the logits, that of the values the probabilities (relative to the largest one so far, so that
// halves hold them).  Logits are kept in base 2.  The reference that exponentials are taken against follows the maximum
// lazily: it moves only when a logit exceeds it by 2^8, which P in halves and the sums in fp32 bear.
//
// A block's waves take every fourth 64-token tile of its chunk; partial results of chunks are joined by a second kernel.
// The weights of the tokens need the final statistics of their rows, so a further kernel forms the logits again.

#include <math.h>

#include "cache_attend_plan.h"
#include "cache_common.h"

namespace kvp {
namespace {

typedef float floatx4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = kAttendWaves;
constexpr int kThreads = kWaves * kWave;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kSlack = 8.0f;              // how far (base 2) a logit may exceed the reference of its row
constexpr float kValueSlack = 64.0f;        // and a page's value scale the reference scale: 2^8 * 2^6 fits a half
constexpr float kLeastScale = 0x1p-100f;    // value scales below this count as this one's fractions
constexpr int kOutPitch = 132;              // floats per row of partial outputs in LDS

struct AttendArgs {
  CacheArgs c;
  const uint16_t* q;
  uint16_t* out;
  int64_t q_sb, q_sw, q_sh, o_sb, o_sw, o_sh;
  const int32_t* q_lens;
  uint32_t W, G, M, row_tiles, max_len, chunk, chunks;
  FastDiv div_tiles, div_h, div_g, div_chunks;
  float scale2;                             // scale * log2(e)
  int32_t causal;
  float* part_out;                          // [cell][chunk][16][128] unnormalized, or null (one chunk)
  float2* part_stat;                        // [cell][chunk][16] (reference, sum)
  float2* row_stat;                         // [cell][16] (reference, 1 / sum), or null (no weights asked for)
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

__device__ __forceinline__ uint32_t seen_by(const AttendArgs& a, uint32_t n, int32_t m, uint32_t w) {
  if (!a.causal) return n;
  const int64_t p = static_cast<int64_t>(n) - m + w + 1;
  return p < 0 ? 0u : static_cast<uint32_t>(p);   // w < m: at most n
}

__device__ __forceinline__ Rows rows_of(const AttendArgs& a, uint32_t cell) {
  Rows r;
  const uint32_t bh = a.div_tiles.quot(cell);
  r.tile = cell - bh * a.row_tiles;
  r.b = a.div_h.quot(bh);
  r.h = bh - r.b * a.c.H;
  r.n = min(cache_len(a.c, r.b), a.max_len);
  r.m = static_cast<int32_t>(a.W);
  if (a.q_lens) r.m = min(max(a.q_lens[r.b], 0), r.m);
  const uint32_t w0 = a.div_g.quot(r.tile * kTileRows), w1 = a.div_g.quot(min(r.tile * kTileRows + kTileRows, a.M) - 1);
  r.least = r.most = 0;
  if (static_cast<int32_t>(w0) < r.m) {
    r.least = seen_by(a, r.n, r.m, w0);
    r.most = seen_by(a, r.n, r.m, min(w1, static_cast<uint32_t>(r.m) - 1));
  }
  return r;
}

// One query row as operands of the four channel steps: halves of q / 2^e, and what turns their products into base-2 logits.
// Step 2 jj + half of lane group g takes channels 64 jj + 16 g + 8 half ..+7, as the keys are loaded.
__device__ __forceinline__ float load_query(const uint16_t* row, int g, bool valid, float scale2, half8_t qf[4]) {
  uint4 raw[4];
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    raw[s] = make_uint4(0, 0, 0, 0);
    if (valid) raw[s] = *reinterpret_cast<const uint4*>(row + 64 * (s >> 1) + 16 * g + 8 * (s & 1));
  }
  float x[4][8], top = 0.0f;
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    unpack_bf16x8(raw[s], x[s]);
    top = fmaxf(top, abs_max8(x[s]));
  }
  top = fmaxf(top, __shfl_xor(top, 16));
  top = fmaxf(top, __shfl_xor(top, 32));
  const int e = __builtin_amdgcn_frexp_expf(top);   // 0 for a zero row
#pragma unroll
  for (int s = 0; s < 4; ++s)
#pragma unroll
    for (int i = 0; i < 8; ++i) qf[s][i] = static_cast<_Float16>(ldexpf(x[s][i], -e));
  return ldexpf(scale2, e);
}

// Pool page of the 16-token run that starts at token t; runs behind the last token take its page.
__device__ __forceinline__ int64_t run_cell(const AttendArgs& a, uint32_t b, uint32_t h, uint32_t t, uint32_t n) {
  return static_cast<int64_t>(cache_page(a.c, b, min(t, n - 1) >> a.c.bs_log2)) * a.c.H + h;
}

// Keys of 64 tokens: row r of product j is token 16 (r / 4) + 4 j + r mod 4, so that lane group g ends up with tokens 16 g ..+15
__device__ __forceinline__ void load_keys(const AttendArgs& a, int64_t cell, uint32_t t_run, int lane, uint4 k[4][2]) {
  const uint32_t slot = t_run & ((1u << a.c.bs_log2) - 1);
  const uint8_t* p = a.c.k_codes + (cell << (a.c.bs_log2 + 7)) + (slot + (lane & 3)) * kHeadDim + (lane >> 4) * 16;
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int jj = 0; jj < 2; ++jj) k[j][jj] = *reinterpret_cast<const uint4*>(p + 4 * j * kHeadDim + 64 * jj);
}
__device__ __forceinline__ void load_values(const AttendArgs& a, int64_t cell, uint32_t t_run, int lane, uint4 v[8]) {
  const uint32_t slot = t_run & ((1u << a.c.bs_log2) - 1);
  const uint8_t* p = a.c.v_codes + (cell << (a.c.bs_log2 + 7)) + (static_cast<uint32_t>(lane & 15) << a.c.bs_log2) + slot;
#pragma unroll
  for (int c = 0; c < 8; ++c) v[c] = *reinterpret_cast<const uint4*>(p + (static_cast<uint32_t>(16 * c) << a.c.bs_log2));
}

template <int FMT>
__device__ __forceinline__ void logits(const uint4 k[4][2], const half8_t qf[4], floatx4 s[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    s[j] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int jj = 0; jj < 2; ++jj) {
      s[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(decode8_half<FMT>(k[j][jj].x, k[j][jj].y), qf[2 * jj], s[j], 0, 0, 0);
      s[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(decode8_half<FMT>(k[j][jj].z, k[j][jj].w), qf[2 * jj + 1], s[j], 0, 0, 0);
    }
  }
}

template <int FMT>
__global__ __launch_bounds__(kThreads) void cache_attend_kernel(const AttendArgs a) {
  __shared__ __attribute__((aligned(16))) float out_s[kWaves][kTileRows * kOutPitch];
  __shared__ float ref_s[kWaves][kTileRows], sum_s[kWaves][kTileRows], val_s[kWaves];
  const uint32_t cell = a.div_chunks.quot(blockIdx.x), chunk = blockIdx.x - cell * a.chunks;
  const Rows r = rows_of(a, cell);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, col = lane & 15;
  const uint32_t t0 = chunk * a.chunk, t1 = min(r.most, t0 + a.chunk);
  if (a.chunks > 1 && t0 >= t1) return;      // the joining kernel knows which chunks there are

  // this lane's query row
  const uint32_t row = r.tile * kTileRows + col, w = a.div_g.quot(row), head = r.h * a.G + (row - w * a.G);
  const bool valid = row < a.M && static_cast<int32_t>(w) < r.m;
  half8_t qf[4];
  const float qs = load_query(a.q + static_cast<int64_t>(r.b) * a.q_sb + static_cast<int64_t>(w) * a.q_sw + static_cast<int64_t>(head) * a.q_sh, g,
                              valid, a.scale2, qf);
  const uint32_t limit = valid ? seen_by(a, r.n, r.m, w) : 0u;

  floatx4 o[8];
#pragma unroll
  for (int c = 0; c < 8; ++c) o[c] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
  float ref = -3.402823466e38f, sum = 0.0f, vref = kLeastScale;

  for (uint32_t t = t0 + wave * kTileTokens; t < t1; t += kWaves * kTileTokens) {
    const uint32_t run_k = t + 16 * (col >> 2), run = t + 16 * g;   // the runs this lane's keys and its tokens lie in
    uint4 k[4][2], v[8];
    load_keys(a, run_cell(a, r.b, r.h, run_k, r.n), run_k, lane, k);
    const int64_t cell_v = run_cell(a, r.b, r.h, run, r.n);
    load_values(a, cell_v, run, lane, v);
    const float f = a.c.k_scales[cell_v] * qs, vs = a.c.v_scales[cell_v];
    floatx4 s[4];
    logits<FMT>(k, qf, s);
    float x[16], top;
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = s[i >> 2][i & 3] * f;
    if (t + kTileTokens > r.least) {         // some row does not see the whole tile
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = run + i < limit ? x[i] : -INFINITY;
      if (t + kTileTokens > r.n) {           // bytes behind the last token may be anything: 0 * NaN is not 0
        const int live = static_cast<int>(min(max(static_cast<int64_t>(r.n) - run, int64_t(0)), int64_t(16)));
        uint32_t mask[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) mask[i] = static_cast<uint32_t>((1ull << (8 * min(max(live - 4 * i, 0), 4))) - 1);
#pragma unroll
        for (int c = 0; c < 8; ++c) v[c] = make_uint4(v[c].x & mask[0], v[c].y & mask[1], v[c].z & mask[2], v[c].w & mask[3]);
      }
    }
    top = x[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, x[i]);
    if (__builtin_amdgcn_ballot_w64(top > ref + kSlack || vs > kValueSlack * vref)) {   // wave-uniform
      float ref_new = fmaxf(ref, fmaxf(top, __shfl_xor(top, 16)));
      ref_new = fmaxf(ref_new, __shfl_xor(ref_new, 32));
      float v_new = fmaxf(vref, vs);
      v_new = fmaxf(v_new, __shfl_xor(v_new, 16));
      v_new = fmaxf(v_new, __shfl_xor(v_new, 32));
      const float down = __builtin_amdgcn_exp2f(ref - ref_new), down_o = down * (vref / v_new);
      sum *= down;
#pragma unroll
      for (int c = 0; c < 8; ++c) o[c] *= down_o;
      ref = ref_new;
      vref = v_new;
    }
    const float share = vs / vref;
    float p[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      p[i] = __builtin_amdgcn_exp2f(x[i] - ref);
      sum += p[i];
    }
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      half8_t pf;
#pragma unroll
      for (int i = 0; i < 8; ++i) pf[i] = static_cast<_Float16>(p[8 * half + i] * share);
#pragma unroll
      for (int c = 0; c < 8; ++c)
        o[c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(half ? decode8_half<FMT>(v[c].z, v[c].w) : decode8_half<FMT>(v[c].x, v[c].y), pf, o[c], 0, 0, 0);
    }
  }

  sum += __shfl_xor(sum, 16);
  sum += __shfl_xor(sum, 32);
#pragma unroll
  for (int c = 0; c < 8; ++c) *reinterpret_cast<floatx4*>(&out_s[wave][col * kOutPitch + 16 * c + 4 * g]) = o[c];
  if (g == 0) {
    ref_s[wave][col] = ref;
    sum_s[wave][col] = sum;
    if (col == 0) val_s[wave] = vref;
  }
  __syncthreads();
  // the waves' results joined: thread -> (row, eight channels)
  const int orow = threadIdx.x >> 4, ch = (threadIdx.x & 15) * 8;
  float m = ref_s[0][orow];
#pragma unroll
  for (int i = 1; i < kWaves; ++i) m = fmaxf(m, ref_s[i][orow]);
  float z = 0.0f, y[8] = {};
#pragma unroll
  for (int i = 0; i < kWaves; ++i) {
    const float f = __builtin_amdgcn_exp2f(ref_s[i][orow] - m), fv = f * val_s[i];
    z = fmaf(sum_s[i][orow], f, z);
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = fmaf(out_s[i][orow * kOutPitch + ch + j], fv, y[j]);
  }
  if (a.chunks > 1) {
    const int64_t at = (static_cast<int64_t>(cell) * a.chunks + chunk) * kTileRows + orow;
    float4* dst = reinterpret_cast<float4*>(a.part_out + at * kHeadDim + ch);
    dst[0] = make_float4(y[0], y[1], y[2], y[3]);
    dst[1] = make_float4(y[4], y[5], y[6], y[7]);
    if (ch == 0) a.part_stat[at] = make_float2(m, z);
    return;
  }
  const uint32_t r_out = r.tile * kTileRows + orow, w_out = a.div_g.quot(r_out);
  if (r_out >= a.M || static_cast<int32_t>(w_out) >= r.m) return;
  const float inv = z > 0.0f ? 1.0f / z : 0.0f;
  if (a.row_stat && ch == 0) a.row_stat[static_cast<int64_t>(cell) * kTileRows + orow] = make_float2(m, inv);
  uint16_t* dst = a.out + static_cast<int64_t>(r.b) * a.o_sb + static_cast<int64_t>(w_out) * a.o_sw +
                  static_cast<int64_t>(r.h * a.G + (r_out - w_out * a.G)) * a.o_sh + ch;
  *reinterpret_cast<uint4*>(dst) = make_uint4(pack_bf16x2(y[0] * inv, y[1] * inv), pack_bf16x2(y[2] * inv, y[3] * inv),
                                              pack_bf16x2(y[4] * inv, y[5] * inv), pack_bf16x2(y[6] * inv, y[7] * inv));
}

// The chunks of a row tile joined: a block per cell, thread -> (row, eight channels).
__global__ __launch_bounds__(kThreads) void cache_join_kernel(const AttendArgs a) {
  const uint32_t cell = blockIdx.x;
  const Rows r = rows_of(a, cell);
  const int orow = threadIdx.x >> 4, ch = (threadIdx.x & 15) * 8;
  const uint32_t row = r.tile * kTileRows + orow, w = a.div_g.quot(row);
  if (row >= a.M || static_cast<int32_t>(w) >= r.m) return;
  const uint32_t n = (r.most + a.chunk - 1) / a.chunk;
  const float2* st = a.part_stat + static_cast<int64_t>(cell) * a.chunks * kTileRows + orow;
  const float* po = a.part_out + (static_cast<int64_t>(cell) * a.chunks * kTileRows + orow) * kHeadDim + ch;
  float m = -3.402823466e38f;
  for (uint32_t i = 0; i < n; ++i) m = fmaxf(m, st[i * kTileRows].x);
  float z = 0.0f, y[8] = {};
  for (uint32_t i = 0; i < n; ++i) {
    const float2 s = st[i * kTileRows];
    const float f = __builtin_amdgcn_exp2f(s.x - m);
    z = fmaf(s.y, f, z);
    const float4 u = *reinterpret_cast<const float4*>(po + static_cast<int64_t>(i) * kTileRows * kHeadDim);
    const float4 v = *reinterpret_cast<const float4*>(po + static_cast<int64_t>(i) * kTileRows * kHeadDim + 4);
    y[0] = fmaf(u.x, f, y[0]); y[1] = fmaf(u.y, f, y[1]); y[2] = fmaf(u.z, f, y[2]); y[3] = fmaf(u.w, f, y[3]);
    y[4] = fmaf(v.x, f, y[4]); y[5] = fmaf(v.y, f, y[5]); y[6] = fmaf(v.z, f, y[6]); y[7] = fmaf(v.w, f, y[7]);
  }
  const float inv = z > 0.0f ? 1.0f / z : 0.0f;
  if (a.row_stat && ch == 0) a.row_stat[static_cast<int64_t>(cell) * kTileRows + orow] = make_float2(m, inv);
  uint16_t* dst = a.out + static_cast<int64_t>(r.b) * a.o_sb + static_cast<int64_t>(w) * a.o_sw +
                  static_cast<int64_t>(r.h * a.G + (row - w * a.G)) * a.o_sh + ch;
  *reinterpret_cast<uint4*>(dst) = make_uint4(pack_bf16x2(y[0] * inv, y[1] * inv), pack_bf16x2(y[2] * inv, y[3] * inv),
                                              pack_bf16x2(y[4] * inv, y[5] * inv), pack_bf16x2(y[6] * inv, y[7] * inv));
}

// What every token drew: a wave owns 64 tokens of a (sequence, head) and goes through all query rows that see them; its sums
// are complete and formed in one order.
template <int FMT>
__global__ __launch_bounds__(kThreads) void cache_weights_kernel(const AttendArgs a, uint32_t groups, FastDiv div_groups) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, col = lane & 15;
  const uint32_t bh = div_groups.quot(blockIdx.x), t = ((blockIdx.x - bh * groups) * kWaves + wave) * kTileTokens;
  const uint32_t b = a.div_h.quot(bh), h = bh - b * a.c.H;
  const uint32_t n = min(cache_len(a.c, b), a.max_len);
  if (t >= n) return;
  const uint32_t run_k = t + 16 * (col >> 2), run = t + 16 * g;
  uint4 k[4][2];
  load_keys(a, run_cell(a, b, h, run_k, n), run_k, lane, k);
  const float ks = a.c.k_scales[run_cell(a, b, h, run, n)];
  float drawn[16] = {};
  for (uint32_t tile = 0; tile < a.row_tiles; ++tile) {
    const Rows r = rows_of(a, bh * a.row_tiles + tile);
    if (r.most <= t) continue;               // uniform
    const uint32_t row = tile * kTileRows + col, w = a.div_g.quot(row), head = h * a.G + (row - w * a.G);
    const bool valid = row < a.M && static_cast<int32_t>(w) < r.m;
    half8_t qf[4];
    const float qs = load_query(a.q + static_cast<int64_t>(b) * a.q_sb + static_cast<int64_t>(w) * a.q_sw + static_cast<int64_t>(head) * a.q_sh, g,
                                valid, a.scale2, qf);
    const uint32_t limit = valid ? seen_by(a, n, r.m, w) : 0u;
    const float2 st = valid ? a.row_stat[(static_cast<int64_t>(bh) * a.row_tiles + tile) * kTileRows + col] : make_float2(0.0f, 0.0f);
    floatx4 s[4];
    logits<FMT>(k, qf, s);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float p = __builtin_amdgcn_exp2f(s[i >> 2][i & 3] * (ks * qs) - st.x) * st.y;
      drawn[i] += run + i < limit ? p : 0.0f;
    }
  }
#pragma unroll
  for (int i = 0; i < 16; ++i)
#pragma unroll
    for (int d = 1; d < 16; d *= 2) drawn[i] += __shfl_xor(drawn[i], d);
  const int64_t at = static_cast<int64_t>(bh) * a.acc_stride + run;
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (col == i && run + i < n) a.acc_out[at + i] = (a.acc_in ? a.acc_in[at + i] : 0.0f) + drawn[i];
}

}  // namespace
}  // namespace kvp

extern "C" size_t kvp_cache_attend_workspace_bytes(int64_t B, int64_t H, int64_t Hq, int64_t W, int64_t T, int32_t weights) {
  if (B <= 0 || H <= 0 || Hq <= 0 || Hq % H || W <= 0 || T <= 0) return 0;
  return kvp::make_attend_plan(B, H, Hq, W, T, weights != 0).bytes;
}

extern "C" int32_t kvp_cache_attend(const kvp_view* q, const kvp_cache* cache, const int32_t* q_lens, int32_t causal, float scale,
                                    const kvp_view* out, const float* acc_in, float* acc_out, int64_t acc_stride, int64_t max_len,
                                    void* ws, size_t ws_bytes, void* stream) {
  using namespace kvp;
  int32_t rc = check_cache(cache, true);
  if (rc == KVP_OK) rc = check_view(q);
  if (rc == KVP_OK) rc = check_view(out);
  if (rc != KVP_OK) return rc;
  if (acc_in && !acc_out) return KVP_ERR_NULL;
  if (q->L != cache->B || out->L != q->L || out->T != q->T || out->H != q->H || q->H % cache->H) return KVP_ERR_SHAPE;
  const int64_t G = q->H / cache->H, W = q->T, cap = cache->max_blocks * cache->bs;
  if (W >= (1ll << 24) || G >= (1ll << 24) || W * G >= (1ll << 24) || max_len < 0 || !isfinite(scale)) return KVP_ERR_SHAPE;
  if (max_len == 0 || max_len > cap) max_len = cap;
  if (acc_out && acc_stride < max_len) return KVP_ERR_SHAPE;
  if ((reinterpret_cast<uintptr_t>(q_lens) | reinterpret_cast<uintptr_t>(acc_in) | reinterpret_cast<uintptr_t>(acc_out)) & 3u) return KVP_ERR_ALIGN;
  const AttendPlan p = make_attend_plan(cache->B, cache->H, q->H, W, max_len, acc_out != nullptr);
  if (p.cells * p.chunks >= (1ll << 31)) return KVP_ERR_SHAPE;
  if (p.bytes != 0 && (!ws || ws_bytes < p.bytes || !aligned16(ws))) return KVP_ERR_WORKSPACE;
  AttendArgs a{};
  a.c = cache_args(cache);
  a.q = static_cast<const uint16_t*>(q->ptr);
  a.out = static_cast<uint16_t*>(const_cast<void*>(out->ptr));
  a.q_sb = q->stride_l; a.q_sw = q->stride_t; a.q_sh = q->stride_h;
  a.o_sb = out->stride_l; a.o_sw = out->stride_t; a.o_sh = out->stride_h;
  a.q_lens = q_lens;
  a.W = static_cast<uint32_t>(W);
  a.G = static_cast<uint32_t>(G);
  a.M = a.W * a.G;
  a.row_tiles = static_cast<uint32_t>(p.row_tiles);
  a.max_len = static_cast<uint32_t>(max_len);
  a.chunk = static_cast<uint32_t>(p.chunk);
  a.chunks = static_cast<uint32_t>(p.chunks);
  a.div_tiles = FastDiv(a.row_tiles);
  a.div_h = FastDiv(a.c.H);
  a.div_g = FastDiv(a.G);
  a.div_chunks = FastDiv(a.chunks);
  a.scale2 = scale * kLog2e;
  a.causal = causal;
  char* w = static_cast<char*>(ws);
  if (p.chunks > 1) {
    a.part_out = reinterpret_cast<float*>(w);
    a.part_stat = reinterpret_cast<float2*>(w + p.out_bytes);
  }
  a.acc_in = acc_in;
  a.acc_out = acc_out;
  a.acc_stride = acc_stride;
  if (acc_out) a.row_stat = reinterpret_cast<float2*>(w + p.out_bytes + p.stat_bytes);
  const hipStream_t st = as_stream(stream);
  const bool int8 = cache->format == KVP_CACHE_INT8;
  const dim3 grid(static_cast<unsigned>(p.cells * p.chunks));
  if (int8)
    cache_attend_kernel<KVP_CACHE_INT8><<<grid, kThreads, 0, st>>>(a);
  else
    cache_attend_kernel<KVP_CACHE_E4M3><<<grid, kThreads, 0, st>>>(a);
  if (p.chunks > 1) cache_join_kernel<<<dim3(static_cast<unsigned>(p.cells)), kThreads, 0, st>>>(a);
  if (acc_out) {
    const int64_t groups = ceil_div(max_len, kTileTokens * kWaves), blocks = groups * cache->B * cache->H;
    const FastDiv div(static_cast<uint32_t>(groups));
    if (int8)
      cache_weights_kernel<KVP_CACHE_INT8><<<dim3(static_cast<unsigned>(blocks)), kThreads, 0, st>>>(a, static_cast<uint32_t>(groups), div);
    else
      cache_weights_kernel<KVP_CACHE_E4M3><<<dim3(static_cast<unsigned>(blocks)), kThreads, 0, st>>>(a, static_cast<uint32_t>(groups), div);
  }
  return launch_status();
}
