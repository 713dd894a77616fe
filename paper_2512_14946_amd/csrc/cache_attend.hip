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
// halves hold them).  Logits are kept in base 2.  The reference that exponentials are taken against is set 2^10 below the maximum and follows it
// lazily: it moves only when a probability times its page's share exceeds 2^15.5, which halves and the sums in fp32 bear.
//
// A probability has 11 bits as a half, while the result is rounded to the 8 of bf16.  Where a call has one tile of 16 rows it is taken as two halves, 22 bits,
// which costs half a percent beside the memory (us with one, two: 89.0, 89.3 for 4 x 4 x 131072 tokens, 7 rows; 154.6, 155.0 for 33 x 8 x 12000, 4 rows;
// 11.3 both for 8 x 4096).  More rows keep one: 53.9, 55.3 (16 x 8 x 8192, 20 rows), 71.6, 82.2 (64 rows), 1001, 1363 (4 x 8 x 16384, 4096 rows).
//
// This file: up to 128 query rows per (sequence, head) in tiles of 16 or 32, a decode step above all, bound by HBM.  A block's waves take a quarter
// of its chunk each, with the loads of the next 64 tokens always in flight; partial results of chunks are joined by a second kernel.
// The weights of the tokens need the final statistics of their rows: up to 16 rows the logits are kept and the second kernel sums them.
// More rows, and the weights of more than 16: cache_attend_rows.hip.
// 4 x 4 x 131072 tokens, 7 rows: 89 us, 6.06 TB/s (a copy reaches 6.5); 64 x 8 x 16384 (ragged, three quarters of that), 8 rows: 285 us, 5.6 TB/s,
// and 435 with weights: the logits cost 12 us to keep, 78 to store beside the reads, and the joining kernel takes 54; 8 x 4096, 4 rows: 11 us,
// two launches and the latency of length, table, scale and code.  Decoding holds several tiles: 16 x 8 x 8192 tokens take 54 us for 20 rows
// and 118 for 96.

#include <math.h>

#include <type_traits>

#include "cache_attend.h"

namespace kvp {
namespace {

typedef float floatx4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = kAttendWaves;
constexpr int kThreads = kWaves * kWave;
constexpr int kKeptFloats = 4096;           // logits that a wave keeps in LDS: 4 tiles of 16 rows, 8 of 8
constexpr float kMostLog = 15.5f;           // log2 of the most that a probability times its page's share may be: halves end at 2^16
constexpr int kOutPitch = 132;              // floats per row of partial outputs in LDS
constexpr uint32_t kSlice = kJoinTokens;
static_assert(kSlice == 4 * kThreads, "16 threads a tile of 64 tokens");

// One query row as operands of the four channel steps: halves of q / 2^e with the sign of the softmax scale, and the positive factor that turns
// their products with codes into base-2 logits.
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
  const float sign = scale2 < 0.0f ? -1.0f : 1.0f;
#pragma unroll
  for (int s = 0; s < 4; ++s)
#pragma unroll
    for (int i = 0; i < 8; ++i) qf[s][i] = static_cast<_Float16>(ldexpf(x[s][i] * sign, -e));
  return ldexpf(fabsf(scale2), e);
}

__device__ __forceinline__ uint32_t run_k_of(uint32_t t, int col) { return t + 16 * (col >> 2); }

// 16 bytes of codes.  What one block reads streams past the caches; what the row tiles of a chunk share stays in the L2 of their XCD.
// One tile: 90 us against 99 with plain loads (4 x 4 x 131072 tokens); two to six tiles: 86 us against 70 (16 x 8 x 8192, 32 rows).
template <bool SHARED>
__device__ __forceinline__ uint4 load_codes16(const uint8_t* p) {
  if constexpr (SHARED) return *reinterpret_cast<const uint4*>(p);
  return load_stream16(p);
}

// Keys of 64 tokens: row r of product j is token 16 (r / 4) + 4 j + r mod 4, so that lane group g ends up with tokens 16 g ..+15
template <bool SHARED>
__device__ __forceinline__ void load_keys(const AttendArgs& a, int64_t cell, uint32_t t_run, int lane, uint4 k[4][2]) {
  const uint32_t slot = t_run & ((1u << a.c.bs_log2) - 1);
  const uint8_t* p = a.c.k_codes + (cell << (a.c.bs_log2 + 7)) + (slot + (lane & 3)) * kHeadDim + (lane >> 4) * 16;
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int jj = 0; jj < 2; ++jj) k[j][jj] = load_codes16<SHARED>(p + 4 * j * kHeadDim + 64 * jj);
}
template <bool SHARED>
__device__ __forceinline__ void load_values(const AttendArgs& a, int64_t cell, uint32_t t_run, int lane, uint4 v[8]) {
  const uint32_t slot = t_run & ((1u << a.c.bs_log2) - 1);
  const uint8_t* p = a.c.v_codes + (cell << (a.c.bs_log2 + 7)) + (static_cast<uint32_t>(lane & 15) << a.c.bs_log2) + slot;
#pragma unroll
  for (int c = 0; c < 8; ++c) v[c] = load_codes16<SHARED>(p + (static_cast<uint32_t>(16 * c) << a.c.bs_log2));
}

template <int FMT, int R>
__device__ __forceinline__ void logits(const uint4 k[4][2], const half8_t qf[R][4], floatx4 s[R][4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
#pragma unroll
    for (int u = 0; u < R; ++u) s[u][j] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int jj = 0; jj < 2; ++jj) {
      const half8_t lo = decode8_half<FMT>(k[j][jj].x, k[j][jj].y), hi = decode8_half<FMT>(k[j][jj].z, k[j][jj].w);
#pragma unroll
      for (int u = 0; u < R; ++u) {
        s[u][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(lo, qf[u][2 * jj], s[u][j], 0, 0, 0);
        s[u][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(hi, qf[u][2 * jj + 1], s[u][j], 0, 0, 0);
      }
    }
  }
}

// What a lane has stored to LDS is there for the others of its wave: the compiler may not move accesses across, nor take the lanes apart.
__device__ __forceinline__ void wave_step() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

// LOGITS: they are kept for the weights (one row tile); SHARED: several row tiles; R: groups of 16 rows, which share every code's decoding
template <int FMT, bool LOGITS, bool SHARED, int R>
__global__ __launch_bounds__(kThreads) void cache_attend_kernel(const AttendArgs a) {
  constexpr int kRows = 16 * R, kOutFloats = kRows * kOutPitch;
  constexpr int kParts = SHARED || R > 1 ? 1 : 2;   // halves of a probability
  __shared__ __attribute__((aligned(16))) float shared_s[kWaves * (LOGITS ? kKeptFloats : kOutFloats)];   // kept logits, then the waves' results
  __shared__ float ref_s[kWaves][kRows], sum_s[kWaves][kRows], val_s[kWaves];
  uint32_t cell, chunk;
  if (!block_of(a, cell, chunk)) return;
  const Rows r = rows_of(a, cell);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, col = lane & 15;
  const uint32_t t0 = chunk * a.chunk, t1 = min(r.most, t0 + a.chunk);
  if (a.chunks > 1 && t0 >= t1) return;      // the joining kernel knows which chunks there are

  // this lane's query rows
  half8_t qf[R][4];
  float qs[R];
  uint32_t limit[R];
#pragma unroll
  for (int u = 0; u < R; ++u) {
    const uint32_t row = r.tile * kRows + 16 * u + col, w = a.div_g.quot(row), head = r.h * a.G + (row - w * a.G);
    const bool valid = row < a.M && static_cast<int32_t>(w) < r.m;
    qs[u] = load_query(a.q + static_cast<int64_t>(r.b) * a.q_sb + static_cast<int64_t>(w) * a.q_sw + static_cast<int64_t>(head) * a.q_sh, g, valid,
                       a.scale2, qf[u]);
    limit[u] = valid ? seen_by(a, r.n, r.m, w) : 0u;
  }

  // Logits kept for the weights leave by way of LDS, some tiles at a time: loads that a wave requests after a store wait for that
  // store too, and a few stores in every tile cost 129 us of 409 at 64 x 8 x 12288 tokens and 8 rows.
  float* kept_s = reinterpret_cast<float*>(shared_s) + wave * kKeptFloats;
  const uint32_t keep = kKeptFloats / (a.M * kTileTokens);
  uint32_t n_kept = 0;

  floatx4 o[R][8];
  float ref[R], sum[R], vref = kLeastScale, inv_vref = 1.0f / kLeastScale;
#pragma unroll
  for (int u = 0; u < R; ++u) {
#pragma unroll
    for (int c = 0; c < 8; ++c) o[u][c] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    ref[u] = kLeast;
    sum[u] = 0.0f;
  }

  // The keys of the next tile are requested when this tile's are used up, its values likewise, with the scales and the table entries
  // of the tile after it in between: one set of registers, loads in flight all the time, and none waited for before its turn.
  constexpr uint32_t kStep = kTileTokens;
  const uint32_t part_tokens = (t1 > t0 ? (t1 - t0 + kWaves * kTileTokens - 1) / (kWaves * kTileTokens) : 0u) * kTileTokens;   // tokens of a wave
  uint32_t t = t0 + wave * part_tokens;
  const uint32_t t_end = min(t1, t + part_tokens);
  uint4 k[4][2], v[8];
  float ks, vs;
  int32_t entry_k = 0, entry_v = 0;
  if (t < t_end) {
    const int64_t cell_k = run_cell(a, r.b, r.h, run_k_of(t, col), r.n), cell_v = run_cell(a, r.b, r.h, t + 16 * g, r.n);
    load_keys<SHARED>(a, cell_k, run_k_of(t, col), lane, k);
    ks = a.c.k_scales[cell_v];
    vs = a.c.v_scales[cell_v];
    entry_k = run_entry(a, r.b, run_k_of(t + kStep, col), r.n);
    entry_v = run_entry(a, r.b, t + kStep + 16 * g, r.n);
    load_values<SHARED>(a, cell_v, t + 16 * g, lane, v);
  }
  // MORE is known at compile time: behind a branch around the loads, every wait would have to count them as not issued.
  auto tile = [&](auto more_tag) {
    constexpr bool MORE = decltype(more_tag)::value;
    const uint32_t run = t + 16 * g;       // the 16 tokens of this lane
    const float vs_now = vs;
    float f[R];
#pragma unroll
    for (int u = 0; u < R; ++u) f[u] = fmaxf(ks * qs[u], 0x1p-126f);   // never 0: what is masked stays -inf
    floatx4 s[R][4];
    logits<FMT, R>(k, qf, s);
    int64_t cell_v = 0;
    if constexpr (MORE) {
      cell_v = entry_cell(a, r.h, entry_v);
      load_keys<SHARED>(a, entry_cell(a, r.h, entry_k), run_k_of(t + kStep, col), lane, k);
      ks = a.c.k_scales[cell_v];
      vs = a.c.v_scales[cell_v];
      entry_k = run_entry(a, r.b, run_k_of(t + 2 * kStep, col), r.n);
      entry_v = run_entry(a, r.b, run + 2 * kStep, r.n);
    }
    if (t + kTileTokens > r.least) {         // some row does not see the whole tile
#pragma unroll
      for (int u = 0; u < R; ++u)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[u][i >> 2][i & 3] = run + i < limit[u] ? s[u][i >> 2][i & 3] : -INFINITY;
      if (t + kTileTokens > r.n) {           // bytes behind the last token may be anything: 0 * NaN is not 0
        const int live = static_cast<int>(min(max(static_cast<int64_t>(r.n) - run, int64_t(0)), int64_t(16)));
        uint32_t mask[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) mask[i] = static_cast<uint32_t>((1ull << (8 * min(max(live - 4 * i, 0), 4))) - 1);
#pragma unroll
        for (int c = 0; c < 8; ++c) v[c] = make_uint4(v[c].x & mask[0], v[c].y & mask[1], v[c].z & mask[2], v[c].w & mask[3]);
      }
    }
    if constexpr (LOGITS) {
      // to LDS, as they lie in memory: [i][row][g][4]
      if (col < static_cast<int>(a.M)) {
        float4* to = reinterpret_cast<float4*>(kept_s) + (n_kept * 4 * a.M + col) * 4 + g;
#pragma unroll
        for (int i = 0; i < 4; ++i) to[i * a.M * 4] = make_float4(s[0][i][0] * f[0], s[0][i][1] * f[0], s[0][i][2] * f[0], s[0][i][3] * f[0]);
      }
      ++n_kept;
    }
    // Probabilities times the page's share of the reference scale: the share goes into the exponent, and the sum of the tile is divided by it.
    // A share below 2^-60 leaves nothing of a half either way, and a page of zeros has none: both count as 2^-60.
    float log_share = fmaxf(__builtin_amdgcn_logf(vs_now * inv_vref), -60.0f);
    float top[R];
    bool moves = false;
#pragma unroll
    for (int u = 0; u < R; ++u) {
      top[u] = s[u][0][0];
#pragma unroll
      for (int i = 1; i < 16; ++i) top[u] = fmaxf(top[u], s[u][i >> 2][i & 3]);
      top[u] *= f[u];                        // f > 0
      moves = moves || log_share + fmaxf(top[u] - ref[u], 0.0f) > kMostLog;   // a share alone too: what is masked may lie in a page of any scale
    }
    if (__builtin_amdgcn_ballot_w64(moves)) {   // wave-uniform
      float v_new = fmaxf(vref, vs_now);
      v_new = fmaxf(v_new, __shfl_xor(v_new, 16));
      v_new = fmaxf(v_new, __shfl_xor(v_new, 32));
#pragma unroll
      for (int u = 0; u < R; ++u) {
        float most = fmaxf(top[u], __shfl_xor(top[u], 16));
        most = fmaxf(most, __shfl_xor(most, 32));
        const float ref_new = fmaxf(ref[u], most - kBelow);
        const float down = __builtin_amdgcn_exp2f(ref[u] - ref_new), down_o = down * (vref / v_new);
        sum[u] *= down;
#pragma unroll
        for (int c = 0; c < 8; ++c) o[u][c] *= down_o;
        ref[u] = ref_new;
      }
      vref = v_new;
      inv_vref = 1.0f / v_new;
      log_share = fmaxf(__builtin_amdgcn_logf(vs_now * inv_vref), -60.0f);
    }
    const float per_share = __builtin_amdgcn_exp2f(-log_share);
    half8_t pf[kParts][R][2];
#pragma unroll
    for (int u = 0; u < R; ++u) {
      const float off = log_share - ref[u];
      float p[16], part = 0.0f;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        p[i] = __builtin_amdgcn_exp2f(fmaf(s[u][i >> 2][i & 3], f[u], off));
        part += p[i];
      }
      sum[u] = fmaf(part, per_share, sum[u]);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const _Float16 x = static_cast<_Float16>(p[i]);
        pf[0][u][i >> 3][i & 7] = x;
        if constexpr (kParts > 1) pf[1][u][i >> 3][i & 7] = static_cast<_Float16>(p[i] - static_cast<float>(x));
      }
    }
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const half8_t x = half ? decode8_half<FMT>(v[c].z, v[c].w) : decode8_half<FMT>(v[c].x, v[c].y);
#pragma unroll
        for (int u = 0; u < R; ++u)
#pragma unroll
          for (int part = 0; part < kParts; ++part) o[u][c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x, pf[part][u][half], o[u][c], 0, 0, 0);
      }
    if constexpr (MORE) load_values<SHARED>(a, cell_v, run + kStep, lane, v);
    if constexpr (LOGITS) {
      if (!MORE || n_kept == keep) {
        wave_step();
        float4* to = reinterpret_cast<float4*>(a.logits + static_cast<int64_t>(cell) * a.M * a.logit_stride + static_cast<int64_t>(t - (n_kept - 1) * kTileTokens) * a.M);
        for (uint32_t i = lane; i < n_kept * a.M * 16; i += kWave) {
          const float4 u = reinterpret_cast<const float4*>(kept_s)[i];
          store_stream16(to + i, make_uint4(__float_as_uint(u.x), __float_as_uint(u.y), __float_as_uint(u.z), __float_as_uint(u.w)));
        }
        wave_step();   // read before the next tiles' overwrite it
        n_kept = 0;
      }
    }
  };
  for (; t + kStep < t_end; t += kStep) tile(std::true_type{});
  if (t < t_end) tile(std::false_type{});
  if constexpr (LOGITS) __syncthreads();   // the waves' results go where others may still keep logits

#pragma unroll
  for (int u = 0; u < R; ++u) {
    sum[u] += __shfl_xor(sum[u], 16);
    sum[u] += __shfl_xor(sum[u], 32);
    const int in = 16 * u + col;
#pragma unroll
    for (int c = 0; c < 8; ++c) *reinterpret_cast<floatx4*>(&shared_s[wave * kOutFloats + in * kOutPitch + 16 * c + 4 * g]) = o[u][c];
    if (g == 0) {
      ref_s[wave][in] = ref[u];
      sum_s[wave][in] = sum[u];
    }
  }
  if (lane == 0) val_s[wave] = vref;
  __syncthreads();
  // the waves' results joined: thread -> (row, eight channels)
#pragma unroll
  for (int u = 0; u < R; ++u) {
    const int orow = 16 * u + (threadIdx.x >> 4), ch = (threadIdx.x & 15) * 8;
    float m = ref_s[0][orow];
#pragma unroll
    for (int i = 1; i < kWaves; ++i) m = fmaxf(m, ref_s[i][orow]);
    float e[kWaves], z = 0.0f, y[8] = {};
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
      e[i] = __builtin_amdgcn_exp2f(ref_s[i][orow] - m);
      z = fmaf(sum_s[i][orow], e[i], z);
    }
    const float inv = z > 0.0f ? 1.0f / z : 0.0f;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
      const float part = e[i] * inv, scale = val_s[i];   // divided by the sum first, then times the scale: neither leaves binary32's range
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = fmaf(shared_s[i * kOutFloats + orow * kOutPitch + ch + j] * part, scale, y[j]);
    }
    const int64_t at = (static_cast<int64_t>(cell) * a.chunks + chunk) * kRows + orow;
    const uint32_t row = r.tile * kRows + orow, w = a.div_g.quot(row);
    if (a.part_stat && ch == 0) a.part_stat[at] = make_float2(m, z);
    if (a.chunks > 1) {
      if (row >= a.M) continue;
      float4* dst = reinterpret_cast<float4*>(a.part_out + at * kHeadDim + ch);
      dst[0] = make_float4(y[0], y[1], y[2], y[3]);
      dst[1] = make_float4(y[4], y[5], y[6], y[7]);
      continue;
    }
    if (row >= a.M || static_cast<int32_t>(w) >= r.m) continue;
    if (a.row_bias && ch == 0) a.row_bias[static_cast<int64_t>(cell) * kRows + orow] = bias_of(m, z);
    uint16_t* dst = a.out + static_cast<int64_t>(r.b) * a.o_sb + static_cast<int64_t>(w) * a.o_sw + static_cast<int64_t>(r.h * a.G + (row - w * a.G)) * a.o_sh + ch;
    *reinterpret_cast<uint4*>(dst) = make_uint4(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7]));
  }
}

// Row statistics over the chunks of a cell, by the 16 lanes that share `row`: (reference, sum); n chunks, `pitch` rows apart.
__device__ __forceinline__ float2 joined_stats(const float2* st, uint32_t pitch, uint32_t n, uint32_t lane16) {
  float m = kLeast, z = 0.0f;
  for (uint32_t i = lane16; i < n; i += 16) {
    const float2 s = st[static_cast<int64_t>(i) * pitch];
    const float m_new = fmaxf(m, s.x);
    z = fmaf(z, __builtin_amdgcn_exp2f(m - m_new), s.y * __builtin_amdgcn_exp2f(s.x - m_new));
    m = m_new;
  }
#pragma unroll
  for (int d = 1; d < 16; d *= 2) {
    const float m2 = __shfl_xor(m, d), z2 = __shfl_xor(z, d), m_new = fmaxf(m, m2);
    // written so that both lanes of an exchange form the same sum
    const float lo = z * __builtin_amdgcn_exp2f(m - m_new), hi = z2 * __builtin_amdgcn_exp2f(m2 - m_new);
    z = lo + hi;
    m = m_new;
  }
  return make_float2(m, z);
}

// The chunks of a row joined (blocks below n_join: one per row of a cell), and, with logits kept, what every token drew
// (the other blocks: kSlice tokens of a cell each).  Both work out the final statistics of their rows from the chunks'.
__global__ __launch_bounds__(kThreads) void cache_join_kernel(const AttendArgs a, uint32_t n_join, uint32_t join_rows, FastDiv div_rows, uint32_t slices,
                                                              FastDiv div_slices) {
  __shared__ __attribute__((aligned(16))) float4 part_s[8][32];
  __shared__ float2 stat_s[kTileRows];
  const uint32_t tid = threadIdx.x;
  if (blockIdx.x < n_join) {
    const uint32_t cell = div_rows.quot(blockIdx.x), orow = blockIdx.x - cell * join_rows;
    const Rows r = rows_of(a, cell);
    const uint32_t row = r.tile * a.tile_rows + orow, w = a.div_g.quot(row);
    if (row >= a.M || static_cast<int32_t>(w) >= r.m) return;
    const uint32_t n = (r.most + a.chunk - 1) / a.chunk;
    const float2* st = a.part_stat + static_cast<int64_t>(cell) * a.chunks * a.tile_rows + orow;
    const float2 stat = joined_stats(st, a.tile_rows, n, tid & 15);
    if (a.row_bias && tid == 0) a.row_bias[static_cast<int64_t>(cell) * a.tile_rows + orow] = bias_of(stat.x, stat.y);
    const float inv = stat.y > 0.0f ? 1.0f / stat.y : 0.0f;
    const uint32_t group = tid >> 5, ch = tid & 31;
    const float4* po = reinterpret_cast<const float4*>(a.part_out + (static_cast<int64_t>(cell) * a.chunks * a.tile_rows + orow) * kHeadDim) + ch;
    float4 y = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
    for (uint32_t i = group; i < n; i += 8) {
      const float2 s = st[static_cast<int64_t>(i) * a.tile_rows];
      const float f = __builtin_amdgcn_exp2f(s.x - stat.x) * (s.y * inv);   // the chunk's part of the row's weight
      const float4 u = po[static_cast<int64_t>(i) * a.tile_rows * (kHeadDim / 4)];
      y.x = fmaf(u.x, f, y.x); y.y = fmaf(u.y, f, y.y); y.z = fmaf(u.z, f, y.z); y.w = fmaf(u.w, f, y.w);
    }
    part_s[group][ch] = y;
    __syncthreads();
    if (group) return;
#pragma unroll
    for (int i = 1; i < 8; ++i) {
      const float4 u = part_s[i][ch];
      y.x += u.x; y.y += u.y; y.z += u.z; y.w += u.w;
    }
    uint16_t* dst = a.out + static_cast<int64_t>(r.b) * a.o_sb + static_cast<int64_t>(w) * a.o_sw +
                    static_cast<int64_t>(r.h * a.G + (row - w * a.G)) * a.o_sh + ch * 4;
    *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16x2(y.x, y.y), pack_bf16x2(y.z, y.w));
    return;
  }
  // one row tile per (sequence, head) here: a cell is a (sequence, head)
  const uint32_t id = blockIdx.x - n_join, cell = div_slices.quot(id), t0 = (id - cell * slices) * kSlice;
  const Rows r = rows_of(a, cell);
  if (t0 >= r.n) return;
  {
    const uint32_t orow = tid >> 4, w = a.div_g.quot(orow);
    float2 stat = make_float2(0.0f, 0.0f);
    if (orow < a.M && static_cast<int32_t>(w) < r.m)
      stat = joined_stats(a.part_stat + static_cast<int64_t>(cell) * a.chunks * a.tile_rows + orow, a.tile_rows, (r.most + a.chunk - 1) / a.chunk, tid & 15);
    if ((tid & 15) == 0) stat_s[orow] = make_float2(stat.x, stat.y > 0.0f ? 1.0f / stat.y : 0.0f);
  }
  __syncthreads();
  // 16 threads a tile, thread 4 i + g has tokens 16 g + 4 i ..+3
  const uint32_t tile0 = t0 + (tid >> 4) * kTileTokens, t = tile0 + (tid & 3) * 16 + ((tid >> 2) & 3) * 4;
  if (t >= r.n) return;
  float drawn[4] = {};
  if (tile0 < r.most) {   // a tile beyond what any row sees has no logits
    const float* x = a.logits + static_cast<int64_t>(cell) * a.M * a.logit_stride + static_cast<int64_t>(tile0) * a.M + (((tid >> 2) & 3) * a.M * 4 + (tid & 3)) * 4;
    for (uint32_t i = 0; i < a.M; ++i) {
      const float4 u = *reinterpret_cast<const float4*>(x + i * 16);
      const float2 stat = stat_s[i];
      drawn[0] = fmaf(__builtin_amdgcn_exp2f(u.x - stat.x), stat.y, drawn[0]);
      drawn[1] = fmaf(__builtin_amdgcn_exp2f(u.y - stat.x), stat.y, drawn[1]);
      drawn[2] = fmaf(__builtin_amdgcn_exp2f(u.z - stat.x), stat.y, drawn[2]);
      drawn[3] = fmaf(__builtin_amdgcn_exp2f(u.w - stat.x), stat.y, drawn[3]);
    }
  }
  const int64_t at = static_cast<int64_t>(cell) * a.acc_stride + t;
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i)
    if (t + i < r.n) a.acc_out[at + i] = (a.acc_in ? a.acc_in[at + i] : 0.0f) + drawn[i];
}

template <int FMT>
void few_rows_launch(const AttendArgs& a, dim3 grid, bool keep, int64_t tile_rows, hipStream_t st) {
  if (tile_rows == kTileRows)
    (keep              ? cache_attend_kernel<FMT, true, false, 1>
     : a.row_tiles > 1 ? cache_attend_kernel<FMT, false, true, 1>
                       : cache_attend_kernel<FMT, false, false, 1>)<<<grid, kThreads, 0, st>>>(a);
  else
    (a.row_tiles > 1 ? cache_attend_kernel<FMT, false, true, 2> : cache_attend_kernel<FMT, false, false, 2>)<<<grid, kThreads, 0, st>>>(a);
}

}  // namespace
}  // namespace kvp

extern "C" size_t kvp_cache_attend_workspace_bytes(int64_t B, int64_t H, int64_t Hq, int64_t W, int64_t T, int32_t weights) {
  constexpr int64_t kMost = 1ll << 31, kRows = 1ll << 24;   // what a call accepts: nothing below overflows
  if (B <= 0 || H <= 0 || Hq <= 0 || Hq % H || W <= 0 || T <= 0) return 0;
  if (B >= kMost || H >= kMost || B * H >= kMost || T >= kMost || W >= kRows || Hq / H >= kRows || Hq / H * W >= kRows) return 0;
  const kvp::AttendPlan p = kvp::make_attend_plan(B, H, Hq, W, T, weights != 0);
  return kvp::attend_fits(kvp::attend_blocks(p, B * H, Hq / H * W, T, weights != 0)) ? p.bytes : 0;
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
  const AttendBlocks blocks = attend_blocks(p, cache->B * cache->H, W * G, max_len, acc_out != nullptr);
  if (!attend_fits(blocks)) return KVP_ERR_SHAPE;
  if (p.bytes != 0 && (!ws || ws_bytes < p.bytes || !aligned16(ws))) return KVP_ERR_WORKSPACE;
  if (out->ptr == q->ptr) return KVP_ERR_SHAPE;   // several blocks, and the weights' pass, read a query row
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
  a.tile_rows = static_cast<uint32_t>(p.tile_rows);
  a.row_tiles = static_cast<uint32_t>(p.row_tiles);
  a.max_len = static_cast<uint32_t>(max_len);
  a.chunk = static_cast<uint32_t>(p.chunk);
  a.chunks = static_cast<uint32_t>(p.chunks);
  a.div_tiles = FastDiv(a.row_tiles);
  a.div_h = FastDiv(a.c.H);
  a.div_g = FastDiv(a.G);
  a.blocks = static_cast<uint32_t>(p.cells * p.chunks);
  a.per_xcd = static_cast<uint32_t>(blocks.attend / 8);
  a.div_bh = FastDiv(a.chunks * a.row_tiles);
  a.scale2 = scale * kLog2e;
  a.causal = causal;
  char* w = static_cast<char*>(ws);
  if (p.out_bytes) a.part_out = reinterpret_cast<float*>(w);
  if (p.stat_bytes) a.part_stat = reinterpret_cast<float2*>(w + p.out_bytes);
  if (p.row_bytes) a.row_bias = reinterpret_cast<float*>(w + p.out_bytes + p.stat_bytes);
  if (p.logit_bytes) a.logits = reinterpret_cast<float*>(w + p.out_bytes + p.stat_bytes + p.row_bytes);
  a.logit_stride = p.logit_stride;
  a.acc_in = acc_in;
  a.acc_out = acc_out;
  a.acc_stride = acc_stride;
  const hipStream_t st = as_stream(stream);
  const bool int8 = cache->format == KVP_CACHE_INT8;
  const dim3 grid(a.per_xcd * 8);
  const bool keep = p.logit_bytes != 0;
  if (p.tile_rows == kManyRows)
    attend_rows_launch(a, cache->format, st);
  else if (int8)
    few_rows_launch<KVP_CACHE_INT8>(a, grid, keep, p.tile_rows, st);
  else
    few_rows_launch<KVP_CACHE_E4M3>(a, grid, keep, p.tile_rows, st);
  const uint32_t join_rows = std::min(a.M, a.tile_rows), slices = static_cast<uint32_t>(ceil_div(max_len, kSlice));
  if (blocks.join_rows + blocks.join_sums > 0)
    cache_join_kernel<<<dim3(static_cast<unsigned>(blocks.join_rows + blocks.join_sums)), kThreads, 0, st>>>(
        a, static_cast<uint32_t>(blocks.join_rows), join_rows, FastDiv(join_rows), slices, FastDiv(slices));
  if (blocks.sums > 0) weights_rows_launch(a, cache->format, st);
  return launch_status();
}
