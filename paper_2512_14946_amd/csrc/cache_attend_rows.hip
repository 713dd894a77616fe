// kvp_cache_attend with many query rows per (sequence, head): prompts, chunks of prompts; and the weights of more than 16 rows.
//
// Bound by the matrix and vector pipes, no longer by the cache's bytes, so every code is turned into a half once per block: a block
// of eight waves owns 256 rows, 32 per wave, and stages 64 tokens at a time in LDS as operands of v_mfma_f32_32x32x16_f16.
// Four buffers, one barrier per tile.  The arithmetic is that of cache_attend.hip: S^T = K Q^T leaves a lane with one query row
// and 32 of the 64 tokens, which are those that its operand of O^T = V^T P^T takes if the values' tokens are dealt out in the same order, so
// probabilities stay in the lane.  A tile has four runs of 16 tokens; a run lies in one page, so scales are uniform over the wave.
// The halves of a block are half a tile apart, so that one's products run beside the other's exponentials.  4 x 8 x 16384 keys, 4096 rows
// (causal): 1.00 to 1.09 ms, by the card, 1.06 to 0.97 PFLOP/s; a large library product of halves reaches 1.20.  Bound by power: 3500
// cycles a tile where the products alone take 2048 and the exponentials and staging 2300, at 1.75 GHz of 2.4.
// A probability is one half, of 11 bits for a result of 8: two, as for few rows, take 1.36 ms, and 387 us for 322 of 2 x 4 ragged to 30011 keys, 1421 rows.
// Measured against it at the same sizes, ms: both halves in step 1.03; 64 rows per wave, four waves 1.43 to 1.79; two blocks of 128 rows per CU
// 1.21; halves held apart by two barriers a tile 1.09 to 1.13; products and exponentials interleaved by hand 1.09 to 1.15, products
// and staging 1.07.
//
// LDS holds operands in the order of the lanes that read them (1 KB each, no conflicts), one or two slots further apart than that, so that
// the writes, whose neighbouring lanes belong to different operands, spread over the banks too.

#include <math.h>

#include <type_traits>

#include "cache_attend.h"

namespace kvp {
namespace {

typedef float floatx16 __attribute__((ext_vector_type(16)));

constexpr int kWaves = 8;
constexpr int kThreads = kWaves * kWave;
constexpr int kKeyPitch = 65, kValuePitch = 66;   // 16-byte slots from one operand to the next
constexpr float kLeastLog = -100.0f;         // log2 of value scales: one below counts as this one's fraction
constexpr float kMostPart = 60000.0f;        // most that eight probabilities, as halves, may sum to before the reference moves; just after it did, 2^13
constexpr int kBuffers = 4;       // tiles in LDS: being multiplied, next, being staged, and one of slack
static_assert(kManyRows == 32 * kWaves, "a wave owns 32 rows");

__device__ __forceinline__ half8_t as_half8(uint4 v) { return __builtin_bit_cast(half8_t, v); }
__device__ __forceinline__ uint4 as_uint4(half8_t v) { return __builtin_bit_cast(uint4, v); }
// row (of 32) of accumulator register v in lane half hb
__device__ __forceinline__ int acc_row(int hb, int v) { return hb * 4 + (v >> 2) * 8 + (v & 3); }

// One query row as operands of the eight 16-channel steps (this lane: channels 16 c + 8 hb ..+7), halves of q / 2^e with the sign
// of the softmax scale; returns the positive factor that makes base-2 logits of their products with codes.
__device__ __forceinline__ float load_query32(const uint16_t* row, int hb, bool valid, float scale2, half8_t qf[8]) {
  uint4 raw[8];
  float top = 0.0f;
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    raw[c] = make_uint4(0, 0, 0, 0);
    if (valid) raw[c] = *reinterpret_cast<const uint4*>(row + 16 * c + 8 * hb);
  }
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    float x[8];
    unpack_bf16x8(raw[c], x);
    top = fmaxf(top, abs_max8(x));
  }
  top = fmaxf(top, __shfl_xor(top, 32));
  const int e = __builtin_amdgcn_frexp_expf(top);   // 0 for a zero row
  const float sign = scale2 < 0.0f ? -1.0f : 1.0f;
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    float x[8];
    unpack_bf16x8(raw[c], x);
#pragma unroll
    for (int i = 0; i < 8; ++i) qf[c][i] = static_cast<_Float16>(ldexpf(x[i] * sign, -e));
  }
  return ldexpf(fabsf(scale2), e);
}

// Barrier of the block that leaves loads from memory in flight.
__device__ __forceinline__ void block_step() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

template <int FMT>
__global__ __launch_bounds__(kThreads, 2) void attend_rows_kernel(const AttendArgs a) {
  __shared__ uint4 k_s[kBuffers][16 * kKeyPitch], v_s[kBuffers][16 * kValuePitch];   // operands: keys [token block][channel step], values [channel block][run]
  __shared__ __attribute__((aligned(16))) float ks_s[kBuffers][4], vs_s[kBuffers][4];   // scales of the runs, of the values their log2
  uint32_t cell, chunk;
  if (!block_of(a, cell, chunk)) return;
  const Rows r = rows_of(a, cell);
  const uint32_t t0 = chunk * a.chunk, t1 = min(r.most, t0 + a.chunk);
  if (a.chunks > 1 && t0 >= t1) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), hb = lane >> 5, col = lane & 31;

  // this wave's 32 rows
  const uint32_t row0 = r.tile * kManyRows + wave * 32, row = row0 + col, w = a.div_g.quot(row), head = r.h * a.G + (row - w * a.G);
  const bool valid = row < a.M && static_cast<int32_t>(w) < r.m;
  half8_t qf[8];
  const float qs = load_query32(a.q + static_cast<int64_t>(r.b) * a.q_sb + static_cast<int64_t>(w) * a.q_sw + static_cast<int64_t>(head) * a.q_sh, hb,
                                valid, a.scale2, qf);
  const uint32_t limit = valid ? seen_by(a, r.n, r.m, w) : 0u;
  floatx16 o[4];
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[c][i] = 0.0f;
  // Tokens seen by the wave's first row, hence by all (rows that are none count for nothing); a tile below that needs no mask.
  uint32_t least = ~0u;
  if (row0 < a.M && static_cast<int32_t>(a.div_g.quot(row0)) < r.m) least = seen_by(a, r.n, r.m, a.div_g.quot(row0));
  float ref = kLeast, sum = 0.0f, vref = kLeastLog;   // vref: log2 of the reference scale

  // Staging: two waves a run of 16 tokens, so that pages and scales are a matter of the scalar unit.  Thread -> keys of token tid / 8,
  // channels 16 (tid mod 8) ..+15; values of channel 64 (wave mod 2) + lane, the whole run.
  const uint32_t bs_mask = (1u << a.c.bs_log2) - 1, run = wave >> 1;
  const int ch = (wave & 1) * 64 + lane;
  // two tiles' codes are on their way at any time: a tile's work is shorter than what memory takes
  uint4 kc[2], vc[2];
  float ks_c[2], vs_c[2];
  int32_t entry[2];
  int32_t zero = 0;   // in a vector register, so that addresses built with it are vector addresses
  asm volatile("" : "+v"(zero));
  // Everything by way of vector loads, whose waits are counted: a scalar load is waited for at the next barrier, and a scale's
  // cache line takes longer than a tile.
  auto next_entry = [&](uint32_t t, int set) {
    entry[set] = a.c.table[static_cast<int64_t>(r.b) * a.c.table_stride + (min(t + 16 * run, r.n - 1) >> a.c.bs_log2) + zero];
  };
  auto load_codes = [&](uint32_t t, int set) {
    const int64_t at = entry_cell(a, r.h, __builtin_amdgcn_readfirstlane(entry[set])), codes = at << (a.c.bs_log2 + 7);
    const uint32_t slot = (t + 16 * run) & bs_mask;
    kc[set] = *reinterpret_cast<const uint4*>(a.c.k_codes + codes + slot * kHeadDim + ((tid & 127) >> 3) * kHeadDim + (tid & 7) * 16);
    vc[set] = *reinterpret_cast<const uint4*>(a.c.v_codes + codes + slot + (static_cast<uint32_t>(ch) << a.c.bs_log2));
    ks_c[set] = a.c.k_scales[at + zero];
    vs_c[set] = a.c.v_scales[at + zero];
  };
  auto store_codes = [&](int buf, uint32_t t, int set) {
    const int c = tid & 7;
    if (t + kTileTokens > r.n) {             // bytes behind the last token may be anything: 0 * NaN is not 0
      const int live = static_cast<int>(min(max(static_cast<int64_t>(r.n) - (t + 16 * run), int64_t(0)), int64_t(16)));
      uint32_t* x = reinterpret_cast<uint32_t*>(&vc[set]);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] &= static_cast<uint32_t>((1ull << (8 * min(max(live - 4 * i, 0), 4))) - 1);
    }
    uint4* to = &k_s[buf][((wave >> 2) * 8 + c) * kKeyPitch + ((tid >> 3) & 31)];
    to[0] = as_uint4(decode8_half<FMT>(kc[set].x, kc[set].y));
    to[32] = as_uint4(decode8_half<FMT>(kc[set].z, kc[set].w));
    to = &v_s[buf][((ch >> 5) * 4 + run) * kValuePitch + (ch & 31)];
    // tokens of a run in the order of the logits' registers: 0-3 and 8-11 in the lower lanes, 4-7 and 12-15 in the upper
    to[0] = as_uint4(decode8_half<FMT>(vc[set].x, vc[set].z));
    to[32] = as_uint4(decode8_half<FMT>(vc[set].y, vc[set].w));
    if ((tid & 127) == 0) {
      ks_s[buf][run] = ks_c[set];
      vs_s[buf][run] = __builtin_amdgcn_logf(vs_c[set]);
    }
  };

  const uint32_t tiles = t1 > t0 ? (t1 - t0 + kTileTokens - 1) / kTileTokens : 0u;
  if (tiles > 0) {
    next_entry(t0, 0);
    next_entry(t0 + kTileTokens, 1);
    load_codes(t0, 0);
    next_entry(t0 + 2 * kTileTokens, 0);
    load_codes(t0 + kTileTokens, 1);        // behind the last tile: its last page again
    next_entry(t0 + 3 * kTileTokens, 1);
    store_codes(0, t0, 0);
    load_codes(t0 + 2 * kTileTokens, 0);
    next_entry(t0 + 4 * kTileTokens, 0);
    store_codes(1, t0 + kTileTokens, 1);
    load_codes(t0 + 3 * kTileTokens, 1);
    next_entry(t0 + 5 * kTileTokens, 1);
  }
  floatx16 s[2];
  half8_t pf[4];
  // The products of a step: values of a tile (PV), logits of the next (QK; behind the last tile, of whatever LDS holds: not used).
  // Operands come from LDS four at a time, two groups ahead of the four products that use them; consecutive products belong to
  // different accumulators.
  auto products = [&](auto pv_tag, int buf_v, int buf_k) {
    constexpr int kAhead = 3;
    constexpr int kPV = decltype(pv_tag)::value ? 4 : 0, kGroups = kPV + 4;
    half8_t x[kAhead][4];
    auto fetch = [&](auto g_tag) {
      constexpr int g = decltype(g_tag)::value;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (g < kPV)
          x[g % kAhead][j] = as_half8(v_s[buf_v][(j * 4 + g) * kValuePitch + lane]);
        else
          x[g % kAhead][j] = as_half8(k_s[buf_k][((j & 1) * 8 + 2 * (g - kPV) + (j >> 1)) * kKeyPitch + lane]);
      }
    };
#pragma unroll
    for (int tb = 0; tb < 2; ++tb)
#pragma unroll
      for (int k = 0; k < 16; ++k) s[tb][k] = 0.0f;
    auto group = [&](auto g_tag) {
      constexpr int g = decltype(g_tag)::value;
      if constexpr (g + kAhead - 1 < kGroups) fetch(std::integral_constant<int, g + kAhead - 1>{});
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (g < kPV)
          o[j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[g % kAhead][j], pf[g], o[j], 0, 0, 0);
        else
          s[j & 1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[g % kAhead][j], qf[2 * (g - kPV) + (j >> 1)], s[j & 1], 0, 0, 0);
      }
      if constexpr (g + kAhead - 1 < kGroups) __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);   // four reads of LDS,
      __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);                                           // then four products
    };
    fetch(std::integral_constant<int, 0>{});
    if constexpr (kAhead > 2) fetch(std::integral_constant<int, 1>{});
    __builtin_amdgcn_sched_group_barrier(0x100, 4 * (kAhead - 1), 0);
    group(std::integral_constant<int, 0>{});
    group(std::integral_constant<int, 1>{});
    group(std::integral_constant<int, 2>{});
    group(std::integral_constant<int, 3>{});
    if constexpr (kGroups == 8) {
      group(std::integral_constant<int, 4>{});
      group(std::integral_constant<int, 5>{});
      group(std::integral_constant<int, 6>{});
      group(std::integral_constant<int, 7>{});
    }
  };

  block_step();
  auto softmax = [&](uint32_t t, int buf) {
    {
      const float4 k4 = *reinterpret_cast<const float4*>(ks_s[buf]), v4 = *reinterpret_cast<const float4*>(vs_s[buf]);
      const float v_u[4] = {v4.x, v4.y, v4.z, v4.w};
      const float f[4] = {fmaxf(k4.x * qs, 0x1p-126f), fmaxf(k4.y * qs, 0x1p-126f), fmaxf(k4.z * qs, 0x1p-126f), fmaxf(k4.w * qs, 0x1p-126f)};
      if (t + kTileTokens > least) {         // some row does not see the whole tile; a factor is never 0: what is masked stays -inf
#pragma unroll
        for (int k = 0; k < 32; ++k) {
          const uint32_t tok = t + 32 * (k >> 4) + acc_row(hb, k & 15);
          s[k >> 4][k & 15] = tok < limit ? s[k >> 4][k & 15] : -INFINITY;
        }
      }
      // Probabilities times the page's share of the reference scale, which goes into the exponent (see cache_attend.hip).  The maximum is
      // not looked for: exponentials are taken against the present reference, and only if a run's sum comes near what halves hold
      // (or is not finite, as in the first tile), the reference moves and they are taken again.
      float total, worst;
      auto exponentials = [&]() {
        total = worst = 0.0f;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const float log_share = fmaxf(v_u[u] - vref, -60.0f), off = log_share - ref;
          float p[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) p[k] = __builtin_amdgcn_exp2f(fmaf(s[u >> 1][8 * (u & 1) + k], f[u], off));
          const float part = ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
          worst = fmaxf(worst, part);
          total = fmaf(part, __builtin_amdgcn_exp2f(-log_share), total);
#pragma unroll
          for (int k = 0; k < 8; ++k) pf[u][k] = static_cast<_Float16>(p[k]);
        }
      };
      exponentials();
      if (__builtin_amdgcn_ballot_w64(!(worst < kMostPart))) {
        float top = -INFINITY;
#pragma unroll
        for (int k = 0; k < 32; ++k) top = fmaxf(top, s[k >> 4][k & 15] * f[k >> 3]);
        const float ref_new = fmaxf(ref, fmaxf(top, __shfl_xor(top, 32)) - kBelow);
        const float v_new = fmaxf(vref, fmaxf(fmaxf(v_u[0], v_u[1]), fmaxf(v_u[2], v_u[3])));
        const float down = __builtin_amdgcn_exp2f(ref - ref_new), down_o = down * __builtin_amdgcn_exp2f(vref - v_new);
        sum *= down;
#pragma unroll
        for (int c = 0; c < 4; ++c) o[c] *= down_o;
        ref = ref_new;
        vref = v_new;
        exponentials();
      }
      sum += total;
    }
  };
  auto stage = [&](uint32_t i, int set) {
    const uint32_t t = t0 + i * kTileTokens;
    store_codes((i + 2) & (kBuffers - 1), t + 2 * kTileTokens, set);   // behind the last tile: into a buffer that is not read any more
    load_codes(t + 4 * kTileTokens, set);
    next_entry(t + 6 * kTileTokens, set);
  };
  // A SIMD has a wave of either half of the block.  Between two barriers the early one works out the probabilities of tile i, then the products
  // (values of i, keys of i + 1); the late one the products (values of i - 1, keys of i), then the probabilities: vector and matrix
  // instructions of two waves run at the same time, and most of them do (3500 cycles a tile, 4170 with both in step; the clock
  // falls under that load, and 1029 us become 1002).  Either half stages tile i + 2 behind what it does last, so four buffers are enough:
  // i - 1, i, i + 1 are read while i + 2 is written.
  const bool late = wave >= kWaves / 2;
  if (tiles > 0) {
    if (late) block_step();
    products(std::false_type{}, 0, 0);
    auto step = [&](uint32_t i, int set) {
      if (!late) block_step();
      softmax(t0 + i * kTileTokens, i & (kBuffers - 1));
      if (late) {
        stage(i, set);
        block_step();
      }
      products(std::true_type{}, i & (kBuffers - 1), (i + 1) & (kBuffers - 1));
      if (!late) stage(i, set);
    };
    uint32_t i = 0;
    for (; i + 1 < tiles; i += 2) {
      step(i, 0);
      step(i + 1, 1);
    }
    if (i < tiles) step(i, 0);
    if (!late) block_step();
  }

  const float z = sum + __shfl_xor(sum, 32), inv = z > 0.0f ? 1.0f / z : 0.0f, scale = __builtin_amdgcn_exp2f(vref);
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[c][i] = o[c][i] * inv * scale;   // in this order nothing leaves binary32's range
  if (!valid) return;
  const uint32_t in_tile = wave * 32 + col;
  if (a.chunks > 1) {
    const int64_t at = (static_cast<int64_t>(cell) * a.chunks + chunk) * a.tile_rows + in_tile;
    if (hb == 0) a.part_stat[at] = make_float2(ref, z);
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<float4*>(a.part_out + at * kHeadDim + 32 * c + 8 * i + 4 * hb) =
            make_float4(o[c][4 * i], o[c][4 * i + 1], o[c][4 * i + 2], o[c][4 * i + 3]);
    return;
  }
  if (a.row_bias && hb == 0) a.row_bias[static_cast<int64_t>(cell) * a.tile_rows + in_tile] = bias_of(ref, z);
  uint16_t* dst = a.out + static_cast<int64_t>(r.b) * a.o_sb + static_cast<int64_t>(w) * a.o_sw + static_cast<int64_t>(head) * a.o_sh;
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<uint2*>(dst + 32 * c + 8 * i + 4 * hb) =
          make_uint2(pack_bf16x2(o[c][4 * i], o[c][4 * i + 1]), pack_bf16x2(o[c][4 * i + 2], o[c][4 * i + 3]));
}

// What every token drew from all rows: drawn_t = sum over rows 2^(s_rt - bias_r).  A wave owns 32 tokens of a (sequence, head), their keys as
// operands in registers; 64 query rows at a time are copied to LDS for the four waves of a block.  Codes of either format are exact in
// bf16, so the rows need no conversion here.
// S^T = K Q^T: a lane has one query row, whose bias it keeps, and 16 of the tokens; it sums every 32nd row of each, and the
// lanes' sums are joined at the end, always in one order.
// Bound by the latency of a stage (products, exponentials, barrier) and by how many blocks a CU holds.  Blocks of 128 tokens against 512 with 64 per
// wave, whole call in us: 209, 350 (8 x 2048 keys, 8192 rows), 148, 178 (8 x 8192, 2048 rows), 180, 178 (4 x 30011, 1421), 920, 873 (8 x 32768, 4096).
constexpr int kSumThreads = kSumTokens / 32 * kWave;
constexpr int kSumRows = 64;
constexpr int kSumPairs = kSumRows * 8 / kSumThreads;   // runs of 16 channels that a thread copies per stage
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

// eight codes -> bf16 (exact)
template <int FMT>
__device__ __forceinline__ bf16x8_t decode8_bf16(uint32_t w0, uint32_t w1) {
  float x[8];
  decode4<FMT>(w0, x);
  decode4<FMT>(w1, x + 4);
  uint32_t u[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) u[i] = __builtin_amdgcn_perm(__float_as_uint(x[2 * i + 1]), __float_as_uint(x[2 * i]), 0x07060302u);
  return __builtin_bit_cast(bf16x8_t, make_uint4(u[0], u[1], u[2], u[3]));
}

template <int FMT>
__global__ __launch_bounds__(kSumThreads, 2) void weights_rows_kernel(const AttendArgs a, uint32_t groups, FastDiv div_groups) {
  __shared__ uint4 q_s[2][2][8 * 64];                                   // operands [row block][channel step]
  __shared__ float bias_s[2][kSumRows];
  __shared__ uint32_t limit_s[2][kSumRows];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), hb = lane >> 5, col = lane & 31;
  const uint32_t bh = div_groups.quot(blockIdx.x), t0 = (blockIdx.x - bh * groups) * kSumTokens, t = t0 + wave * 32;
  const uint32_t b = a.div_h.quot(bh), h = bh - b * a.c.H;
  const uint32_t n = min(cache_len(a.c, b), a.max_len);
  if (t0 >= n) return;
  int32_t m = static_cast<int32_t>(a.W);
  if (a.q_lens) m = min(max(a.q_lens[b], 0), m);

  // keys of two tokens: step 2 j + e takes channels 32 j + 16 hb + 8 e ..+7
  bf16x8_t kf[8];
  float f[2], drawn[16];   // factors of the runs of 16 tokens; sums: register v of token block tb at 16 tb + v
#pragma unroll
  for (int i = 0; i < 16; ++i) drawn[i] = 0.0f;
#pragma unroll
  for (int u = 0; u < 2; ++u) f[u] = a.c.k_scales[run_cell(a, b, h, t + 16 * u, n)] * a.scale2;
  {
    const uint32_t tok = t + col, run = tok & ~15u;
    const uint8_t* p = a.c.k_codes + (run_cell(a, b, h, run, n) << (a.c.bs_log2 + 7)) + (tok & ((1u << a.c.bs_log2) - 1)) * kHeadDim + hb * 16;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint4 x = *reinterpret_cast<const uint4*>(p + 32 * j);
      kf[2 * j] = decode8_bf16<FMT>(x.x, x.y);
      kf[2 * j + 1] = decode8_bf16<FMT>(x.z, x.w);
    }
  }
  const uint32_t tiles = (a.M + kSumRows - 1) / kSumRows, tile_log2 = __builtin_ctz(a.tile_rows);
  uint4 raw[kSumPairs][2];
  float bias = INFINITY;
  uint32_t limit = 0;
  auto load = [&](uint32_t i) {
#pragma unroll
    for (int u = 0; u < kSumPairs; ++u) {      // eight threads a row, sixteen channels each
      const int at = tid + u * kSumThreads;
      const uint32_t row = i * kSumRows + (at >> 3), w = a.div_g.quot(row), head = h * a.G + (row - w * a.G);
      raw[u][0] = raw[u][1] = make_uint4(0, 0, 0, 0);
      if (row < a.M && static_cast<int32_t>(w) < m) {
        const uint16_t* p = a.q + static_cast<int64_t>(b) * a.q_sb + static_cast<int64_t>(w) * a.q_sw + static_cast<int64_t>(head) * a.q_sh + (at & 7) * 16;
        raw[u][0] = *reinterpret_cast<const uint4*>(p);
        raw[u][1] = *reinterpret_cast<const uint4*>(p + 8);
      }
    }
    if (wave == 0) {
      const uint32_t row = i * kSumRows + lane, w = a.div_g.quot(row);
      bias = INFINITY;
      limit = 0;
      if (row < a.M && static_cast<int32_t>(w) < m) {
        // the tile that the attention launch put this row in, see rows_of
        const uint32_t tile = row >> tile_log2, cell = bh * a.row_tiles + (a.row_tiles - 1 - tile);
        bias = a.row_bias[static_cast<int64_t>(cell) * a.tile_rows + (row - (tile << tile_log2))];
        limit = seen_by(a, n, m, w);
      }
    }
  };
  auto store = [&](int buf) {
#pragma unroll
    for (int u = 0; u < kSumPairs; ++u) {
      const int at = tid + u * kSumThreads, row = at >> 3, step = 2 * ((at & 7) >> 1), half = at & 1;   // channels 16 p ..+15: steps 2 (p / 2) and the next, half p mod 2
#pragma unroll
      for (int j = 0; j < 2; ++j) q_s[buf][row >> 5][(step + j) * 64 + ((half * 32 + (row & 31)) ^ (step + j))] = raw[u][j];
    }
    if (wave == 0) {
      bias_s[buf][lane] = bias;
      limit_s[buf][lane] = limit;
    }
  };
  // the first rows of which any sees a token of this block
  uint32_t first = 0;
  if (a.causal) {
    const int64_t w = static_cast<int64_t>(t0) + m - n;                // tokens of query w and later see token t0
    if (w > 0) first = static_cast<uint32_t>(min(w * a.G, static_cast<int64_t>(a.M))) / kSumRows;
  }
  if (first < tiles) {
    load(first);
    store(0);
  }
  __syncthreads();
  int buf = 0;
  auto sum = [&](auto mask_tag) {
    constexpr bool MASK = decltype(mask_tag)::value;
    floatx16 s[2];
#pragma unroll
    for (int rb = 0; rb < 2; ++rb) {
#pragma unroll
      for (int k = 0; k < 16; ++k) s[rb][k] = 0.0f;
#pragma unroll
      for (int c = 0; c < 8; ++c)
        s[rb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[c], __builtin_bit_cast(bf16x8_t, q_s[buf][rb][c * 64 + (lane ^ c)]), s[rb], 0, 0, 0);
    }
#pragma unroll
    for (int rb = 0; rb < 2; ++rb) {
      const float row_bias = bias_s[buf][32 * rb + col];
      const uint32_t row_limit = MASK ? limit_s[buf][32 * rb + col] : 0u;
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        const float p = __builtin_amdgcn_exp2f(fmaf(s[rb][k], f[k >> 3], -row_bias));
        drawn[k] += !MASK || t + acc_row(hb, k) < row_limit ? p : 0.0f;
      }
    }
  };
  for (uint32_t i = first; i < tiles; ++i, buf ^= 1) {
    if (i + 1 < tiles) load(i + 1);
    const uint32_t w_first = a.div_g.quot(i * kSumRows), last = i * kSumRows + kSumRows - 1;
    const uint32_t least = last < a.M && static_cast<int32_t>(a.div_g.quot(last)) < m ? seen_by(a, n, m, w_first) : 0u;
    if (t + 32 > least)
      sum(std::true_type{});
    else
      sum(std::false_type{});
    if (i + 1 < tiles) store(buf ^ 1);
    __syncthreads();
  }
  // sums over the 32 lanes of a half: lane col ends up with drawn[col / 2]
#pragma unroll
  for (int d = 16; d > 1; d /= 2)
#pragma unroll
    for (int i = 0; i < d / 2; ++i) {
      const bool up = (lane & d) != 0;
      const float mine = up ? drawn[i + d / 2] : drawn[i], other = up ? drawn[i] : drawn[i + d / 2];
      drawn[i] = mine + __shfl_xor(other, d);
    }
  drawn[0] += __shfl_xor(drawn[0], 1);
  const uint32_t tok = t + acc_row(hb, col >> 1);
  if (tok < n && !(col & 1)) {
    const int64_t at = static_cast<int64_t>(bh) * a.acc_stride + tok;
    a.acc_out[at] = (a.acc_in ? a.acc_in[at] : 0.0f) + drawn[0];
  }
}

}  // namespace

void attend_rows_launch(const AttendArgs& a, int format, hipStream_t st) {
  const dim3 grid(a.per_xcd * 8);
  if (format == KVP_CACHE_INT8)
    attend_rows_kernel<KVP_CACHE_INT8><<<grid, kThreads, 0, st>>>(a);
  else
    attend_rows_kernel<KVP_CACHE_E4M3><<<grid, kThreads, 0, st>>>(a);
}

void weights_rows_launch(const AttendArgs& a, int format, hipStream_t st) {
  const int64_t groups = ceil_div(a.max_len, kSumTokens), blocks = groups * a.c.B * a.c.H;
  const FastDiv div(static_cast<uint32_t>(groups));
  const dim3 grid(static_cast<unsigned>(blocks));
  if (format == KVP_CACHE_INT8)
    weights_rows_kernel<KVP_CACHE_INT8><<<grid, kSumThreads, 0, st>>>(a, static_cast<uint32_t>(groups), div);
  else
    weights_rows_kernel<KVP_CACHE_E4M3><<<grid, kSumThreads, 0, st>>>(a, static_cast<uint32_t>(groups), div);
}

}  // namespace kvp
