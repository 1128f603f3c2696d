// Attention over a cache held in 4 bits (nova_kv_q4_attn).
//
// A row of the cache is k = offset + scale * c with 4-bit codes c, so
//   q . k_j = scale_j (q . c_j) + offset_j sum(q)
//   out     = (sum_j (p_j scale'_j) c'_j + sum_j p_j offset'_j) / sum_j p_j
// and both products run on the matrix cores over the codes themselves.
//
// Scores of bf16 queries: on the fp16 cores, with codes as (c - 8) * 2^-9 like the
// values below (nine instructions for eight codes), and the query times a power of two
// that brings its row's largest magnitude to [2^13, 2^14): fp16 holds a bf16 number
// exactly down to 2^-29 of the largest. (Two 7-bit digits on the integer cores take 32
// instructions a round less, 405 us of the 409 below, but a coordinate 2^10 below the
// largest keeps 4 bits of them.)
// Of fp32 queries: on the 8-bit integer cores, exact. A word's codes are two words of
// bytes (three instructions); the query is a fixed-point number of three digits of
// 8 bits of its row's largest magnitude.
//
// Values: on the fp16 cores, as (c - 8) * 2^-9: a nibble masked in place is the fp16
// denormal c * 2^-24 (c * 2^-20, its bits four higher), which one packed multiply-add
// scales and centres exactly. (The cores multiply the denormal itself exactly
// too, but align it with the sum so far by its exponent field, ten bits above its
// value, and cut those bits off the sum: 1e-5 of an output, towards one side.)
//
// With 4 query heads a KV head, bf16 (8 KV heads of 128): 64 sequences of 32K tokens
// take 409 us, 5.6 TB/s of HBM, which bounds them; one of 128K 39 us, the reads'
// 24 us, their ramp and 9 us of merge; one of 2000 tokens 9.8 us, latency.
// fp32: 5 sequences of up to 5003 tokens, 10 rows a KV head, 19.7 us, latency and vector issue.
#include <algorithm>
#include <initializer_list>
#include <type_traits>

#include "q4_common.h"

namespace novakv {

namespace {

using namespace q4;

constexpr int kRound = 32;  // tokens a wave takes at a time

// D: head_dim. WIDE: fp32 queries. NT: tiles of 16 rows a wave. W: waves of a
// workgroup. TILED: each wave has rows of its own and all tokens, else the waves
// share the rows and divide the tokens. ALIGNED: blocks of a multiple of 16 rows.
template <int D, bool WIDE, int NT, int W, bool TILED, bool ALIGNED>
__global__ __launch_bounds__(64 * W, W > 4 ? 1 : NT > 1 ? 1 : WIDE && D == 128 ? 2 : 3) void q4_attn_kernel(const Q4AttnArgs a) {
  constexpr int kWaves = W, WT = TILED ? 1 : W;
  constexpr int kSteps = D / (WIDE ? 64 : 32);  // matrix steps of a score
  constexpr int kTiles = D / 16;          // output tiles
  constexpr int kKeyWords = D / 32;       // words of a lane's part of a key row
  constexpr int kDigits = 3;              // 8-bit digits of an fp32 query
  constexpr float kTopQ = 127.f * 256 * 256;  // the largest fixed-point number
  // A logit in front of its row's factor alpha: keys times this, so that
  // the products of large ones (up to 2^114) with scaled queries stay in fp32.
  constexpr int kKeyExp = 6;
  constexpr float kKeyUnit = 0x1p-6f;
  constexpr int kProbParts = WIDE ? 3 : 1;  // and of a probability
  // log2 of the largest scaled probability after a rescale, and how far it may
  // grow before the next one: 2^14 fits fp16, 2^11 units of 1 are 11 bits. Scaled
  // by the value's scale or, where that is less, 2^-8 of its offset's magnitude (of
  // code 8), at least 2^-70: sums of probabilities and of offsets stay in range too.
  constexpr float kTop = WIDE ? 10.f : 6.f, kSlack = WIDE ? 1.f : 8.f;
  constexpr int kRowGroups = kWaves / WT; // waves on rows of their own
  constexpr int kRows = 16 * NT * kRowGroups;
  using Lds = FinishLds<D, NT, W, TILED>;

  __shared__ __align__(16) uint32_t s_rows[ALIGNED ? 1 : kWaves][kRound];
  __shared__ __align__(16) float s_scale[kWaves][2 * kRound], s_offset[kWaves][2 * kRound], s_log[kWaves][2 * kRound];
  __shared__ float s_ref[kWaves][16 * NT], s_sum[kWaves][16 * NT];
  __shared__ __align__(16) float s_merge[Lds::kMerge];
  __shared__ float s_inv[kRows];
  __shared__ int s_last;

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int lane = threadIdx.x & 63, n = lane & 15, j = lane >> 4;
  const int tw = wave % WT, rw = wave / WT;

  Tile g;
  place_tile(a, kRows, g);
  // The queries are requested first: nothing of them waits for the sequence's
  // length. (Rows past the sequence's own are padding, whatever they hold.)
  const int row0 = g.row0 + rw * 16 * NT;
  uint4 qraw[NT][kKeyWords][WIDE ? 2 : 1];
  for (int t = 0; t < NT; ++t) {
    const int row = row0 + 16 * t + n, i = row / a.gqa, h = row - i * a.gqa;
    const size_t at = ((static_cast<size_t>(g.b) * a.n_q + i) * a.num_q_heads + g.kv * a.gqa + h) * D + 8 * kKeyWords * j;
    for (int s = 0; s < kKeyWords; ++s)
      for (int y = 0; y < (WIDE ? 2 : 1); ++y) {
        qraw[t][s][y] = make_uint4(0u, 0u, 0u, 0u);
        if (i < a.n_q)
          qraw[t][s][y] = WIDE ? reinterpret_cast<const uint4 *>(static_cast<const float *>(a.q) + at + 8 * s)[y]
                               : *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(a.q) + at + 8 * s);
      }
  }
  if (!find_span(a, kRows, kRound * WT, g)) return;
  const int b = g.b, kv = g.kv, rows_valid = g.rows_valid, lo = g.lo, t0 = g.t0, t1 = g.t1;

  // this wave's rows
  const int row1 = min(row0 + 16 * NT, rows_valid);
  const bool idle = row0 >= rows_valid;
  const int inner_lo = idle ? 0 : g.first_pos(a, row1 - 1), inner_hi = idle ? 0 : g.last_pos(a, row0) + 1;

  // Rounds of 32 tokens, the codes, scales and offsets of one requested while
  // the round before is computed, its block-table entries one round earlier.
  const int bs = a.layout.block_size, bps = a.layout.blocks_per_seq;
  const uint32_t block_rows = static_cast<uint32_t>(a.num_kv_heads) * bs, head_row = static_cast<uint32_t>(kv) * bs;
  const int32_t *table = a.layout.block_table ? a.layout.block_table + static_cast<size_t>(b) * bps : nullptr;
  const uint32_t *sq = reinterpret_cast<const uint32_t *>(lane < 32 ? a.k_sq : a.v_sq);
  const uint32_t k_lane = n * (D / 2) + 4 * kKeyWords * j, v_lane = 4 * j * (D / 2) + 4 * (n & (D / 8 - 1));
  constexpr int kStep = kRound * WT;
  int look = t0 + kRound * tw + (lane & 31);  // the lane's token of the round that is looked up next
  int look_blk = look / bs, look_row = look - look_blk * bs;
  const int step_blk = kStep / bs, step_row = kStep - step_blk * bs;
  int phys = -1, phys_tok = 0, phys_row = 0;
  auto look_up = [&]() {
    phys = -1;
    phys_tok = look;
    phys_row = look_row;
    if (look_blk < bps) {
      const long long own = static_cast<long long>(b) * bps + look_blk;
      phys = table ? table[look_blk] : own < a.num_blocks ? static_cast<int>(own) : -1;
    }
    look += kStep;
    look_blk += step_blk;
    look_row += step_row;
    if (look_row >= bs) look_row -= bs, ++look_blk;
  };
  struct Round {
    uint32_t kw[2][kKeyWords], vw[8], sq;
    bool ok;
  };
  // Requests the round that was looked up. A token outside the span counts as
  // masked; one in a block that holds nothing too, in its place a row at the
  // pool's start is read.
  auto request = [&](Round &r) {
    const bool held = static_cast<uint32_t>(phys) < static_cast<uint32_t>(a.num_blocks);
    r.ok = held && phys_tok < t1 && phys_tok >= lo;
    uint32_t row = static_cast<uint32_t>(phys) * block_rows + head_row + phys_row;
    if constexpr (ALIGNED) {  // blocks of a multiple of 16 rows: a half round's rows follow each other
      if (!held) row = lane & 15;
      for (int h = 0; h < 2; ++h) {
        const size_t first = static_cast<size_t>(static_cast<uint32_t>(__builtin_amdgcn_readlane(row, 16 * h))) * (D / 2);
        const uint8_t *k = a.k_codes + first, *v = a.v_codes + first;
        if constexpr (D == 128) {
          const uint4 w = *reinterpret_cast<const uint4 *>(k + k_lane);
          r.kw[h][0] = w.x, r.kw[h][1] = w.y, r.kw[h][2] = w.z, r.kw[h][3] = w.w;
        } else {
          const uint2 w = *reinterpret_cast<const uint2 *>(k + k_lane);
          r.kw[h][0] = w.x, r.kw[h][1] = w.y;
        }
        for (int e = 0; e < 4; ++e) r.vw[4 * h + e] = *reinterpret_cast<const uint32_t *>(v + (v_lane + e * (D / 2)));
      }
    } else {
      if (!r.ok) row = 0;
      s_rows[wave][lane & 31] = row;
      __builtin_amdgcn_wave_barrier();
      for (int h = 0; h < 2; ++h) {
        const uint8_t *k = a.k_codes + static_cast<size_t>(s_rows[wave][16 * h + n]) * (D / 2) + 4 * kKeyWords * j;
        if constexpr (D == 128) {
          const uint4 w = *reinterpret_cast<const uint4 *>(k);
          r.kw[h][0] = w.x, r.kw[h][1] = w.y, r.kw[h][2] = w.z, r.kw[h][3] = w.w;
        } else {
          const uint2 w = *reinterpret_cast<const uint2 *>(k);
          r.kw[h][0] = w.x, r.kw[h][1] = w.y;
        }
        for (int e = 0; e < 4; ++e)
          r.vw[4 * h + e] = *reinterpret_cast<const uint32_t *>(
              a.v_codes + static_cast<size_t>(s_rows[wave][16 * h + 4 * j + e]) * (D / 2) + 4 * (n & (D / 8 - 1)));
      }
      __builtin_amdgcn_wave_barrier();
    }
    r.sq = sq[row];
  };

  Round cur, next;
  const bool any = !idle && t0 + kRound * tw < t1;
  if (any) {
    look_up();
    request(cur);
    look_up();
  }

  int4_t qf[NT][WIDE ? kDigits : 1][kSteps];
  float alpha[NT], qsum[NT], ref[NT], sum[NT], off_sum[NT];
  int row_lo[NT], row_hi[NT];
  float4_t acc[NT][kTiles];
  for (int t = 0; t < NT; ++t) {
    const int row = row0 + 16 * t + n;
    const bool on = row < rows_valid;
    row_hi[t] = on ? g.last_pos(a, row) + 1 : 0;
    row_lo[t] = on ? g.first_pos(a, row) : 0;
    float x[kKeyWords][8];
    float top = 0.f;
    bool finite = true;
    for (int s = 0; s < kKeyWords; ++s) {
      for (int y = 0; y < (WIDE ? 2 : 1); ++y) {
        const uint32_t u[4] = {qraw[t][s][y].x, qraw[t][s][y].y, qraw[t][s][y].z, qraw[t][s][y].w};
        for (int e = 0; e < 4; ++e) {
          if constexpr (WIDE) {
            x[s][4 * y + e] = __uint_as_float(u[e]);
          } else {
            x[s][2 * e] = __uint_as_float(u[e] << 16);
            x[s][2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
          }
        }
      }
      for (int e = 0; e < 8; ++e) {
        finite = finite && fabsf(x[s][e]) < __builtin_inff();
        top = fmaxf(top, fabsf(x[s][e]));
      }
    }
    top = max_rows32(max_rows16(finite ? top : __builtin_inff()));
    const bool usable = top < __builtin_inff();
    // a row that is not finite: NaN logits, of what it attends
    if constexpr (WIDE) {
      const float lift = top < 0x1p-60f ? 0x1p60f : 1.f;  // kTopQ over a smaller magnitude may be no float
      const float to_fixed = usable && top > 0.f ? kTopQ / (top * lift) : 1.f;
      int total = 0;
      for (int s = 0; s < kSteps; ++s)
        for (int d = 0; d < kDigits; ++d) qf[t][d][s] = int4_t{0, 0, 0, 0};
      for (int s = 0; s < kKeyWords; ++s) {
        for (int e = 0; e < 8; ++e) {
          int f = usable ? static_cast<int>(rintf(x[s][e] * lift * to_fixed)) : 0;
          total += f;
          // byte e / 2 of the word of even (odd) coordinates of code word s; digits from the lowest, balanced
          for (int d = 0; d < kDigits; ++d) {
            const int digit = d == kDigits - 1 ? f : ((f + 128) & 255) - 128;
            f = (f - digit) >> 8;
            qf[t][d][s / 2][2 * (s % 2) + e % 2] |= (digit & 255) << (8 * (e / 2));
          }
        }
      }
      total += __shfl_xor(total, 16);
      total += __shfl_xor(total, 32);
      qsum[t] = usable ? static_cast<float>(total) * 0x1p-16f : __builtin_nanf("");
      alpha[t] = ldexpf(a.qscale / to_fixed, 16 + kKeyExp) / lift;
    } else {
      const int up = usable && top > 0.f ? min(13 - ilogbf(top), 120) : 0;
      const float unit = ldexpf(1.f, up);
      float total = 0.f;
      for (int s = 0; s < kKeyWords; ++s) {
        half8_t h;
        for (int e = 0; e < 8; ++e) {  // slots as value_pair has the nibbles: 0, 4, 1, 5, 2, 6, 3, 7
          h[2 * (e & 3) + (e >> 2)] = static_cast<_Float16>(usable ? x[s][e] * unit : __builtin_nanf(""));
          total += x[s][e] * unit;
        }
        qf[t][0][s] = __builtin_bit_cast(int4_t, h);
      }
      qsum[t] = add_rows32(add_rows16(total)) * 0x1p-9f;
      alpha[t] = ldexpf(a.qscale, 9 - up + kKeyExp);
    }
    alpha[t] = fminf(fmaxf(alpha[t], 0x1p-126f), 0x1p127f);  // finite: zero queries have logits of zero
    ref[t] = kNone;
    sum[t] = off_sum[t] = 0.f;
    for (int o = 0; o < kTiles; ++o) acc[t][o] = float4_t{0.f, 0.f, 0.f, 0.f};
  }

  for (int tb = t0 + kRound * tw; any && tb < t1; tb += kStep) {
    request(next);  // past the last round: rows at the pool's start or of a block's end, masked
    look_up();

    const uint32_t valid = static_cast<uint32_t>(__ballot(cur.ok));
    {
      float scale = __uint_as_float(cur.sq << 16), offset = __uint_as_float(cur.sq & 0xffff0000u);
      if (!WIDE || lane >= 32) offset = __builtin_fmaf(8.f, scale, offset);  // on the fp16 cores codes count from 8
      if (lane < 32) scale *= kKeyUnit, offset *= kKeyUnit;
      s_scale[wave][lane] = cur.ok ? scale : 0.f;
      s_offset[wave][lane] = cur.ok ? offset : 0.f;
      s_log[wave][lane] = __builtin_amdgcn_logf(fmaxf(fmaxf(fabsf(scale), fabsf(offset) * 0x1p-8f), 0x1p-70f));
    }
    __builtin_amdgcn_wave_barrier();
    // of the lane's 8 tokens, 4j + i and 16 + 4j + i, as its scores have them
    float ks[8], ko[8], vs[8], vo8[8];
    for (int h = 0; h < 2; ++h) {
      const float4 x[4] = {*reinterpret_cast<const float4 *>(&s_scale[wave][16 * h + 4 * j]),
                           *reinterpret_cast<const float4 *>(&s_offset[wave][16 * h + 4 * j]),
                           *reinterpret_cast<const float4 *>(&s_scale[wave][32 + 16 * h + 4 * j]),
                           *reinterpret_cast<const float4 *>(&s_offset[wave][32 + 16 * h + 4 * j])};
      float *to[4] = {ks, ko, vs, vo8};
      for (int y = 0; y < 4; ++y)
        to[y][4 * h] = x[y].x, to[y][4 * h + 1] = x[y].y, to[y][4 * h + 2] = x[y].z, to[y][4 * h + 3] = x[y].w;
    }
    __builtin_amdgcn_wave_barrier();

    const bool inner = valid == 0xffffffffu && tb >= inner_lo && tb + kRound <= inner_hi;
    float dots[NT][8];  // query times codes, of the lane's tokens
    if constexpr (WIDE) {
      int4_t kc[2][kSteps];  // the keys' codes in bytes: even coordinates of a word, then odd ones
      for (int h = 0; h < 2; ++h)
        for (int s = 0; s < kKeyWords; ++s) {
          kc[h][s / 2][2 * (s % 2)] = static_cast<int>(cur.kw[h][s] & 0x0f0f0f0fu);
          kc[h][s / 2][2 * (s % 2) + 1] = static_cast<int>((cur.kw[h][s] >> 4) & 0x0f0f0f0fu);
        }
      for (int t = 0; t < NT; ++t)
        for (int h = 0; h < 2; ++h) {
          int4_t d[kDigits];
          for (int x = 0; x < kDigits; ++x) {
            d[x] = int4_t{0, 0, 0, 0};
            for (int s = 0; s < kSteps; ++s) d[x] = __builtin_amdgcn_mfma_i32_16x16x64_i8(kc[h][s], qf[t][x][s], d[x], 0, 0, 0);
          }
          for (int i = 0; i < 4; ++i)
            dots[t][4 * h + i] = __builtin_fmaf(0x1p-16f, static_cast<float>((d[1][i] << 8) + d[0][i]), static_cast<float>(d[2][i]));
        }
    } else {
      for (int h = 0; h < 2; ++h) {
        float4_t d[NT];
        for (int t = 0; t < NT; ++t) d[t] = float4_t{0.f, 0.f, 0.f, 0.f};
        for (int s = 0; s < kSteps; ++s) {
          const uint32_t w = cur.kw[h][s];
          const half8_t c = __builtin_bit_cast(half8_t, make_uint4(value_pair<0>(w), value_pair<1>(w), value_pair<2>(w), value_pair<3>(w)));
          for (int t = 0; t < NT; ++t)
            d[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(c, __builtin_bit_cast(half8_t, qf[t][0][s]), d[t], 0, 0, 0);
          if (s % 2) __builtin_amdgcn_sched_barrier(0);  // the others stay packed until here: unpacked together they spill, 453 us
        }
        for (int t = 0; t < NT; ++t)
          for (int i = 0; i < 4; ++i) dots[t][4 * h + i] = d[t][i];
      }
    }
    half8_t pf[NT][kProbParts];
    for (int t = 0; t < NT; ++t) {
      float z[8], bound = kNone, scale[8], offset[8];
      for (int e = 0; e < 8; ++e) {
        z[e] = ks[e] * dots[t][e] + ko[e] * qsum[t];
        scale[e] = vs[e];
        offset[e] = vo8[e];
      }
      if (!inner) {  // without branches in it, inner rounds copy nothing
        for (int e = 0; e < 8; ++e) {
          const int m = 16 * (e >> 2) + 4 * j + (e & 3);
          const bool seen = ((valid >> m) & 1u) & (tb + m >= row_lo[t]) & (tb + m < row_hi[t]);
          z[e] = seen ? z[e] : kNone;
          scale[e] = seen ? scale[e] : 0.f;  // whatever a hidden token's scale and offset are
          offset[e] = seen ? offset[e] : 0.f;
        }
      }
      for (int e = 0; e < 8; ++e)
        bound = fmaxf(bound, __builtin_fmaf(z[e], alpha[t], s_log[wave][32 + 16 * (e >> 2) + 4 * j + (e & 3)]));
      if (__any(bound > ref[t] + (kTop + kSlack))) {
        const float most = max_rows32(max_rows16(bound));
        const float next = fmaxf(ref[t], most - kTop);
        const float f = next == kNone ? 1.f : half_factor(ref[t] - next);
        ref[t] = next;
        for (int y = 0; y < 2; ++y) {
          sum[t] *= f;
          off_sum[t] *= f;
          for (int o = 0; o < kTiles; ++o) acc[t][o] *= f;
        }
      }
      const float r = ref[t] == kNone ? 0.f : ref[t];
      for (int e = 0; e < 8; ++e) {
        const float p = exp2_raw(__builtin_fmaf(z[e], alpha[t], -r));
        const float ps = p * scale[e];
        sum[t] += p;
        off_sum[t] += p * offset[e];
        if constexpr (WIDE) {  // units of 1, units of 2^-11, what is left
          const float high = rintf(ps), rest = ps - high, mid = rintf(rest * 0x1p11f) * 0x1p-11f;
          pf[t][0][e] = static_cast<_Float16>(high);
          pf[t][1][e] = static_cast<_Float16>(mid);
          pf[t][2][e] = static_cast<_Float16>(rest - mid);
        } else {
          pf[t][0][e] = static_cast<_Float16>(ps);
        }
      }
    }

    __builtin_amdgcn_sched_barrier(0);  // the codes of values stay packed until here
    // The same coordinate's codes of two tokens in one word: the low half of the
    // tokens' words, then the high one (head_dim 64: lanes 0..7 of a row take the
    // low one, lanes 8..15 the high one).
    auto values = [&](auto k, const int o, const uint32_t *pair) {
      const half8_t c = __builtin_bit_cast(half8_t, make_uint4(value_pair<k()>(pair[0]), value_pair<k()>(pair[1]),
                                                               value_pair<k()>(pair[2]), value_pair<k()>(pair[3])));
      for (int t = 0; t < NT; ++t)
        for (int x = 0; x < kProbParts; ++x)
          acc[t][o] = __builtin_amdgcn_mfma_f32_16x16x32_f16(c, pf[t][x], acc[t][o], 0, 0, 0);
    };
    for (int half = 0; half < D / 64; ++half) {
      const uint32_t pick = D == 128 ? (half ? 0x07060302u : 0x05040100u) : n < 8 ? 0x05040100u : 0x07060302u;
      uint32_t pair[4];
      for (int e = 0; e < 4; ++e) pair[e] = __builtin_amdgcn_perm(cur.vw[2 * e + 1], cur.vw[2 * e], pick);
      values(std::integral_constant<int, 0>{}, 4 * half, pair);
      values(std::integral_constant<int, 1>{}, 4 * half + 1, pair);
      values(std::integral_constant<int, 2>{}, 4 * half + 2, pair);
      values(std::integral_constant<int, 3>{}, 4 * half + 3, pair);
    }
    cur = next;
  }

  // the wave's partials
  for (int t = 0; t < NT; ++t) {
    sum[t] = add_rows32(add_rows16(sum[t]));
    off_sum[t] = add_rows32(add_rows16(off_sum[t]));
    if (sum[t] != sum[t]) ref[t] = fmaxf(ref[t], 0.f);  // NaN logits move no reference, but attend
    for (int o = 0; o < kTiles; ++o)
      for (int i = 0; i < 4; ++i) acc[t][o][i] = acc[t][o][i] * 0x1p9f + off_sum[t];
  }
  finish_rows<D, NT, W, TILED>(a, g, {s_merge, s_ref, s_sum, s_inv, &s_last}, wave, lane, acc, ref, sum);
}

int most_splits(const int tile_rows, const long long tiles, const long long span) {
  const long long limit = tile_rows >= 128 ? kMaxSplitsTiled : kMaxSplits;
  return static_cast<int>(std::max<long long>(1, std::min({limit, (span + 127) / 128, kMaxCounters / tiles})));
}

}  // namespace

// Rows per workgroup: up to 16 (32) rows take one (two) matrix tiles, the
// workgroup's waves dividing the tokens; more rows take 32 a wave, 128 or 256 a
// workgroup (fp32: 16 and 128, which leaves registers for two waves a SIMD: 2 x 2048
// over 8192 tokens 1504 us, 8 x 16 over 4096 61 us; 32 a wave took 1.2 and 1.5 times as long).
Q4AttnPlan plan_q4_attn(const int batch, const int n_q, const int num_q_heads, const int num_kv_heads,
                        const int head_dim, const int q_bf16, const int max_seq_len, const int window) {
  Q4AttnPlan p{};
  const int gqa = num_q_heads / num_kv_heads;
  const long long rows = static_cast<long long>(n_q) * gqa;
  auto tiles_of = [&](const int tile_rows) { return (rows + tile_rows - 1) / tile_rows * batch * num_kv_heads; };
  // A launch takes rounds of the workgroups that the CUs hold, each its setup
  // and tail beside its tokens; splits add the merge, by rows. Fitted to sweeps
  // over both (8 KV heads of 128, bf16, us): one sequence of 128K tokens 36.2 in
  // 32 splits of 12 waves, 38.6 in 64 of 4 waves, 46.2 in 32 of 4; of 2000 tokens
  // 15.2 in 3 of 12, 10.4 in 16 of 4; 32 x 8192 55.6 whole by 12 waves, 57.2 in 3 of
  // 4; 64 x 500 12.8 whole by 4 waves, 19.5 by 12; 64 queries over 32K tokens 137 in 16
  // splits of 128 rows, 158 of 256; 8 x 64 over 2000 tokens 82 in tiles of 128, 102 of
  // 256; 2 x 2048 over 8192 tokens 620 in tiles of 128, 525 of 256.
  const double size = head_dim == 128 ? 1.0 : 0.75;
  // token[k - 1]: ns of a CU for a token where k workgroups share it
  auto consider = [&](const int tile_rows, const int waves, const int step, const int setup,
                      const std::initializer_list<double> token, const int split, const double merge) {
    const long long tiles = tiles_of(tile_rows), queries = std::min(n_q, tile_rows / gqa + 1);  // of a tile
    const long long span = window > 0 ? std::min<long long>(max_seq_len, window + queries) : max_seq_len;
    const double row_ns = static_cast<double>(std::min<long long>(rows, tile_rows));
    const int per_cu = static_cast<int>(token.size());
    for (int n = 1; n <= most_splits(tile_rows, tiles, span); ++n) {
      const long long chunk = ((span + n - 1) / n + step - 1) / step * step;
      const long long groups = tiles * n, rounds = (groups + 256 * per_cu - 1) / (256 * per_cu);
      const int share = static_cast<int>(std::min<long long>(per_cu, (groups + 255) / 256));
      const double each = chunk * size * token.begin()[share - 1] * share;
      const double words = groups * row_ns * (head_dim + 2);  // of the partials, 1.2 TB/s
      const double cost = rounds * (setup + each) + (n > 1 ? split + merge * row_ns * n + words / 300 : 0);
      if (p.waves == 0 || cost < p.cost) p.cost = cost, p.waves = waves, p.n_split = n, p.tile_rows = tile_rows;
    }
  };
  const int most_rows = rows <= 16 ? 16 : rows <= 32 ? 32 : 256;
  if (rows > 32 && q_bf16) {
    consider(128, 4, 64, 10000, {29, 23}, 10000, 19);
    if (rows <= 128) consider(256, 8, 128, 10000, {27}, 10000, 19);  // half of the waves have no rows, and unpack only
    else consider(256, 8, 128, 12000, {42}, 10000, 19);
  } else if (rows > 32) {
    consider(128, 8, kRound, 10000, {51}, 10000, 19);
  } else if (rows > 16) {
    consider(32, 4, 4 * kRound, 10000, {13}, 3500, 10);
    consider(32, 8, 8 * kRound, 10000, {8.5}, 3500, 10);
  } else if (q_bf16) {
    consider(16, 4, 4 * kRound, 6500, {9, 6.2, 5.7}, 3500, 10);
    consider(16, 12, 12 * kRound, 7000, {5.8}, 3500, 5);
  } else {
    consider(16, 4, 4 * kRound, 6500, {9.9, 8}, 3500, 10);
    consider(16, 8, 8 * kRound, 7000, {7.5}, 3500, 5);
  }
  p.row_tiles = static_cast<int>((rows + p.tile_rows - 1) / p.tile_rows);
  // The counters of all shapes lie at the workspace's start; its size covers
  // every window, type and tile (tiles of 256 rows need no less than ones of 128).
  const long long tiles = tiles_of(most_rows);
  const int most = most_splits(most_rows, tiles, max_seq_len);
  p.off_part = kMaxCounters * sizeof(int);
  if (most > 1) {
    const size_t part = static_cast<size_t>(tiles) * most * most_rows * (head_dim + 2) * sizeof(float);
    p.total = p.off_part + ((part + 255) & ~static_cast<size_t>(255));
  }
  return p;
}

hipError_t launch_q4_attn(const Q4AttnArgs &a, const Q4AttnPlan &plan, hipStream_t stream) {
  const unsigned tiles = static_cast<unsigned>(a.batch) * a.num_kv_heads * a.row_tiles;
  auto go = [&](auto d, auto wide, auto nt, auto w, auto tiled) {
    // blocks of a multiple of 16 rows: a round needs two addresses instead of ten a lane
    if (a.layout.block_size % 16 == 0)
      q4_attn_kernel<d(), wide(), nt(), w(), tiled(), true><<<tiles * a.n_split, 64 * w(), 0, stream>>>(a);
    else
      q4_attn_kernel<d(), wide(), nt(), w(), tiled(), false><<<tiles * a.n_split, 64 * w(), 0, stream>>>(a);
    return hipGetLastError();
  };
  if (a.q_bf16 && plan.tile_rows >= 128) return launch_q4_tile(a, plan, stream);
  using std::false_type;
  using std::integral_constant;
  using std::true_type;
  constexpr integral_constant<int, 1> one{};
  constexpr integral_constant<int, 2> two{};
  constexpr integral_constant<int, 4> w4{};
  constexpr integral_constant<int, 8> w8{};
  constexpr integral_constant<int, 12> w12{};
  auto by_rows = [&](auto d, auto wide) {
    if constexpr (wide())
      if (plan.tile_rows == 128) return go(d, wide, one, w8, true_type{});
    if (plan.tile_rows == 32) return plan.waves == 4 ? go(d, wide, two, w4, false_type{}) : go(d, wide, two, w8, false_type{});
    if (plan.waves == 4) return go(d, wide, one, w4, false_type{});
    if constexpr (wide()) return go(d, wide, one, w8, false_type{});
    else return go(d, wide, one, w12, false_type{});
  };
  auto by_type = [&](auto d) { return a.q_bf16 ? by_rows(d, false_type{}) : by_rows(d, true_type{}); };
  return a.head_dim == 128 ? by_type(integral_constant<int, 128>{}) : by_type(integral_constant<int, 64>{});
}

}  // namespace novakv
