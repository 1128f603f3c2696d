// Attention of 33 to 128 query rows per KV head over the 2-bit cache (nova_kv_chunk_attn: short chunks of prompts).
//
// A workgroup of eight waves takes 128 rows, 16 a wave, and 32 or 64 tokens a round. The waves
// gather the tokens' codewords once, between them, from the codebooks in LDS to fragments
// in LDS, in the order in which the matrix cores take them: a key's pairs of groups as they
// come, values transposed in registers, two tokens at a time. Both codebooks of head_dim 128 leave
// 32 KiB beside them, so keys and values have one buffer each, used and filled in turn: while a
// round's scores are made its values are gathered, while its weights meet the values the next
// round's keys are.
//
// Tiles of 256 rows (chunk_wide.hip) for such calls leave half of their waves idle: 32 queries of 4 heads over 16384
// tokens 101 us here, 240 there; over 8192 tokens of 16 sequences 220 in both. Far from the matrix cores' 7 and 58 us:
// 25 us are a workgroup's setup (over 64 tokens), whose transforms come in element by element, and a round of
// 32 tokens has two barriers. Parts of queries and probabilities: as in chunk_rows.hip.
//
// Queries go through R_K^-T and sums back through R_V on the matrix cores, without leaving the
// wave: the transform's rows are dealt to the tiles so that a lane's results are its next operand.
#include <type_traits>

#include "chunk_common.h"

namespace novakv {

namespace {

using namespace chunk;

constexpr int kWaves = 8, kThreads = 64 * kWaves;
constexpr int NT = 1;  // tiles of 16 rows a wave

template <int D, bool SQ>
struct Lds {
  static constexpr int kTiles = D / 16, kSteps = D / 32;
  static constexpr int kHalves = D == 128 && !SQ ? 1 : 2;  // 32 tokens each of a round
  static constexpr int kTokens = 32 * kHalves, kRuns = 2 * kHalves;  // runs of 16 tokens
  static constexpr int kKeyFrags = kRuns * kSteps, kValueFrags = kHalves * kTiles;
  static constexpr int kBook = D / kGroupDim * kCodebookSize * 8;
  static constexpr int kKeys = (SQ ? 1 : 2) * kBook;                // [run + kRuns * step][lane] 16 bytes
  static constexpr int kValues = kKeys + kKeyFrags * 1024;          // [half * kTiles + tile][lane]
  static constexpr int kTok = kValues + kValueFrags * 1024;         // [round mod 2][rho, scale, offset, exponent][kTokens] fp32
  static constexpr int kLoopEnd = kTok + 2 * 4 * kTokens * 4;
  // in front of and behind the loop: a transform's parts [tile][step][hi, lo][lane] 16 bytes; the splits' merge
  using Finish = q4::FinishLds<D, NT, kWaves, true>;
  static constexpr int kFrags = kTiles * kSteps * 2 * 1024, kMerge = Finish::kMerge * 4;
  static constexpr int kOther = kFrags > kMerge ? kFrags : kMerge;
  static constexpr int kInv = kLoopEnd > kOther ? kLoopEnd : kOther;  // [row] fp32
  static constexpr int kTops = kInv + Finish::kRows * 4;              // [wave]
  static constexpr int kLast = kTops + kWaves * 4;
  static constexpr int kBytes = kLast + 16;
  static_assert(kBytes <= 160 * 1024, "LDS of a workgroup");
  static_assert(kKeyFrags % kWaves == 0 && kRuns * 2 * (kTiles / 4) % kWaves == 0, "the waves share the gathers evenly");
};

// A transform's parts in LDS: each wave makes a tile of them. element(o, m, k): the element that
// tile o's row m has in slot k of the contraction's D; returns the exponent of their scale.
template <int D, typename F>
__device__ __forceinline__ int stage_transform(half8_t *to, float *tops, const int wave, const int lane, F element) {
  constexpr int kTiles = D / 16, kSteps = D / 32;
  float raw[kSteps][8], top = 0.f;
  if (wave < kTiles)
    for (int s = 0; s < kSteps; ++s)
      for (int e = 0; e < 8; ++e) {
        raw[s][e] = element(wave, lane & 15, 32 * s + 8 * (lane >> 4) + e);
        top = fmaxf(top, fabsf(raw[s][e]));
      }
  top = wave_max(top);
  if (lane == 0) tops[wave] = top;
  __syncthreads();
  for (int u = 0; u < kWaves; ++u) top = fmaxf(top, tops[u]);
  const int up = up_to_14(top);
  if (wave < kTiles)
    for (int s = 0; s < kSteps; ++s) {
      half8_t h, l;
      for (int e = 0; e < 8; ++e) {
        _Float16 hi, lo;
        split_half(ldexpf(raw[s][e], up), hi, lo);
        h[e] = hi, l[e] = lo;
      }
      to[((wave * kSteps + s) * 2) * 64 + lane] = h;
      to[((wave * kSteps + s) * 2 + 1) * 64 + lane] = l;
    }
  __syncthreads();
  return up;
}

// A row tile times a staged transform, x in two parts (LOW) or one.
template <int D, bool LOW>
__device__ __forceinline__ void transform_rows(const half8_t *t, const int lane, const half8_t (&xh)[D / 32], const half8_t (&xl)[D / 32],
                                               float4_t (&out)[D / 16]) {
  constexpr int kTiles = D / 16, kSteps = D / 32;
  for (int o = 0; o < kTiles; ++o) {
    out[o] = float4_t{0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < kSteps; ++s) {
      const half8_t h = t[((o * kSteps + s) * 2) * 64 + lane], l = t[((o * kSteps + s) * 2 + 1) * 64 + lane];
      out[o] = __builtin_amdgcn_mfma_f32_16x16x32_f16(h, xh[s], out[o], 0, 0, 0);
      out[o] = __builtin_amdgcn_mfma_f32_16x16x32_f16(l, xh[s], out[o], 0, 0, 0);
      if constexpr (LOW) out[o] = __builtin_amdgcn_mfma_f32_16x16x32_f16(h, xl[s], out[o], 0, 0, 0);
    }
  }
}

// D: head_dim. WIDE: fp32 queries. SQ: the scalar value arm. KS: key scales.
// ALIGNED: blocks of a multiple of 16 rows.
template <int D, bool WIDE, bool SQ, bool KS, bool ALIGNED>
__global__ __launch_bounds__(kThreads, 2) void chunk_tile_kernel(const ChunkArgs a) {
  using M = Lds<D, SQ>;
  constexpr int kParts = WIDE ? 2 : 1, L = D / kGroupDim, kSteps = M::kSteps, kTiles = M::kTiles;
  constexpr int kHalves = M::kHalves, kTokens = M::kTokens, kRuns = M::kRuns;
  constexpr int kKeyUnits = M::kKeyFrags / kWaves, kValueUnits = kRuns * 2 * (kTiles / 4) / kWaves;
  __shared__ __align__(16) uint8_t s_lds[M::kBytes];
  uint2 *const s_key_book = reinterpret_cast<uint2 *>(s_lds), *const s_value_book = s_key_book + L * kCodebookSize;
  half8_t *const s_keys = reinterpret_cast<half8_t *>(s_lds + M::kKeys), *const s_values = reinterpret_cast<half8_t *>(s_lds + M::kValues);
  float *const s_tok = reinterpret_cast<float *>(s_lds + M::kTok), *const s_tops = reinterpret_cast<float *>(s_lds + M::kTops);
  half8_t *const s_frags = reinterpret_cast<half8_t *>(s_lds);

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int lane = threadIdx.x & 63, n = lane & 15, j = lane >> 4;
  Tile g;
  q4::place_tile(a, M::Finish::kRows, g);
  if (!q4::find_span(a, M::Finish::kRows, kTokens, g)) return;
  const int b = g.b, kv = g.kv;
  const Spans span(a, g);
  const int c0 = span.c0, c1 = span.c1;
  // this wave's rows
  const int row0 = g.row0 + 16 * NT * wave, row1 = min(row0 + 16 * NT, g.rows_valid);
  const bool idle = row0 >= g.rows_valid;
  const int wave_lo = idle ? 0 : g.first_pos(a, row0), wave_hi = idle ? 0 : g.last_pos(a, row1 - 1) + 1;
  const int inner_lo = idle ? 0 : g.first_pos(a, row1 - 1), inner_hi = idle ? 0 : g.last_pos(a, row0) + 1;
  int row_lo[NT], row_hi[NT];
  size_t q_at[NT];
  for (int t = 0; t < NT; ++t) {
    const int row = row0 + 16 * t + n;
    const bool on = row < g.rows_valid;
    const int i = row / a.gqa, h = row - i * a.gqa;
    row_hi[t] = on ? g.last_pos(a, row) + 1 : 0;
    row_lo[t] = on ? g.first_pos(a, row) : 0;
    q_at[t] = on ? ((static_cast<size_t>(b) * a.n_q + i) * a.num_q_heads + kv * a.gqa + h) * D + 8 * j : ~static_cast<size_t>(0);
  }
  auto load_row = [&](const int t, float (&x)[kSteps][8]) {
    for (int s = 0; s < kSteps; ++s)
      for (int e = 0; e < 8; ++e) x[s][e] = 0.f;
    if (q_at[t] != ~static_cast<size_t>(0))
      for (int s = 0; s < kSteps; ++s) load_query<WIDE>(a.q, q_at[t] + 32 * s, x[s]);
  };

  Sums<D, NT> y;
  y.clear();
  if (span.codes) {
    // ---- q' = q R_K^-T. Tile o's row m is coordinate (D / 4) (m / 4) + 4 o + m % 4, so that a lane's results
    // are its coordinates (D / 4) j + 8 s + e of the score's steps.
    const void *tk = transform_of(a.t_k_inv_t, kv, D, a.t_bf16);
    const int up_t = stage_transform<D>(s_frags, s_tops, wave, lane, [&](const int o, const int m, const int k) {
      return t1_value(tk, static_cast<size_t>(k) * D + (D / 4) * (m >> 2) + 4 * o + (m & 3), a.t_bf16);
    });
    half8_t qf[NT][kSteps][kParts];
    float alpha[NT], shift[NT];
    for (int t = 0; t < NT; ++t) {
      float x[kSteps][8];
      load_row(t, x);
      float top = 0.f, dot = 0.f;
      bool finite = true;
      for (int s = 0; s < kSteps; ++s)
        for (int e = 0; e < 8; ++e) {
          finite = finite && fabsf(x[s][e]) < __builtin_inff();
          top = fmaxf(top, fabsf(x[s][e]));
          dot = __builtin_fmaf(x[s][e], a.kbar[kv * D + 32 * s + 8 * j + e], dot);
        }
      shift[t] = add_rows32(add_rows16(dot)) * a.qscale;
      top = max_rows32(max_rows16(finite ? top : __builtin_inff()));
      const bool usable = top < __builtin_inff();
      const int up = up_to_14(top);
      half8_t xh[kSteps], xl[kSteps];
      for (int s = 0; s < kSteps; ++s)
        for (int e = 0; e < 8; ++e) {
          _Float16 hi, lo;
          split_half(usable ? ldexpf(x[s][e], up) : __builtin_nanf(""), hi, lo);  // a row that is not finite: NaN scores
          xh[s][e] = hi, xl[s][e] = lo;
        }
      float4_t out[kTiles];
      transform_rows<D, WIDE>(s_frags, lane, xh, xl, out);
      // |out| <= D 2^28: times 2^-20 it fits fp16
      for (int s = 0; s < kSteps; ++s)
        for (int e = 0; e < 8; ++e) {
          _Float16 hi, lo;
          split_half(out[2 * s + (e >> 2)][e & 3] * 0x1p-20f, hi, lo);
          qf[t][s][0][e] = hi;
          if constexpr (WIDE) qf[t][s][1][e] = lo;
        }
      alpha[t] = fminf(fmaxf(ldexpf(a.qscale, 20 - up - up_t), 0x1p-126f), 0x1p126f);
    }
    __syncthreads();
    stage_book<L, kThreads>(s_key_book, a.cb_k, a.cb_fp8, kv);
    if constexpr (!SQ) stage_book<L, kThreads>(s_value_book, a.cb_v, a.cb_fp8, kv);

    // ---- this wave's share of the gathers: run `run` of a round's 16-token runs; of its keys, steps
    // key_step + .. ; of its values, two of each four tokens, from 2 twin on
    const int run = wave % kRuns, key_step = wave / kRuns, twin = (wave / kRuns) & 1;
    const int bs = a.layout.block_size;
    const int bs_log = (bs & (bs - 1)) == 0 ? 31 - __builtin_clz(bs) : -1;
    const int32_t *table = a.layout.block_table ? a.layout.block_table + static_cast<size_t>(b) * a.layout.blocks_per_seq : nullptr;
    const long long first_block = static_cast<long long>(b) * a.layout.blocks_per_seq;
    // Where a token's rows lie: [0] the run's first (ALIGNED), or the lane's key, then its two values.
    constexpr int kPlaces = ALIGNED ? 1 : 3;
    struct Look {
      int phys[kPlaces], row[kPlaces];
    };
    int look_tb = c0 & ~31;
    auto look_up = [&](Look &k) {
      // nothing outside the attended tokens' own runs of 16 (elsewhere: tokens) is looked up
      auto find = [&](const int i, const int tok) {
        const int blk = bs_log >= 0 ? tok >> bs_log : tok / bs;
        k.row[i] = tok - blk * bs;
        k.phys[i] = table ? table[blk] : static_cast<int>(first_block + blk);
      };
      const int first = look_tb + 16 * run;
      if constexpr (ALIGNED) {
        find(0, __builtin_amdgcn_readfirstlane(min(max(first, c0 & ~15), (c1 - 1) & ~15)));
      } else {
        auto inside = [&](const int tok) { return min(max(tok, c0), c1 - 1); };
        find(0, inside(first + n));
        find(1, inside(first + 4 * j + 2 * twin));
        find(2, inside(first + 4 * j + 2 * twin + 1));
      }
      look_tb += kTokens;
    };
    auto row_at = [&](const Look &k, const int i) {  // i: 0 the lane's key, 1 and 2 its values
      const int p = ALIGNED ? 0 : i;
      const size_t row = (static_cast<size_t>(k.phys[p]) * a.num_kv_heads + kv) * bs + k.row[p];
      return ALIGNED ? row + (i == 0 ? n : 4 * j + 2 * twin + i - 1) : row;
    };
    struct KeyCodes {
      uint16_t code[kKeyUnits], rho;
      uint32_t sq;
    };
    struct ValueCodes {
      uint8_t code[kValueUnits][2];
    };
    auto request_keys = [&](const Look &k, KeyCodes &c) {
      const size_t row = row_at(k, 0);
      for (int u = 0; u < kKeyUnits; ++u)
        c.code[u] = *reinterpret_cast<const uint16_t *>(a.k_codes + row * L + (L / 4) * j + 2 * (key_step + u * (kWaves / kRuns)));
      c.rho = 0, c.sq = 0;
      if (wave < kRuns) {
        if constexpr (KS) c.rho = a.k_scales[row];
        if constexpr (SQ) c.sq = reinterpret_cast<const uint32_t *>(a.v_sq)[row];
      }
    };
    auto request_values = [&](const Look &k, ValueCodes &c) {
      for (int u = 0; u < kValueUnits; ++u) {
        const int p = (wave / kRuns + u * (kWaves / kRuns)) >> 1;
        for (int e = 0; e < 2; ++e) c.code[u][e] = a.v_codes[row_at(k, 1 + e) * L + value_group<D>(n, p)];
      }
    };
    auto put_keys = [&](const KeyCodes &c, const int tb, const int parity) {
      for (int u = 0; u < kKeyUnits; ++u) {
        const int st = key_step + u * (kWaves / kRuns);
        const uint2 *book = s_key_book + ((L / 4) * j + 2 * st) * kCodebookSize;
        const uint2 w0 = book[c.code[u] & 0xffu], w1 = book[kCodebookSize + (c.code[u] >> 8)];
        s_keys[(run + kRuns * st) * 64 + lane] = __builtin_bit_cast(half8_t, make_uint4(w0.x, w0.y, w1.x, w1.y));
      }
      if constexpr (KS || SQ) {
        if (wave < kRuns && lane < 16) {
          const int tok = tb + 16 * run + lane;
          float *to = s_tok + parity * 4 * kTokens + 16 * run + lane;
          float rho = KS ? bf16_bits_to_float(c.rho) : 1.f;
          if constexpr (SQ) {
            const Grid v = grid_of(c.sq, tok >= c0 && tok < c1, rho);
            to[kTokens] = v.scale, to[2 * kTokens] = v.offset, to[3 * kTokens] = v.expo;
          }
          to[0] = rho;
        }
      }
    };
    auto put_values = [&](const ValueCodes &c) {
      for (int u = 0; u < kValueUnits; ++u) {
        const int p = (wave / kRuns + u * (kWaves / kRuns)) >> 1;
        uint2 w[2];
        for (int e = 0; e < 2; ++e) {
          if constexpr (SQ) w[e] = centred_levels(c.code[u][e]);
          else w[e] = s_value_book[value_group<D>(n, p) * kCodebookSize + c.code[u][e]];
        }
        uint32_t *to = reinterpret_cast<uint32_t *>(s_values + ((run >> 1) * kTiles + 4 * p) * 64 + lane) + 2 * (run & 1) + twin;
        for (int x = 0; x < 4; ++x) to[x * 256] = x < 2 ? half_pair(w[0].x, w[1].x, x & 1) : half_pair(w[0].y, w[1].y, x & 1);
      }
    };

    Look here, ahead, next;
    KeyCodes keys;
    ValueCodes values;
    look_up(here);
    look_up(ahead);
    request_keys(here, keys);
    request_values(here, values);
    look_up(next);
    __syncthreads();  // the codebooks are there
    put_keys(keys, c0 & ~31, 0);
    request_keys(ahead, keys);
    __syncthreads();
    for (int tb = c0 & ~31, parity = 0; tb < c1; tb += kTokens, parity ^= 1) {
      const bool mine = !idle && tb < wave_hi && tb + kTokens > wave_lo;
      float4_t s[NT][kRuns];
      if (mine) {
        for (int x = 0; x < kRuns; ++x) {
          for (int t = 0; t < NT; ++t) s[t][x] = float4_t{0.f, 0.f, 0.f, 0.f};
          for (int st = 0; st < kSteps; ++st) {
            const half8_t k = s_keys[(x + kRuns * st) * 64 + lane];
            for (int t = 0; t < NT; ++t)
              for (int p = 0; p < kParts; ++p) s[t][x] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, qf[t][st][p], s[t][x], 0, 0, 0);
          }
        }
      }
      put_values(values);
      request_values(ahead, values);
      __syncthreads();
      put_keys(keys, tb + kTokens, parity ^ 1);  // past the end: the last tokens again
      request_keys(next, keys);
      ahead = next;
      look_up(next);
      if (mine) {
        const float *tok = s_tok + parity * 4 * kTokens + 4 * j;
        if constexpr (KS || SQ) {
          for (int x = 0; x < kRuns; ++x) {
            const float4 rho = *reinterpret_cast<const float4 *>(tok + 16 * x);
            for (int t = 0; t < NT; ++t) s[t][x][0] *= rho.x, s[t][x][1] *= rho.y, s[t][x][2] *= rho.z, s[t][x][3] *= rho.w;
          }
        }
        if (!(tb >= max(inner_lo, c0) && tb + kTokens <= min(inner_hi, c1))) {
          for (int t = 0; t < NT; ++t)
            for (int x = 0; x < kRuns; ++x)
              for (int i = 0; i < 4; ++i) {
                const int m = tb + 16 * x + 4 * j + i;
                const bool seen = static_cast<int>(m >= max(c0, row_lo[t])) & static_cast<int>(m < min(c1, row_hi[t]));
                s[t][x][i] = seen ? s[t][x][i] : kNone;
              }
        }
        float bound[NT];
        for (int t = 0; t < NT; ++t) {
          bound[t] = kNone;
          for (int x = 0; x < kRuns; ++x)
            for (int i = 0; i < 4; ++i) {
              if constexpr (SQ) bound[t] = fmaxf(bound[t], __builtin_fmaf(s[t][x][i], alpha[t], tok[3 * kTokens + 16 * x + i]));
              else bound[t] = fmaxf(bound[t], s[t][x][i]);
            }
          if constexpr (!SQ) bound[t] *= alpha[t];
        }
        y.raise(bound);
        half8_t pf[NT][kHalves][kParts];
        for (int t = 0; t < NT; ++t) {
          const float r = y.ref[t] == kNone ? 0.f : y.ref[t];
          for (int x = 0; x < kRuns; ++x)
            for (int i = 0; i < 4; ++i) {
              float p = exp2_raw(__builtin_fmaf(s[t][x][i], alpha[t], -r));
              y.sum[t] += p;
              if constexpr (SQ) {
                y.off_sum[t] = __builtin_fmaf(p, tok[2 * kTokens + 16 * x + i], y.off_sum[t]);
                p *= tok[kTokens + 16 * x + i];
              }
              const int e = 4 * (x & 1) + i;
              if constexpr (WIDE) {
                _Float16 hi, lo;
                split_half(p, hi, lo);
                pf[t][x >> 1][0][e] = hi, pf[t][x >> 1][1][e] = lo;
              } else {
                pf[t][x >> 1][0][e] = static_cast<_Float16>(p);
              }
            }
        }
        for (int h = 0; h < kHalves; ++h)
          for (int o = 0; o < kTiles; ++o) {
            const half8_t v = s_values[(h * kTiles + o) * 64 + lane];
            for (int t = 0; t < NT; ++t)
              for (int p = 0; p < kParts; ++p) y.acc[t][o] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, pf[t][h][p], y.acc[t][o], 0, 0, 0);
          }
      }
      __syncthreads();
    }

    // ---- back through R_V: tile o's row m is coordinate q4::out_coord
    const void *tv = transform_of(a.t_v, kv, D, a.t_bf16);
    const int up_v = stage_transform<D>(s_frags, s_tops, wave, lane, [&](const int o, const int m, const int k) {
      const int e = k & 7, jj = (k >> 3) & 3, h = k >> 5;
      return t1_value(tv, static_cast<size_t>(q4::out_coord<D>(o, m & 3, m >> 2)) * D + code_coord<D>(2 * h + (e >> 2), 4 * jj + (e & 3)),
                      a.t_bf16);
    });
    for (int t = 0; t < NT; ++t) {
      if constexpr (SQ) {
        const float off = add_rows32(add_rows16(y.off_sum[t]));
        for (int o = 0; o < kTiles; ++o) y.acc[t][o] += off;
        y.off_sum[t] = 0.f;
      }
      float top = 0.f;
      for (int o = 0; o < kTiles; ++o)
        for (int i = 0; i < 4; ++i) top = fmaxf(top, fabsf(y.acc[t][o][i]));
      const int up = up_to_14(max_rows32(max_rows16(top)));
      half8_t xh[kSteps], xl[kSteps];
      for (int s = 0; s < kSteps; ++s)
        for (int e = 0; e < 8; ++e) {
          _Float16 hi, lo;
          split_half(ldexpf(y.acc[t][2 * s + (e >> 2)][e & 3], up), hi, lo);
          xh[s][e] = hi, xl[s][e] = lo;
        }
      transform_rows<D, true>(s_frags, lane, xh, xl, y.acc[t]);
      for (int o = 0; o < kTiles; ++o)
        for (int i = 0; i < 4; ++i) y.acc[t][o][i] = ldexpf(y.acc[t][o][i], -up - up_v);
      if (y.ref[t] != kNone) y.ref[t] += shift[t];
    }
  }
  if (span.banded && !idle) {
    Band<D, WIDE, NT> band(a, b, kv, lane);
    for (int t = 0; t < NT; ++t) {
      float x[kSteps][8];
      load_row(t, x);
      band.set_queries(t, x);
    }
    const int s0 = max(span.low, wave_lo), s1 = min(span.sink1, wave_hi), r0 = max(span.rec0, wave_lo), r1 = min(g.t1, wave_hi);
    for (int tb = s0 & ~31; tb < s1; tb += 32) band.attend(tb, s0, s1, row_lo, row_hi, y);
    for (int tb = r0 & ~31; tb < r1; tb += 32) band.attend(tb, r0, r1, row_lo, row_hi, y);
  }
  for (int t = 0; t < NT; ++t) {
    y.sum[t] = add_rows32(add_rows16(y.sum[t]));
    if (y.sum[t] != y.sum[t] && !(y.ref[t] > kNone)) y.ref[t] = 0.f;  // NaN logits move no reference, but attend
  }
  __syncthreads();  // the transform is done with
  q4::finish_rows<D, NT, kWaves, true>(
      a, g, {reinterpret_cast<float *>(s_lds), nullptr, nullptr, reinterpret_cast<float *>(s_lds + M::kInv), reinterpret_cast<int *>(s_lds + M::kLast)},
      wave, lane, y.acc, y.ref, y.sum);
}

}  // namespace

hipError_t launch_chunk_tile(const ChunkArgs &a, const ChunkPlan &plan, hipStream_t stream) {
  const unsigned groups = static_cast<unsigned>(a.batch) * a.num_kv_heads * plan.row_tiles * plan.n_split;
  using std::false_type;
  using std::integral_constant;
  using std::true_type;
  auto go = [&](auto d, auto wide, auto sq, auto ks, auto aligned) {
    chunk_tile_kernel<d(), wide(), sq(), ks(), aligned()><<<groups, kThreads, 0, stream>>>(a);
    return hipGetLastError();
  };
  auto by_blocks = [&](auto d, auto wide, auto sq, auto ks) {
    return a.layout.block_size % 16 == 0 ? go(d, wide, sq, ks, true_type{}) : go(d, wide, sq, ks, false_type{});
  };
  auto by_keys = [&](auto d, auto wide, auto sq) { return a.k_scales ? by_blocks(d, wide, sq, true_type{}) : by_blocks(d, wide, sq, false_type{}); };
  auto by_values = [&](auto d, auto wide) { return a.v_sq ? by_keys(d, wide, true_type{}) : by_keys(d, wide, false_type{}); };
  auto by_type = [&](auto d) { return a.q_bf16 ? by_values(d, false_type{}) : by_values(d, true_type{}); };
  return a.head_dim == 128 ? by_type(integral_constant<int, 128>{}) : by_type(integral_constant<int, 64>{});
}

}  // namespace novakv
