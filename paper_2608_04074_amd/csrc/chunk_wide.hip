// Attention of many query rows over the 2-bit cache (nova_kv_chunk_attn with more than 128 rows
// per KV head: chunks of prompts).
//
// A workgroup of eight waves takes 256 rows, 32 a wave, and 64 (32) tokens a round. The waves
// gather the tokens' codewords once, between them, from the codebooks in LDS to fragments in LDS,
// in the order in which the matrix cores take them: a key's pairs of groups as they come, values
// transposed in registers, a few tokens at a time. What a token has beside its codes (key scale, the
// scalar arm's grid) every lane loads for one of 16 tokens, and the row of 16 lanes shares it.
//
// Keys and values have two buffers each, which just fit beside both codebooks of head_dim 128 with 32
// tokens, so a round has one barrier, and makes the next round's scores beside its own weights.
//
// Bound by issue: of a round's cycles the matrix cores, the vector units (four instructions a score, an
// exponential counting twice, and the gathers) and LDS are busy 39, 47 and 41 percent, and overlap in part. Two
// sequences' 2048 queries of 4 heads over 8192 tokens take 551 us (889 TFLOP/s); one buffer and two barriers 650,
// the two waves of a SIMD in opposite phases 777, each wave gathering for itself 902. Parts of queries and
// probabilities: as in chunk_rows.hip; two of each (fp32) take 1023 us.
//
// Queries go through R_K^-T and sums back through R_V on the matrix cores, without leaving the
// wave: the transform's rows are dealt to the tiles so that a lane's results are its next operand.
#include <type_traits>

#include "chunk_common.h"

namespace novakv {

namespace {

using namespace chunk;

constexpr int kWaves = 8, kThreads = 64 * kWaves, kRows = 32 * kWaves;
typedef float float16_t __attribute__((ext_vector_type(16)));

// A lane (row n = lane % 32, j = lane / 32) holds, of a tile of 32 by its 32 rows, the tile's rows 8 (i / 4) + 4 j + i % 4.
__device__ __forceinline__ constexpr int tile_row(const int i, const int j) { return 8 * (i >> 2) + 4 * j + (i & 3); }
// f(0) .. f(15), as constants.
template <typename F>
__device__ __forceinline__ void each16(F f) {
  using std::integral_constant;
  f(integral_constant<int, 0>{}), f(integral_constant<int, 1>{}), f(integral_constant<int, 2>{}), f(integral_constant<int, 3>{});
  f(integral_constant<int, 4>{}), f(integral_constant<int, 5>{}), f(integral_constant<int, 6>{}), f(integral_constant<int, 7>{});
  f(integral_constant<int, 8>{}), f(integral_constant<int, 9>{}), f(integral_constant<int, 10>{}), f(integral_constant<int, 11>{});
  f(integral_constant<int, 12>{}), f(integral_constant<int, 13>{}), f(integral_constant<int, 14>{}), f(integral_constant<int, 15>{});
}
// The value of lane I of the lane's row of 16 (DPP row_newbcast).
template <int I>
__device__ __forceinline__ float of_row16(const float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x150 + I, 0xf, 0xf, false));
}
// Coordinate of output tile c's row m: a lane's codewords of a group are rows of all tiles.
template <int D>
__device__ __forceinline__ int coord(const int c, const int m) {
  return D == 128 ? 4 * m + c : 4 * (m & 15) + 2 * (m >> 4) + c;
}

// LDS of a workgroup, in bytes.
template <int D, bool SQ>
struct Lds {
  static constexpr int kTiles = D / 32, kSteps = D / 16;
  static constexpr int kTokens = D == 128 && !SQ ? 32 : 64, kRuns = kTokens / 32;  // a round's tokens, runs of 32
  static constexpr int kKeyFrags = kRuns * kSteps, kValueFrags = 2 * kRuns * kTiles;
  static constexpr int kBook = D / kGroupDim * kCodebookSize * 8;
  static constexpr int kKeys = (SQ ? 1 : 2) * kBook;             // [round mod 2][run * kSteps + step][lane] 16 bytes
  static constexpr int kValues = kKeys + 2 * kKeyFrags * 1024;   // [round mod 2][(2 * run + half) * kTiles + tile][lane]
  static constexpr int kLoopEnd = kValues + 2 * kValueFrags * 1024;
  // in front of and behind the loop: a transform's parts [tile][step][hi, lo][lane] 16 bytes, made of its rows [D][D + 1]
  static constexpr int kRaw = kTiles * kSteps * 2 * 1024, kTops = kRaw + D * (D + 1) * 4, kTransformEnd = kTops + kWaves * 4;
  static constexpr int kMost = kLoopEnd > kTransformEnd ? kLoopEnd : kTransformEnd;
  static constexpr int kLast = 0;  // at the end
  static constexpr int kBytes = kMost;
  static_assert(kBytes <= 160 * 1024, "LDS of a workgroup");
  static_assert(kKeyFrags % kWaves == 0, "the waves share the gathers evenly");
};

// A [D][D] transform's parts in LDS: element(o, m, k) gives the place (row * (D + 1) + column) of what
// tile o's row m has in slot k of the contraction's D. Returns the exponent of their scale. The array comes in as
// it lies: the slots' own order would be 64 requests a load.
template <int D, typename M, typename F>
__device__ __forceinline__ int stage_transform(uint8_t *lds, const void *t, const int bf16, const int wave, const int lane, F element) {
  constexpr int kPieces = D * D / 4 / kThreads, kFrags = M::kTiles * M::kSteps;
  half8_t *const to = reinterpret_cast<half8_t *>(lds);
  float *const raw = reinterpret_cast<float *>(lds + M::kRaw), *const tops = reinterpret_cast<float *>(lds + M::kTops);
  T4 piece[kPieces];
  for (int i = 0; i < kPieces; ++i) piece[i] = load_t4(t, 4 * (static_cast<size_t>(i) * kThreads + threadIdx.x), bf16);
  float top = 0.f;
  for (int i = 0; i < kPieces; ++i) {
    const int x = 4 * (i * kThreads + threadIdx.x);
    const float4 v = t4_value(piece[i], bf16);
    float *p = raw + (x / D) * (D + 1) + x % D;
    p[0] = v.x, p[1] = v.y, p[2] = v.z, p[3] = v.w;
    top = fmaxf(fmaxf(top, fmaxf(fabsf(v.x), fabsf(v.y))), fmaxf(fabsf(v.z), fabsf(v.w)));
  }
  top = wave_max(top);
  if (lane == 0) tops[wave] = top;
  __syncthreads();
  for (int u = 0; u < kWaves; ++u) top = fmaxf(top, tops[u]);
  const int up = up_to_14(top);
  const float scale = ldexpf(1.f, up);
  for (int f = wave; f < kFrags; f += kWaves) {
    const int o = f / M::kSteps, s = f % M::kSteps;
    half8_t h, l;
    for (int e = 0; e < 8; ++e) {
      _Float16 hi, lo;
      split_half(raw[element(o, lane & 31, 16 * s + 8 * (lane >> 5) + e)] * scale, hi, lo);
      h[e] = hi, l[e] = lo;
    }
    to[2 * f * 64 + lane] = h;
    to[(2 * f + 1) * 64 + lane] = l;
  }
  __syncthreads();
  return up;
}

// A row tile times a staged transform, x in two parts (LOW) or one.
template <int D, bool LOW>
__device__ __forceinline__ void transform_rows(const half8_t *t, const int lane, const half8_t (&xh)[D / 16], const half8_t (&xl)[D / 16],
                                               float16_t (&out)[D / 32]) {
  for (int o = 0; o < D / 32; ++o) {
    for (int i = 0; i < 16; ++i) out[o][i] = 0.f;
    for (int s = 0; s < D / 16; ++s) {
      const half8_t h = t[((o * (D / 16) + s) * 2) * 64 + lane], l = t[((o * (D / 16) + s) * 2 + 1) * 64 + lane];
      out[o] = __builtin_amdgcn_mfma_f32_32x32x16_f16(h, xh[s], out[o], 0, 0, 0);
      out[o] = __builtin_amdgcn_mfma_f32_32x32x16_f16(l, xh[s], out[o], 0, 0, 0);
      if constexpr (LOW) out[o] = __builtin_amdgcn_mfma_f32_32x32x16_f16(h, xl[s], out[o], 0, 0, 0);
    }
  }
}

// A wave's sums over its 32 rows (lane: row lane mod 32), in front of the division.
template <int D>
struct Sums32 {
  float ref = kNone, sum = 0.f, off_sum = 0.f;
  float16_t acc[D / 32];
  __device__ __forceinline__ Sums32() {
    for (int o = 0; o < D / 32; ++o)
      for (int i = 0; i < 16; ++i) acc[o][i] = 0.f;
  }
  // as Sums::raise
  __device__ __forceinline__ void raise(const float bound) {
    if (!__any(bound > ref + (kTop + kSlack))) return;
    const float to = fmaxf(ref, max_rows32(bound) - kTop);
    const float f = to == kNone ? 1.f : half_factor(ref - to);
    ref = to;
    for (int y = 0; y < 2; ++y) {
      sum *= f;
      off_sum *= f;
      for (int o = 0; o < D / 32; ++o) acc[o] *= f;
    }
  }
};

// As Band, over 32 rows.
template <int D, bool WIDE>
struct Band32 {
  static constexpr int kQParts = WIDE ? 3 : 1, kPParts = WIDE ? 3 : 2, kSteps = D / 16, kTiles = D / 32;
  const ChunkArgs &a;
  size_t rows;  // of the (sequence, KV head)
  int n, j;
  bf16x8 q[kSteps][kQParts];

  __device__ __forceinline__ Band32(const ChunkArgs &args, const int b, const int kv, const int lane, const float (&x)[kSteps][8])
      : a(args), rows((static_cast<size_t>(b) * args.num_kv_heads + kv) * (args.n_sink + args.n_rec)), n(lane & 31), j(lane >> 5) {
    for (int s = 0; s < kSteps; ++s)
      for (int e = 0; e < 8; ++e) {
        if constexpr (WIDE) {
          __bf16 u, v, w;
          split_bf16(x[s][e], u, v, w);
          q[s][0][e] = u, q[s][1][e] = v, q[s][2][e] = w;
        } else {
          q[s][0][e] = static_cast<__bf16>(x[s][e]);
        }
      }
  }
  // Positions [from, to) of the 32 from tb on, for rows that attend [row_lo, row_hi).
  __device__ __forceinline__ void attend(const int tb, const int from, const int to, const int row_lo, const int row_hi, Sums32<D> &y) const {
    auto row_of = [&](const int tok) { return (rows + band_slot(min(max(tok, from), to - 1), a.n_sink, a.n_rec)) * D; };
    // all loads in front of their first use
    const uint16_t *k = a.band_k + row_of(tb + n) + 8 * j;
    bf16x8 keys[kSteps];
    for (int st = 0; st < kSteps; ++st) keys[st] = *reinterpret_cast<const bf16x8 *>(k + 16 * st);
    uint32_t v[16][kTiles / 2];  // a lane's 16 tokens, its coordinates in all tiles
    for (int i = 0; i < 16; ++i) {
      const uint16_t *p = a.band_v + row_of(tb + tile_row(i, j));
      for (int w = 0; w < kTiles / 2; ++w) v[i][w] = *reinterpret_cast<const uint32_t *>(p + coord<D>(2 * w, n));
    }
    float16_t s;
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
    for (int st = 0; st < kSteps; ++st) {
      const bf16x8 kf = keys[st];
      for (int p = 0; p < kQParts; ++p) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, q[st][p], s, 0, 0, 0);
    }
    float bound = kNone;
    for (int i = 0; i < 16; ++i) {
      const int tok = tb + tile_row(i, j);
      bool bad = false;
      for (int w = 0; w < kTiles / 2; ++w) {
        bad |= (v[i][w] & 0x7f80u) == 0x7f80u || (v[i][w] & 0x7f800000u) == 0x7f800000u;
      }
      // A value that is not finite would reach the rows it is hidden from (0 * NaN): the token's
      // score becomes NaN instead, and the value 0.
      const uint64_t any = __ballot(bad);
      const bool odd = static_cast<uint32_t>(any >> (32 * j)) != 0;
      for (int w = 0; w < kTiles / 2; ++w) v[i][w] = odd ? 0u : v[i][w];
      const bool seen = static_cast<int>(tok >= max(from, row_lo)) & static_cast<int>(tok < min(to, row_hi));
      s[i] = seen ? (odd ? __builtin_nanf("") : s[i] * a.qscale) : kNone;
      bound = fmaxf(bound, s[i]);
    }
    y.raise(bound);
    const float r = y.ref == kNone ? 0.f : y.ref;
    for (int u = 0; u < 2; ++u) {  // 16 tokens each: slot e is the lane's token 8 u + e
      bf16x8 pf[kPParts];
      for (int e = 0; e < 8; ++e) {
        const float p = exp2_raw(s[8 * u + e] - r);
        y.sum += p;
        __bf16 x, z, w;
        split_bf16(p, x, z, w);
        pf[0][e] = x, pf[1][e] = z;
        if constexpr (kPParts == 3) pf[2][e] = w;
      }
      for (int o = 0; o < kTiles; ++o) {
        uint32_t w[4];
        for (int x = 0; x < 4; ++x) w[x] = half_pair(v[8 * u + 2 * x][o / 2], v[8 * u + 2 * x + 1][o / 2], o & 1);
        const bf16x8 vf = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
        for (int p = 0; p < kPParts; ++p) y.acc[o] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[p], y.acc[o], 0, 0, 0);
      }
    }
  }
};

// D: head_dim. WIDE: fp32 queries. SQ: the scalar value arm. KS: key scales. ALIGNED: blocks of a multiple of 16 rows.
template <int D, bool WIDE, bool SQ, bool KS, bool ALIGNED>
__global__ __launch_bounds__(kThreads, 2) void chunk_wide_kernel(const ChunkArgs a) {
  using M = Lds<D, SQ>;
  constexpr int kParts = WIDE ? 2 : 1, L = D / kGroupDim, kSteps = M::kSteps, kTiles = M::kTiles, kTokens = M::kTokens, kRuns = M::kRuns;
  constexpr int kKeyUnits = M::kKeyFrags / kWaves;                // of a wave: fragments of keys
  constexpr int kValueTokens = kTokens * L / (64 * kWaves);       // of a lane: tokens of a value group, 2 or 4
  __shared__ __align__(16) uint8_t s_lds[M::kBytes];
  uint2 *const s_key_book = reinterpret_cast<uint2 *>(s_lds), *const s_value_book = s_key_book + L * kCodebookSize;
  half8_t *const s_keys = reinterpret_cast<half8_t *>(s_lds + M::kKeys), *const s_values = reinterpret_cast<half8_t *>(s_lds + M::kValues);
  const half8_t *const s_frags = reinterpret_cast<const half8_t *>(s_lds);

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int lane = threadIdx.x & 63, n = lane & 31, j = lane >> 5;
  Tile g;
  q4::place_tile(a, kRows, g);
  if (!q4::find_span(a, kRows, kTokens, g)) return;
  const int b = g.b, kv = g.kv;
  const Spans span(a, g);
  const int c0 = span.c0, c1 = span.c1;
  // this wave's rows
  const int row0 = g.row0 + 32 * wave, row1 = min(row0 + 32, g.rows_valid);
  const bool idle = row0 >= g.rows_valid;
  const int wave_lo = idle ? 0 : g.first_pos(a, row0), wave_hi = idle ? 0 : g.last_pos(a, row1 - 1) + 1;
  const int inner_lo = idle ? 0 : g.first_pos(a, row1 - 1), inner_hi = idle ? 0 : g.last_pos(a, row0) + 1;  // seen by all of them
  const int row = row0 + n;
  const bool on = row < g.rows_valid;
  const int row_hi = on ? g.last_pos(a, row) + 1 : 0, row_lo = on ? g.first_pos(a, row) : 0;
  auto load_row = [&](float (&x)[kSteps][8]) {  // coordinates 16 s + 8 j + e
    for (int s = 0; s < kSteps; ++s)
      for (int e = 0; e < 8; ++e) x[s][e] = 0.f;
    if (!on) return;
    const int i = row / a.gqa, h = row - i * a.gqa;
    const size_t at = ((static_cast<size_t>(b) * a.n_q + i) * a.num_q_heads + kv * a.gqa + h) * D + 8 * j;
    for (int s = 0; s < kSteps; ++s) load_query<WIDE>(a.q, at + 16 * s, x[s]);
  };

  Sums32<D> y;
  if (span.codes) {
    // ---- q' = q R_K^-T. A lane's results f = 16 o + i are its coordinates (D / 2) j + f, eight for each of the scores' steps.
    const int up_t = stage_transform<D, M>(s_lds, transform_of(a.t_k_inv_t, kv, D, a.t_bf16), a.t_bf16, wave, lane,
                                           [](const int o, const int m, const int k) {
                                             return k * (D + 1) + (D / 2) * ((m >> 2) & 1) + 16 * o + 4 * (m >> 3) + (m & 3);
                                           });
    half8_t qf[kSteps][kParts];
    float alpha, shift;
    {
      float x[kSteps][8];
      load_row(x);
      float top = 0.f, dot = 0.f;
      bool finite = true;
      for (int s = 0; s < kSteps; ++s)
        for (int e = 0; e < 8; ++e) {
          finite = finite && fabsf(x[s][e]) < __builtin_inff();
          top = fmaxf(top, fabsf(x[s][e]));
          dot = __builtin_fmaf(x[s][e], a.kbar[kv * D + 16 * s + 8 * j + e], dot);
        }
      shift = add_rows32(dot) * a.qscale;
      top = max_rows32(finite ? top : __builtin_inff());
      const bool usable = top < __builtin_inff();
      const int up = up_to_14(top);
      const float scale = ldexpf(1.f, up);
      half8_t xh[kSteps], xl[kSteps];
      for (int s = 0; s < kSteps; ++s)
        for (int e = 0; e < 8; ++e) {
          _Float16 hi, lo;
          split_half(usable ? x[s][e] * scale : __builtin_nanf(""), hi, lo);  // a row that is not finite: NaN scores
          xh[s][e] = hi, xl[s][e] = lo;
        }
      float16_t out[kTiles];
      transform_rows<D, WIDE>(s_frags, lane, xh, xl, out);
      // |out| <= D 2^28: times 2^-20 it fits fp16
      for (int s = 0; s < kSteps; ++s)
        for (int e = 0; e < 8; ++e) {
          _Float16 hi, lo;
          split_half(out[s >> 1][8 * (s & 1) + e] * 0x1p-20f, hi, lo);
          qf[s][0][e] = hi;
          if constexpr (WIDE) qf[s][1][e] = lo;
        }
      alpha = fminf(fmaxf(ldexpf(a.qscale, 20 - up - up_t), 0x1p-126f), 0x1p126f);
    }
    __syncthreads();
    stage_book<L, kThreads>(s_key_book, a.cb_k, a.cb_fp8, kv);
    if constexpr (!SQ) stage_book<L, kThreads>(s_value_book, a.cb_v, a.cb_fp8, kv);

    // ---- this wave's share of the gathers: keys of run `run`, steps key_step and on; a lane's value group and the
    // first of its tokens, whose pairs (fours) of coordinates are parts of a fragment's lane
    const int run = wave % kRuns, key_step = wave / kRuns;
    const int step16 = kTokens == 64 ? wave >> 1 : wave >> 2;
    const int eight = D == 64 ? (lane >> 4) & 1 : kTokens == 64 ? wave & 1 : (wave >> 1) & 1;
    const int pair = kValueTokens == 4 ? 0 : wave & 1;
    const int group = D == 128 ? n : lane & 15, value_token = 8 * eight + 4 * j + 2 * pair;
    const int extra_token = tile_row(lane & 15, j);  // of a run, whose scale or grid this lane has for its row of 16 lanes
    const int bs = a.layout.block_size;
    const Blocks blocks(a.layout, b, a.seq_lens + b);
    // Where a round's tokens lie. ALIGNED: the first row of each 16, looked up by a lane of each row; else the rows of the
    // lane's key, its values and its extras' tokens.
    constexpr int kPlaces = ALIGNED ? 1 : 1 + kValueTokens + kRuns;
    struct Look {
      int entry[kPlaces], block[kPlaces], row[kPlaces];  // as loaded: arithmetic on it would wait for it
    };
    struct Places {
      size_t key[2], value[ALIGNED ? 1 : kValueTokens], extra[2 * kRuns];  // key, extra: of both runs of 16 (else: [0] the lane's own)
    };
    int look_tb = c0 & ~31;
    auto look_up = [&](Look &k) {
      // nothing outside the attended tokens' own runs of 16 (elsewhere: tokens) is looked up
      auto find = [&](const int i, const int tok) {
        const int blk = a.block_of(tok);
        k.row[i] = tok - blk * bs;
        k.block[i] = blk;
        k.entry[i] = blocks.entry(blk);
      };
      if constexpr (ALIGNED) {
        find(0, min(max(look_tb + 16 * ((lane >> 4) & (2 * kRuns - 1)), c0 & ~15), (c1 - 1) & ~15));
      } else {
        auto inside = [&](const int tok) { return min(max(tok, c0), c1 - 1); };
        find(0, inside(look_tb + 32 * run + n));
        for (int i = 0; i < kValueTokens; ++i) find(1 + i, inside(look_tb + 16 * step16 + value_token + i));
        if constexpr (KS || SQ)
          for (int x = 0; x < kRuns; ++x) find(1 + kValueTokens + x, inside(look_tb + 32 * x + extra_token));
      }
      look_tb += kTokens;
    };
    auto place = [&](const Look &k) {
      auto row_of = [&](const int phys, const int row) { return (static_cast<size_t>(phys) * a.num_kv_heads + kv) * bs + row; };
      Places p;
      if constexpr (ALIGNED) {
        auto first_of = [&](const int run16) {
          return row_of(blocks.phys(__builtin_amdgcn_readlane(k.entry[0], 16 * run16), __builtin_amdgcn_readlane(k.block[0], 16 * run16)),
                        __builtin_amdgcn_readlane(k.row[0], 16 * run16));
        };
        p.key[0] = first_of(2 * run), p.key[1] = first_of(2 * run + 1), p.value[0] = first_of(step16);
        for (int i = 0; i < 2 * kRuns; ++i) p.extra[i] = KS || SQ ? first_of(i) : 0;
      } else {
        p.key[0] = row_of(blocks.phys(k.entry[0], k.block[0]), k.row[0]);
        for (int i = 0; i < kValueTokens; ++i) p.value[i] = row_of(blocks.phys(k.entry[1 + i], k.block[1 + i]), k.row[1 + i]);
        for (int x = 0; x < kRuns; ++x) {
          const int i = kPlaces - kRuns + x;
          p.extra[2 * x] = KS || SQ ? row_of(blocks.phys(k.entry[i], k.block[i]), k.row[i]) : 0;
        }
      }
      return p;
    };
    // row of a lane's token of a run of 32
    auto row_in = [&](const size_t first, const size_t second, const int tok) { return ALIGNED ? (tok & 16 ? second : first) + (tok & 15) : first; };
    struct KeyCodes {
      uint32_t code[kKeyUnits];
    };
    struct ValueCodes {
      uint32_t code[kValueTokens];
    };
    struct Extras {
      uint32_t rho[kRuns], sq[kRuns];
    };
    auto request_keys = [&](const Places &p, KeyCodes &c) {
      const uint8_t *from = a.k_codes + row_in(p.key[0], p.key[1], n) * L + (L / 2) * j + 2 * key_step;
      for (int u = 0; u < kKeyUnits; ++u) c.code[u] = *reinterpret_cast<const uint16_t *>(from + 2 * u * (kWaves / kRuns));
    };
    auto request_values = [&](const Places &p, ValueCodes &c, Extras &x) {
      if constexpr (ALIGNED) {
        const uint8_t *from = a.v_codes + p.value[0] * L + (value_token * L + group);
        for (int i = 0; i < kValueTokens; ++i) c.code[i] = from[i * L];
      } else {
        for (int i = 0; i < kValueTokens; ++i) c.code[i] = a.v_codes[p.value[i] * L + group];
      }
      for (int r = 0; r < kRuns; ++r) {
        if constexpr (KS || SQ) {
          const size_t at = row_in(p.extra[2 * r], p.extra[2 * r + 1], extra_token);
          if constexpr (KS) x.rho[r] = a.k_scales[at];
          if constexpr (SQ) x.sq[r] = reinterpret_cast<const uint32_t *>(a.v_sq)[at];
        }
      }
    };
    auto put_keys = [&](const KeyCodes &c, const int parity) {
      for (int u = 0; u < kKeyUnits; ++u) {
        const int st = key_step + u * (kWaves / kRuns);
        const uint2 *book = s_key_book + ((L / 2) * j + 2 * st) * kCodebookSize;
        const uint2 w0 = book[c.code[u] & 0xffu], w1 = book[kCodebookSize + (c.code[u] >> 8)];
        s_keys[(parity * M::kKeyFrags + run * kSteps + st) * 64 + lane] = __builtin_bit_cast(half8_t, make_uint4(w0.x, w0.y, w1.x, w1.y));
      }
    };
    auto put_values = [&](const ValueCodes &c, const int parity) {
      uint2 w[kValueTokens];
      for (int i = 0; i < kValueTokens; ++i) {
        if constexpr (SQ) w[i] = centred_levels(c.code[i]);
        else w[i] = s_value_book[group * kCodebookSize + c.code[i]];
      }
      for (int x = 0; x < 4; ++x) {  // coordinate x of the group: tile and row of the fragment's lanes
        const int tile = D == 128 ? x : x & 1, m = D == 128 ? n : group + 16 * (x >> 1);
        uint32_t *to = reinterpret_cast<uint32_t *>(s_values + (parity * M::kValueFrags + step16 * kTiles + tile) * 64 + 32 * j + m) + 2 * eight + pair;
        uint32_t u[kValueTokens / 2];
        for (int i = 0; i < kValueTokens / 2; ++i)
          u[i] = x < 2 ? half_pair(w[2 * i].x, w[2 * i + 1].x, x & 1) : half_pair(w[2 * i].y, w[2 * i + 1].y, x & 1);
        if constexpr (kValueTokens == 4) *reinterpret_cast<uint2 *>(to) = make_uint2(u[0], u[1]);
        else *to = u[0];
      }
    };

    // ---- a round's scores
    auto make_scores = [&](const int parity, float16_t (&s)[kRuns]) {
      for (int x = 0; x < kRuns; ++x)
        for (int i = 0; i < 16; ++i) s[x][i] = 0.f;
      for (int st = 0; st < kSteps; ++st)
        for (int x = 0; x < kRuns; ++x) {
          const half8_t k = s_keys[(parity * M::kKeyFrags + x * kSteps + st) * 64 + lane];
          for (int p = 0; p < kParts; ++p) s[x] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k, qf[st][p], s[x], 0, 0, 0);
        }
    };
    // ---- their weights, which meet the values
    auto weigh = [&](const int tb, const int parity, const Extras &extra, float16_t (&s)[kRuns]) {
      float scale[kRuns], offset[kRuns], expo[kRuns];
      if constexpr (KS || SQ) {
        for (int x = 0; x < kRuns; ++x) {
          float rho = 1.f;
          if constexpr (KS) rho = __uint_as_float(extra.rho[x] << 16);
          if constexpr (SQ) {
            const int tok = tb + 32 * x + extra_token;
            const Grid v = grid_of(extra.sq[x], tok >= c0 && tok < c1, rho);
            scale[x] = v.scale, offset[x] = v.offset, expo[x] = v.expo;
          }
          each16([&](auto i) { s[x][i()] *= of_row16<i()>(rho); });
        }
      }
      if (!(tb >= max(inner_lo, c0) && tb + kTokens <= min(inner_hi, c1))) {
        for (int x = 0; x < kRuns; ++x)
          for (int i = 0; i < 16; ++i) {
            const int m = tb + 32 * x + tile_row(i, j);
            const bool seen = static_cast<int>(m >= max(c0, row_lo)) & static_cast<int>(m < min(c1, row_hi));
            s[x][i] = seen ? s[x][i] : kNone;
          }
      }
      float bound = kNone;
      for (int x = 0; x < kRuns; ++x) {
        if constexpr (SQ) each16([&](auto i) { bound = fmaxf(bound, __builtin_fmaf(s[x][i()], alpha, of_row16<i()>(expo[x]))); });
        else
          for (int i = 0; i < 16; ++i) bound = fmaxf(bound, s[x][i]);
      }
      if constexpr (!SQ) bound *= alpha;
      y.raise(bound);
      const float r = y.ref == kNone ? 0.f : y.ref;
      half8_t pf[2 * kRuns][kParts];
      for (int x = 0; x < kRuns; ++x)
        each16([&](auto i) {
          float p = exp2_raw(__builtin_fmaf(s[x][i()], alpha, -r));
          y.sum += p;  // not of fp16 parts: small weights of many tokens would be lost
          if constexpr (SQ) {
            y.off_sum = __builtin_fmaf(of_row16<i()>(offset[x]), p, y.off_sum);
            p *= of_row16<i()>(scale[x]);
          }
          half8_t *to = pf[2 * x + i() / 8];
          if constexpr (WIDE) {
            _Float16 hi, lo;
            split_half(p, hi, lo);
            to[0][i() % 8] = hi, to[kParts - 1][i() % 8] = lo;
          } else {
            to[0][i() % 8] = static_cast<_Float16>(p);
          }
        });
      for (int u = 0; u < 2 * kRuns; ++u)
        for (int o = 0; o < kTiles; ++o) {
          const half8_t v = s_values[(parity * M::kValueFrags + u * kTiles + o) * 64 + lane];
          for (int p = 0; p < kParts; ++p) y.acc[o] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, pf[u][p], y.acc[o], 0, 0, 0);
        }
    };

    // Round i: the next round's scores, this one's weights; the codes of keys of round i + 2 and values of i + 1 become
    // fragments, those of the rounds behind are requested (past the end: the last tokens again).
    Look look;
    KeyCodes keys;
    ValueCodes values;
    Extras extra, extra_next;
    float16_t s0[kRuns], s1[kRuns];
    look_up(look);
    Places ahead = place(look);
    request_keys(ahead, keys);
    request_values(ahead, values, extra);
    look_up(look);
    ahead = place(look);
    look_up(look);
    __syncthreads();  // the codebooks are there
    put_keys(keys, 0);
    put_values(values, 0);
    request_keys(ahead, keys);
    request_values(ahead, values, extra_next);
    ahead = place(look);
    look_up(look);
    put_keys(keys, 1);
    request_keys(ahead, keys);
    __syncthreads();
    make_scores(0, s0);
    __syncthreads();
    auto round = [&](const int tb, const int parity, float16_t (&now)[kRuns], float16_t (&next)[kRuns]) {
      make_scores(parity ^ 1, next);
      put_values(values, parity ^ 1);
      put_keys(keys, parity);
      const Extras beside = extra;
      extra = extra_next;
      request_values(ahead, values, extra_next);
      ahead = place(look);
      request_keys(ahead, keys);
      look_up(look);
      weigh(tb, parity, beside, now);
      __syncthreads();
    };
    for (int tb = c0 & ~31;;) {
      round(tb, 0, s0, s1);
      if ((tb += kTokens) >= c1) break;
      round(tb, 1, s1, s0);
      if ((tb += kTokens) >= c1) break;
    }

    // ---- back through R_V
    const int up_v = stage_transform<D, M>(s_lds, transform_of(a.t_v, kv, D, a.t_bf16), a.t_bf16, wave, lane,
                                           [](const int o, const int m, const int k) {
                                             const int f = 8 * (k >> 4) + (k & 7);
                                             return coord<D>(o, m) * (D + 1) + coord<D>(f >> 4, tile_row(f & 15, (k >> 3) & 1));
                                           });
    if constexpr (SQ) {
      const float off = add_rows32(y.off_sum);
      for (int o = 0; o < kTiles; ++o)
        for (int i = 0; i < 16; ++i) y.acc[o][i] += off;
    }
    float top = 0.f;
    for (int o = 0; o < kTiles; ++o)
      for (int i = 0; i < 16; ++i) top = fmaxf(top, fabsf(y.acc[o][i]));
    const int up = up_to_14(max_rows32(top));
    const float scale = ldexpf(1.f, up);
    half8_t xh[kSteps], xl[kSteps];
    for (int s = 0; s < kSteps; ++s)
      for (int e = 0; e < 8; ++e) {
        _Float16 hi, lo;
        split_half(y.acc[s >> 1][8 * (s & 1) + e] * scale, hi, lo);
        xh[s][e] = hi, xl[s][e] = lo;
      }
    transform_rows<D, true>(s_frags, lane, xh, xl, y.acc);
    for (int o = 0; o < kTiles; ++o)
      for (int i = 0; i < 16; ++i) y.acc[o][i] = ldexpf(y.acc[o][i], -up - up_v);
    if (y.ref != kNone) y.ref += shift;
  }
  if (span.banded && !idle) {
    float x[kSteps][8];
    load_row(x);
    const Band32<D, WIDE> band(a, b, kv, lane, x);
    const int s0 = max(span.low, wave_lo), s1 = min(span.sink1, wave_hi), r0 = max(span.rec0, wave_lo), r1 = min(g.t1, wave_hi);
    for (int tb = s0 & ~31; tb < s1; tb += 32) band.attend(tb, s0, s1, row_lo, row_hi, y);
    for (int tb = r0 & ~31; tb < r1; tb += 32) band.attend(tb, r0, r1, row_lo, row_hi, y);
  }
  y.sum = add_rows32(y.sum);
  if (y.sum != y.sum && !(y.ref > kNone)) y.ref = 0.f;  // NaN logits move no reference, but attend

  // A lane's values in fours of coordinates from 4 tile_row(x, j) on (D = 64: registers x and x + 8).
  const q4::TileRows<D, kRows> rows{a, g};
  float *const part = rows.part();
  auto four = [&](const int x) {
    return D == 128 ? make_float4(y.acc[0][x], y.acc[1][x], y.acc[kTiles - 2][x], y.acc[kTiles - 1][x])
                    : make_float4(y.acc[0][x], y.acc[1][x], y.acc[0][(x + 8) & 15], y.acc[1][(x + 8) & 15]);
  };
  if (!part) {
    if (!on) return;
    const float f = rows.inverse(row - g.row0, y.ref, y.sum);
    for (int x = 0; x < D / 8; ++x) q4::store_out(a, rows.out_at(row - g.row0) + 4 * tile_row(x, j), rows.scaled(four(x), f));
    return;
  }
  // Splits: their values lie as the lanes hold them, so that the words of a store (8 bytes each, with device
  // coherence) follow each other; the last workgroup of the tile to arrive merges them, in their order.
  if (!idle) {
    uint64_t *words = reinterpret_cast<uint64_t *>(part) + wave * (D / 4) * 64 + lane;
    for (int x = 0; x < D / 8; ++x) {
      const float4 v = four(x);
      q4::publish2(reinterpret_cast<float *>(words + 2 * x * 64), v.x, v.y);
      q4::publish2(reinterpret_cast<float *>(words + (2 * x + 1) * 64), v.z, v.w);
    }
    if (j == 0) q4::publish2(part + kRows * D + 2 * (32 * wave + n), y.ref, y.sum);
  }
  int *const s_last = reinterpret_cast<int *>(s_lds + M::kLast);
  __builtin_amdgcn_s_waitcnt(0);  // this thread's words have landed
  __syncthreads();
  int *const counter = a.counters + static_cast<size_t>(g.unit) * a.row_tiles + g.tile;
  if (threadIdx.x == 0)
    *s_last = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == a.n_split - 1;
  __syncthreads();
  if (!*s_last) return;
  if (threadIdx.x == 0) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  if (idle) return;
  const float *const parts = part - g.split * rows.kSlot;
  auto stat = [&](const int u) { return q4::fetch2(parts + u * rows.kSlot + kRows * D + 2 * (32 * wave + n)); };
  float most = kNone, l = 0.f;
#pragma unroll 8
  for (int u = 0; u < a.n_split; ++u) most = fmaxf(most, stat(u).x);
  for (int o = 0; o < kTiles; ++o)
    for (int i = 0; i < 16; ++i) y.acc[o][i] = 0.f;
  constexpr int kAhead = 256 / D;  // splits whose words are requested at once
  for (int first = 0; first < a.n_split; first += kAhead) {
    float2 ml[kAhead], v[kAhead][D / 4];
    for (int z = 0; z < kAhead; ++z) {
      const int u = min(first + z, a.n_split - 1);
      ml[z] = stat(u);
      const uint64_t *words = reinterpret_cast<const uint64_t *>(parts + u * rows.kSlot) + wave * (D / 4) * 64 + lane;
      for (int x = 0; x < D / 4; ++x) v[z][x] = q4::fetch2(reinterpret_cast<const float *>(words + x * 64));
    }
    for (int z = 0; z < kAhead; ++z) {
      // a split of no weight counts all the same: it may hold a NaN
      const bool some = first + z < a.n_split && ml[z].x != kNone;
      const float f = some ? half_factor(ml[z].x - most) : 0.f;
      if (some) l += f * ml[z].y * f;
      auto of = [&](const float value) { return some ? f * value * f : 0.f; };
      for (int x = 0; x < D / 8; ++x) {
        const float2 p = v[z][2 * x], q = v[z][2 * x + 1];
        y.acc[0][x] += of(p.x), y.acc[1][x] += of(p.y);
        if constexpr (D == 128) y.acc[kTiles - 2][x] += of(q.x), y.acc[kTiles - 1][x] += of(q.y);
        else y.acc[0][(x + 8) & 15] += of(q.x), y.acc[1][(x + 8) & 15] += of(q.y);
      }
    }
  }
  if (!on) return;
  const float f = rows.inverse(row - g.row0, most, l);
  for (int x = 0; x < D / 8; ++x) q4::store_out(a, rows.out_at(row - g.row0) + 4 * tile_row(x, j), rows.scaled(four(x), f));
}

}  // namespace

hipError_t launch_chunk_wide(const ChunkArgs &a, const ChunkPlan &plan, hipStream_t stream) {
  const unsigned groups = static_cast<unsigned>(a.batch) * a.num_kv_heads * plan.row_tiles * plan.n_split;
  using std::false_type;
  using std::integral_constant;
  using std::true_type;
  auto go = [&](auto d, auto wide, auto sq, auto ks, auto aligned) {
    chunk_wide_kernel<d(), wide(), sq(), ks(), aligned()><<<groups, kThreads, 0, stream>>>(a);
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
