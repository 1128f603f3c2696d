// Attention of a few query rows (query tokens times query heads of a KV head) over the 2-bit
// cache (nova_kv_chunk_attn): drafted tokens, short chunks, single tokens.
//
//   z_j = rho_j (q R_K^-T) . r_j + q . k_bar,  out = (sum_j p_j s_j / sum_j p_j) R_V^T
//
// over codewords r_j, s_j that are fp16 and so enter the matrix cores exactly. A workgroup
// has 16 (32) rows, turns their queries into the key transform's coordinates once, and its
// waves divide the tokens, 32 a round: a lane gathers a token's key codewords from the
// codebook in LDS, which are a matrix operand as they come, and eight tokens' codewords of a
// value group, which it transposes in registers. The sums go back through R_V once, merged over
// the waves.
//
// Queries and probabilities (times the scalar arm's scales) enter as one fp16 part in bf16 calls: half a step of them is
// 2^-12, an eighth of the half step that their outputs are rounded by, and a second part would double the matrix
// instructions. Those of fp32 calls enter as two parts (22 bits): 64 sequences of up to 16K tokens, four drafted
// tokens of 4 heads each, take 452 us in fp32. Weights are summed in fp32 before they are rounded.
//
// The same in bf16 takes 173 us (2.3 TB/s of the cache). No unit is at its limit: LDS is busy in 39% of the cycles (the
// gathers, 64 reads of eight bytes a token and head, two thirds of it bank conflicts), the vector units in 43, the
// matrix cores in 11; one workgroup a CU beside 128 KiB of codebooks leaves two waves a SIMD, and a round's gathers,
// products, weights and gathers follow each other. A short call is the workgroup's setup: 20 us over 2000 tokens,
// whether in splits of 512, 256 or 128 tokens.
//
// Positions that a band holds are attended first, with their exact bf16 rows on the bf16
// cores; their share joins behind R_V.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "chunk_common.h"

namespace novakv {

namespace {

using namespace chunk;

constexpr int kRound = 32;  // tokens a wave takes at a time
constexpr int W = 8;        // waves

template <int D, bool WIDE, int NT, bool SQ, bool ALIGNED>
struct Lds {
  static constexpr int kRows = 16 * NT, kParts = WIDE ? 2 : 1, kStride = D + 4, kQStride = D + 8;
  static constexpr int kBook = D / kGroupDim * kCodebookSize * 8;
  // while codes are attended
  static constexpr int kQ = (SQ ? 1 : 2) * kBook;                       // q' [part][row][D + 8] fp16
  static constexpr int kTok = kQ + kParts * kRows * kQStride * 2;       // [wave][rho, scale, offset, exponent][32] fp32
  static constexpr int kRowAt = kTok + W * 4 * kRound * 4;              // [wave][32] rows of tokens, 64 bits (ALIGNED: none)
  static constexpr int kLoopEnd = kRowAt + (ALIGNED ? 0 : W * kRound * 8);
  // while waves are merged
  static constexpr int kPart = 0;                                       // [wave][row][D + 4] fp32
  static constexpr int kMerged = W * kRows * kStride * 4;               // [row][D + 4]
  static constexpr int kMergeEnd = kMerged + kRows * kStride * 4;
  // always
  static constexpr int kStat = kLoopEnd > kMergeEnd ? kLoopEnd : kMergeEnd;  // [ref, sum][wave][row], [ref, sum][row], inverse [row]
  static constexpr int kTops = kStat + (2 * W + 3) * kRows * 4;              // [wave]
  static constexpr int kLast = kTops + W * 4;
  static constexpr int kBytes = kLast + 16;
  static_assert(kBytes <= 160 * 1024, "LDS of a workgroup");
};

// D: head_dim. WIDE: fp32 queries. NT: tiles of 16 rows. SQ: the scalar value arm.
// ALIGNED: blocks of a multiple of 16 rows.
template <int D, bool WIDE, int NT, bool SQ, bool ALIGNED>
__global__ __launch_bounds__(64 * W, 1) void chunk_rows_kernel(const ChunkArgs a) {
  using M = Lds<D, WIDE, NT, SQ, ALIGNED>;
  constexpr int kThreads = 64 * W, kRows = M::kRows, kParts = M::kParts;
  constexpr int L = D / kGroupDim, kSteps = D / 32, kTiles = D / 16, kWords = D / 64;
  __shared__ __align__(16) uint8_t s_lds[M::kBytes];
  uint2 *const s_key = reinterpret_cast<uint2 *>(s_lds), *const s_value = s_key + L * kCodebookSize;
  _Float16 *const s_q = reinterpret_cast<_Float16 *>(s_lds + M::kQ);
  float *const s_part = reinterpret_cast<float *>(s_lds + M::kPart), *const s_merged = reinterpret_cast<float *>(s_lds + M::kMerged);
  float *const s_ref = reinterpret_cast<float *>(s_lds + M::kStat), *const s_sum = s_ref + W * kRows;
  float *const s_mref = s_sum + W * kRows, *const s_msum = s_mref + kRows, *const s_inv = s_msum + kRows;
  float *const s_tops = reinterpret_cast<float *>(s_lds + M::kTops);

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int lane = threadIdx.x & 63, n = lane & 15, j = lane >> 4;
  float *const s_tok = reinterpret_cast<float *>(s_lds + M::kTok) + wave * 4 * kRound;
  uint64_t *const s_row_at = reinterpret_cast<uint64_t *>(s_lds + M::kRowAt) + wave * kRound;

  Tile g;
  q4::place_tile(a, kRows, g);
  if (!q4::find_span(a, kRows, kRound * W, g)) return;
  const int b = g.b, kv = g.kv;
  const Spans span(a, g);
  const int c0 = span.c0, c1 = span.c1;

  // this lane's rows: their queries, and the attended positions [row_lo, row_hi)
  int row_lo[NT], row_hi[NT];
  float q[NT][kSteps][8];  // coordinates 32 s + 8 j + e
  for (int t = 0; t < NT; ++t) {
    const int row = g.row0 + 16 * t + n;
    const bool on = row < g.rows_valid;
    const int i = row / a.gqa, h = row - i * a.gqa;
    row_hi[t] = on ? g.last_pos(a, row) + 1 : 0;
    row_lo[t] = on ? g.first_pos(a, row) : 0;
    const size_t at = ((static_cast<size_t>(b) * a.n_q + i) * a.num_q_heads + kv * a.gqa + h) * D + 8 * j;
    for (int s = 0; s < kSteps; ++s)
      for (int e = 0; e < 8; ++e) q[t][s][e] = 0.f;
    if (!on) continue;
    for (int s = 0; s < kSteps; ++s) load_query<WIDE>(a.q, at + 32 * s, q[t][s]);
  }

  Sums<D, NT> y;
  auto &ref = y.ref, &sum = y.sum, &off_sum = y.off_sum;
  auto &acc = y.acc;
  // The waves' sums, whose tile o's row m is coordinate coord(o, m), merged: s_merged, s_mref, s_msum.
  // shift: what the logits of a row lack.
  auto merge_waves = [&](auto coord, const float (&shift)[NT]) {
    for (int t = 0; t < NT; ++t) {
      sum[t] = add_rows32(add_rows16(sum[t]));
      float r = ref[t] == kNone ? kNone : ref[t] + shift[t];
      if (sum[t] != sum[t]) r = r == r && r != kNone ? r : 0.f;  // NaN logits move no reference, but attend
      float *row = s_part + (wave * kRows + 16 * t + n) * M::kStride;
      for (int y = 0; y < kTiles / 4; ++y)
        for (int i = 0; i < 4; ++i)
          *reinterpret_cast<float4 *>(row + coord(4 * y, 4 * j + i)) =
              make_float4(acc[t][4 * y][i], acc[t][4 * y + 1][i], acc[t][4 * y + 2][i], acc[t][4 * y + 3][i]);
      if (j == 0) s_ref[wave * kRows + 16 * t + n] = r, s_sum[wave * kRows + 16 * t + n] = sum[t];
    }
    __syncthreads();
    for (int x = threadIdx.x; x < kRows * (D / 4); x += kThreads) {
      const int r = x / (D / 4), c = 4 * (x % (D / 4));
      float most = kNone, l = 0.f;
      for (int u = 0; u < W; ++u) most = fmaxf(most, s_ref[u * kRows + r]);
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int u = 0; u < W; ++u) {
        if (s_ref[u * kRows + r] == kNone) continue;
        const float f = half_factor(s_ref[u * kRows + r] - most);
        const float4 y = *reinterpret_cast<const float4 *>(s_part + (u * kRows + r) * M::kStride + c);
        l += f * s_sum[u * kRows + r] * f;
        v.x += f * y.x * f, v.y += f * y.y * f, v.z += f * y.z * f, v.w += f * y.w * f;
      }
      *reinterpret_cast<float4 *>(s_merged + r * M::kStride + c) = v;
      if (c == 0) s_mref[r] = most, s_msum[r] = l;
    }
    __syncthreads();
  };

  // ---- the band: exact rows
  // This thread's part of the outputs: rows 16 t + n, coordinates 16 wave + 4 j .. + 3.
  float4 other[NT];
  float other_ref[NT], other_sum[NT];
  for (int t = 0; t < NT; ++t) other[t] = make_float4(0.f, 0.f, 0.f, 0.f), other_ref[t] = kNone, other_sum[t] = 0.f;
  if (span.banded) {
    y.clear();
    Band<D, WIDE, NT> band(a, b, kv, lane);
    for (int t = 0; t < NT; ++t) band.set_queries(t, q[t]);
    for (int tb = (span.low & ~31) + kRound * wave; tb < span.sink1; tb += kRound * W)
      band.attend(tb, span.low, span.sink1, row_lo, row_hi, y);
    for (int tb = (span.rec0 & ~31) + kRound * wave; tb < g.t1; tb += kRound * W) band.attend(tb, span.rec0, g.t1, row_lo, row_hi, y);
    float none[NT];
    for (int t = 0; t < NT; ++t) none[t] = 0.f;
    merge_waves([](const int o, const int m) { return q4::out_coord<D>(o, m & 3, m >> 2); }, none);
    for (int t = 0; t < NT; ++t) {
      other[t] = *reinterpret_cast<const float4 *>(s_merged + (16 * t + n) * M::kStride + 16 * (wave & (kTiles - 1)) + 4 * j);
      other_ref[t] = s_mref[16 * t + n];
      other_sum[t] = s_msum[16 * t + n];
    }
    __syncthreads();
  }

  y.clear();
  float shift[NT];
  for (int t = 0; t < NT; ++t) shift[t] = 0.f;
  if (span.codes) {
    // ---- q' = q R_K^-T: each wave makes 16 of its coordinates for all rows
    const void *tk = transform_of(a.t_k_inv_t, kv, D, a.t_bf16);
    const bool makes = wave < kTiles;
    float raw[kSteps][8], top_t = 0.f;
    for (int s = 0; s < kSteps; ++s)
      for (int e = 0; e < 8; ++e) {
        raw[s][e] = makes ? t1_value(tk, static_cast<size_t>(32 * s + 8 * j + e) * D + 16 * wave + n, a.t_bf16) : 0.f;
        top_t = fmaxf(top_t, fabsf(raw[s][e]));
      }
    stage_book<L, kThreads>(s_key, a.cb_k, a.cb_fp8, kv);
    if constexpr (!SQ) stage_book<L, kThreads>(s_value, a.cb_v, a.cb_fp8, kv);
    top_t = wave_max(top_t);
    if (lane == 0) s_tops[wave] = top_t;
    __syncthreads();
    for (int u = 0; u < W; ++u) top_t = fmaxf(top_t, s_tops[u]);
    const int up_t = up_to_14(top_t);
    half8_t th[kSteps], tl[kSteps];
    for (int s = 0; s < kSteps; ++s)
      for (int e = 0; e < 8; ++e) {
        _Float16 hi, lo;
        split_half(ldexpf(raw[s][e], up_t), hi, lo);
        th[s][e] = hi, tl[s][e] = lo;
      }
    float alpha[NT];
    for (int t = 0; t < NT; ++t) {
      float top = 0.f, dot = 0.f;
      bool finite = true;
      for (int s = 0; s < kSteps; ++s)
        for (int e = 0; e < 8; ++e) {
          finite = finite && fabsf(q[t][s][e]) < __builtin_inff();
          top = fmaxf(top, fabsf(q[t][s][e]));
          dot = __builtin_fmaf(q[t][s][e], a.kbar[kv * D + 32 * s + 8 * j + e], dot);
        }
      shift[t] = add_rows32(add_rows16(dot)) * a.qscale;
      top = max_rows32(max_rows16(finite ? top : __builtin_inff()));
      const bool usable = top < __builtin_inff();
      const int up = up_to_14(top);
      float4_t out = {0.f, 0.f, 0.f, 0.f};
      for (int s = 0; s < kSteps; ++s) {
        half8_t qh, ql;
        for (int e = 0; e < 8; ++e) {
          _Float16 hi, lo;
          split_half(usable ? ldexpf(q[t][s][e], up) : __builtin_nanf(""), hi, lo);  // a row that is not finite: NaN scores
          qh[e] = hi, ql[e] = lo;
        }
        out = __builtin_amdgcn_mfma_f32_16x16x32_f16(th[s], qh, out, 0, 0, 0);
        out = __builtin_amdgcn_mfma_f32_16x16x32_f16(tl[s], qh, out, 0, 0, 0);
        if constexpr (WIDE) out = __builtin_amdgcn_mfma_f32_16x16x32_f16(th[s], ql, out, 0, 0, 0);
      }
      // |out| <= D 2^28: times 2^-20 it fits fp16
      if (makes) {
        _Float16 part[2][4];
        for (int i = 0; i < 4; ++i) split_half(out[i] * 0x1p-20f, part[0][i], part[1][i]);
        for (int p = 0; p < kParts; ++p)
          *reinterpret_cast<lut::half4_t *>(s_q + (p * kRows + 16 * t + n) * M::kQStride + 16 * wave + 4 * j) =
              lut::half4_t{part[p][0], part[p][1], part[p][2], part[p][3]};
      }
      alpha[t] = fminf(fmaxf(ldexpf(a.qscale, 20 - up - up_t), 0x1p-126f), 0x1p126f);
    }
    __syncthreads();
    half8_t qf[NT][kSteps][kParts];  // in the codewords' order: coordinates (D / 4) j + 8 s + e
    for (int t = 0; t < NT; ++t)
      for (int s = 0; s < kSteps; ++s)
        for (int p = 0; p < kParts; ++p)
          qf[t][s][p] = *reinterpret_cast<const half8_t *>(s_q + (p * kRows + 16 * t + n) * M::kQStride + (D / 4) * j + 8 * s);

    // ---- rounds of 32 tokens: block-table entries two rounds ahead, codes one
    const int bs = a.layout.block_size;
    const int bs_log = (bs & (bs - 1)) == 0 ? 31 - __builtin_clz(bs) : -1;
    const int32_t *table = a.layout.block_table ? a.layout.block_table + static_cast<size_t>(b) * a.layout.blocks_per_seq : nullptr;
    const long long first_block = static_cast<long long>(b) * a.layout.blocks_per_seq;
    int look = (c0 & ~31) + kRound * wave + (lane & 31), phys = 0, phys_row = 0;
    auto look_up = [&]() {
      // nothing outside the attended tokens' own runs of 16 (elsewhere: tokens) is looked up
      const int tok = ALIGNED ? min(max(look & ~15, c0 & ~15), (c1 - 1) & ~15) + (look & 15) : min(max(look, c0), c1 - 1);
      const int blk = bs_log >= 0 ? tok >> bs_log : tok / bs;
      phys_row = tok - blk * bs;
      phys = table ? table[blk] : static_cast<int>(first_block + blk);
      look += kRound * W;
    };
    struct Round {
      uint32_t kw[2][kWords], vw[8], sq;
      uint16_t rho;
    };
    const uint32_t k_lane = (L / 4) * j, v_lane = 4 * (n & (L / 4 - 1));
    auto request = [&](Round &r) {
      size_t mine;
      auto read_key = [&](const int x, const size_t row) {
        const uint8_t *p = a.k_codes + row * L + k_lane;
        if constexpr (D == 128) {
          const uint2 w = *reinterpret_cast<const uint2 *>(p);
          r.kw[x][0] = w.x, r.kw[x][1] = w.y;
        } else {
          r.kw[x][0] = *reinterpret_cast<const uint32_t *>(p);
        }
      };
      if constexpr (ALIGNED) {
        size_t first[2];
        for (int x = 0; x < 2; ++x) {
          const int p = __builtin_amdgcn_readlane(phys, 16 * x), row = __builtin_amdgcn_readlane(phys_row, 16 * x);
          first[x] = (static_cast<size_t>(p) * a.num_kv_heads + kv) * bs + row;
          read_key(x, first[x] + n);
        }
        for (int e = 0; e < 8; ++e)
          r.vw[e] = *reinterpret_cast<const uint32_t *>(a.v_codes + (first[e >> 2] + 4 * j + (e & 3)) * L + v_lane);
        mine = first[(lane >> 4) & 1] + n;
      } else {
        mine = (static_cast<size_t>(phys) * a.num_kv_heads + kv) * bs + phys_row;
        s_row_at[lane & 31] = mine;
        __builtin_amdgcn_wave_barrier();
        for (int x = 0; x < 2; ++x) read_key(x, s_row_at[16 * x + n]);
        for (int e = 0; e < 8; ++e)
          r.vw[e] = *reinterpret_cast<const uint32_t *>(a.v_codes + s_row_at[16 * (e >> 2) + 4 * j + (e & 3)] * L + v_lane);
        __builtin_amdgcn_wave_barrier();
      }
      r.rho = 0, r.sq = 0;
      if (a.k_scales) r.rho = a.k_scales[mine];
      if constexpr (SQ) r.sq = reinterpret_cast<const uint32_t *>(a.v_sq)[mine];
    };
    const int inner_lo = g.first_pos(a, g.row1 - 1), inner_hi = g.last_pos(a, g.row0) + 1;  // seen by all rows
    Round cur;
    look_up();
    request(cur);
    look_up();
    for (int tb = (c0 & ~31) + kRound * wave; tb < c1; tb += kRound * W) {
      const Round now = cur;
      request(cur);  // past the end: the last tokens again
      look_up();
      const bool scaled = SQ || a.k_scales;
      if (scaled) {  // lane l: token l mod 32
        const int tok = tb + (lane & 31);
        const bool in = tok >= c0 && tok < c1;
        float rho = a.k_scales ? bf16_bits_to_float(now.rho) : 1.f;
        if constexpr (SQ) {
          const Grid v = grid_of(now.sq, in, rho);
          if (lane < 32) s_tok[kRound + lane] = v.scale, s_tok[2 * kRound + lane] = v.offset, s_tok[3 * kRound + lane] = v.expo;
        }
        if (lane < 32) s_tok[lane] = rho;
        __builtin_amdgcn_wave_barrier();
      }
      float4_t s[NT][2];
      for (int x = 0; x < 2; ++x) {
        for (int t = 0; t < NT; ++t) s[t][x] = float4_t{0.f, 0.f, 0.f, 0.f};
        for (int st = 0; st < kSteps; ++st) {
          uint2 w[2];
          for (int y = 0; y < 2; ++y) {
            const int gr = 2 * st + y;
            w[y] = s_key[((L / 4) * j + gr) * kCodebookSize + ((now.kw[x][gr / 4] >> (8 * (gr & 3))) & 0xffu)];
          }
          const half8_t kf = __builtin_bit_cast(half8_t, make_uint4(w[0].x, w[0].y, w[1].x, w[1].y));
          for (int t = 0; t < NT; ++t)
            for (int p = 0; p < kParts; ++p) s[t][x] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf, qf[t][st][p], s[t][x], 0, 0, 0);
        }
        if (scaled) {
          const float4 rho = *reinterpret_cast<const float4 *>(&s_tok[16 * x + 4 * j]);
          for (int t = 0; t < NT; ++t) s[t][x][0] *= rho.x, s[t][x][1] *= rho.y, s[t][x][2] *= rho.z, s[t][x][3] *= rho.w;
        }
      }
      if (!(tb >= max(inner_lo, c0) && tb + kRound <= min(inner_hi, c1))) {
        for (int t = 0; t < NT; ++t)
          for (int x = 0; x < 2; ++x)
            for (int i = 0; i < 4; ++i) {
              const int tok = tb + 16 * x + 4 * j + i;
              const bool seen = tok >= max(c0, row_lo[t]) && tok < min(c1, row_hi[t]);
              s[t][x][i] = seen ? s[t][x][i] : kNone;
            }
      }
      float scale[8], offset[8], expo[8];
      if constexpr (SQ) {
        for (int x = 0; x < 2; ++x) {
          const float4 u = *reinterpret_cast<const float4 *>(&s_tok[kRound + 16 * x + 4 * j]);
          const float4 v = *reinterpret_cast<const float4 *>(&s_tok[2 * kRound + 16 * x + 4 * j]);
          const float4 w = *reinterpret_cast<const float4 *>(&s_tok[3 * kRound + 16 * x + 4 * j]);
          scale[4 * x] = u.x, scale[4 * x + 1] = u.y, scale[4 * x + 2] = u.z, scale[4 * x + 3] = u.w;
          offset[4 * x] = v.x, offset[4 * x + 1] = v.y, offset[4 * x + 2] = v.z, offset[4 * x + 3] = v.w;
          expo[4 * x] = w.x, expo[4 * x + 1] = w.y, expo[4 * x + 2] = w.z, expo[4 * x + 3] = w.w;
        }
        __builtin_amdgcn_wave_barrier();
      }
      float bound[NT];
      for (int t = 0; t < NT; ++t) {
        bound[t] = kNone;
        if constexpr (SQ) {
          for (int e = 0; e < 8; ++e) bound[t] = fmaxf(bound[t], __builtin_fmaf(s[t][e >> 2][e & 3], alpha[t], expo[e]));
        } else {
          for (int e = 0; e < 8; ++e) bound[t] = fmaxf(bound[t], s[t][e >> 2][e & 3]);
          bound[t] *= alpha[t];
        }
      }
      y.raise(bound);
      half8_t pf[NT][kParts];
      for (int t = 0; t < NT; ++t) {
        const float r = ref[t] == kNone ? 0.f : ref[t];
        for (int e = 0; e < 8; ++e) {
          float p = exp2_raw(__builtin_fmaf(s[t][e >> 2][e & 3], alpha[t], -r));
          sum[t] += p;
          if constexpr (SQ) {
            off_sum[t] = __builtin_fmaf(p, offset[e], off_sum[t]);
            p *= scale[e];
          }
          if constexpr (WIDE) {
            _Float16 hi, lo;
            split_half(p, hi, lo);
            pf[t][0][e] = hi, pf[t][1][e] = lo;
          } else {
            pf[t][0][e] = static_cast<_Float16>(p);
          }
        }
      }
      for (int p = 0; p < kTiles / 4; ++p) {
        uint2 w[8];
        for (int e = 0; e < 8; ++e) {
          const uint32_t code = D == 128 ? (now.vw[e] >> (16 * (n >> 3) + 8 * p)) & 0xffu : (now.vw[e] >> (8 * (n >> 2))) & 0xffu;
          const int group = value_group<D>(n, p);
          if constexpr (SQ) w[e] = centred_levels(code);
          else w[e] = s_value[group * kCodebookSize + code];
        }
        for (int c = 0; c < 4; ++c) {
          uint32_t u[4];
          for (int x = 0; x < 4; ++x)
            u[x] = c < 2 ? half_pair(w[2 * x].x, w[2 * x + 1].x, c & 1) : half_pair(w[2 * x].y, w[2 * x + 1].y, c & 1);
          const half8_t vf = __builtin_bit_cast(half8_t, make_uint4(u[0], u[1], u[2], u[3]));
          for (int t = 0; t < NT; ++t)
            for (int x = 0; x < kParts; ++x)
              acc[t][4 * p + c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, pf[t][x], acc[t][4 * p + c], 0, 0, 0);
        }
      }
    }
    if constexpr (SQ) {
      for (int t = 0; t < NT; ++t) {
        off_sum[t] = add_rows32(add_rows16(off_sum[t]));
        for (int o = 0; o < kTiles; ++o) acc[t][o] += off_sum[t];
      }
    }
  }

  // ---- back through R_V: each wave makes 16 coordinates of all rows
  const void *tv = transform_of(a.t_v, kv, D, a.t_bf16);
  Eight raw[kSteps];
  float top_t = 0.f;
  for (int s = 0; s < kSteps; ++s) {
    raw[s] = load_eight(tv, static_cast<size_t>(16 * (wave & (kTiles - 1)) + n) * D + 32 * s + 8 * j, a.t_bf16);
    for (int e = 0; e < 8; ++e) top_t = fmaxf(top_t, fabsf(raw[s].x[e]));
  }
  __syncthreads();  // the codebooks are done with
  merge_waves([&](const int o, const int m) { return code_coord<D>(o, m); }, shift);
  const int up_t = up_to_14(wave_max(top_t));
  half8_t th[kSteps], tl[kSteps];
  for (int s = 0; s < kSteps; ++s)
    for (int e = 0; e < 8; ++e) {
      _Float16 hi, lo;
      split_half(ldexpf(raw[s].x[e], up_t), hi, lo);
      th[s][e] = hi, tl[s][e] = lo;
    }
  const q4::TileRows<D, kRows> place{a, g};
  float *const part = place.part();
  for (int t = 0; t < NT; ++t) {
    const int r = 16 * t + n;
    float x[kSteps][8], top = 0.f;
    for (int s = 0; s < kSteps; ++s)
      for (int y = 0; y < 2; ++y) {
        const float4 v = *reinterpret_cast<const float4 *>(s_merged + r * M::kStride + 32 * s + 8 * j + 4 * y);
        x[s][4 * y] = v.x, x[s][4 * y + 1] = v.y, x[s][4 * y + 2] = v.z, x[s][4 * y + 3] = v.w;
        top = fmaxf(fmaxf(top, fmaxf(fabsf(v.x), fabsf(v.y))), fmaxf(fabsf(v.z), fabsf(v.w)));
      }
    const int up = up_to_14(max_rows32(max_rows16(top)));
    float4_t o = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < kSteps; ++s) {
      half8_t xh, xl;
      for (int e = 0; e < 8; ++e) {
        _Float16 hi, lo;
        split_half(ldexpf(x[s][e], up), hi, lo);
        xh[e] = hi, xl[e] = lo;
      }
      o = __builtin_amdgcn_mfma_f32_16x16x32_f16(th[s], xh, o, 0, 0, 0);
      o = __builtin_amdgcn_mfma_f32_16x16x32_f16(tl[s], xh, o, 0, 0, 0);
      o = __builtin_amdgcn_mfma_f32_16x16x32_f16(th[s], xl, o, 0, 0, 0);
    }
    if (wave >= kTiles || r >= place.rows_here()) continue;
    for (int i = 0; i < 4; ++i) o[i] = ldexpf(o[i], -up - up_t);
    float most = s_mref[r], l = s_msum[r];
    float4 v = make_float4(o[0], o[1], o[2], o[3]);
    if (other_ref[t] != kNone) {  // the band's share
      const float to = fmaxf(most, other_ref[t]);
      const float f = most == kNone ? 0.f : half_factor(most - to), h = half_factor(other_ref[t] - to);
      v = make_float4(f * v.x * f + h * other[t].x * h, f * v.y * f + h * other[t].y * h, f * v.z * f + h * other[t].z * h,
                      f * v.w * f + h * other[t].w * h);
      l = f * l * f + h * other_sum[t] * h;
      most = to;
    }
    const int c = 16 * wave + 4 * j;
    if (part) {
      q4::publish4(part + r * D + c, v);
      if (c == 0) q4::publish2(part + kRows * D + 2 * r, most, l);
    } else {
      q4::store_out(a, place.out_at(r) + c, place.scaled(v, place.inverse(r, most, l)));
    }
  }
  if (!part) return;
  __syncthreads();  // the merged rows are read
  int *const s_last = reinterpret_cast<int *>(s_lds + M::kLast);
  q4::merge_splits<D, NT, W, false>(a, g, {s_part, nullptr, nullptr, s_inv, s_last}, n);
}

hipError_t launch_few(const ChunkArgs &a, const ChunkPlan &plan, hipStream_t stream) {
  const unsigned groups = static_cast<unsigned>(a.batch) * a.num_kv_heads * plan.row_tiles * plan.n_split;
  auto go = [&](auto d, auto wide, auto nt, auto sq, auto aligned) {
    chunk_rows_kernel<d(), wide(), nt(), sq(), aligned()><<<groups, 64 * W, 0, stream>>>(a);
    return hipGetLastError();
  };
  using std::false_type;
  using std::integral_constant;
  using std::true_type;
  auto by_blocks = [&](auto d, auto wide, auto nt, auto sq) {
    return a.layout.block_size % 16 == 0 ? go(d, wide, nt, sq, true_type{}) : go(d, wide, nt, sq, false_type{});
  };
  auto by_values = [&](auto d, auto wide, auto nt) { return a.v_sq ? by_blocks(d, wide, nt, true_type{}) : by_blocks(d, wide, nt, false_type{}); };
  auto by_rows = [&](auto d, auto wide) {
    return plan.tile_rows == 16 ? by_values(d, wide, integral_constant<int, 1>{}) : by_values(d, wide, integral_constant<int, 2>{});
  };
  auto by_type = [&](auto d) { return a.q_bf16 ? by_rows(d, false_type{}) : by_rows(d, true_type{}); };
  return a.head_dim == 128 ? by_type(integral_constant<int, 128>{}) : by_type(integral_constant<int, 64>{});
}

}  // namespace

// Rows per workgroup: up to 16 (32) rows take one (two) matrix tiles, the workgroup's waves dividing the
// tokens; more rows take 16 or 32 a wave, 128 or 256 a workgroup (both sides measured: chunk_tile.hip).
ChunkPlan plan_chunk(const int batch, const int n_q, const int num_q_heads, const int num_kv_heads, const int head_dim,
                     const int max_seq_len, const int window) {
  ChunkPlan p{};
  const long long rows = static_cast<long long>(n_q) * (num_q_heads / num_kv_heads);
  p.tile_rows = rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 128 ? 128 : 256;
  p.row_tiles = static_cast<int>((rows + p.tile_rows - 1) / p.tile_rows);
  const long long tiles = static_cast<long long>(p.row_tiles) * batch * num_kv_heads;
  const long long span = window > 0 ? std::min<long long>(max_seq_len, static_cast<long long>(window) + n_q) : max_seq_len;
  const long long limit = p.tile_rows >= 128 ? q4::kMaxSplitsTiled : q4::kMaxSplits;
  auto splits = [&](const long long s) {
    // until the CUs have a workgroup each (so no more counters are used than there are)
    long long n = std::min({limit, (s + 511) / 512, 256 / tiles});
    // One workgroup merges a tile's splits, for about as long a split as 32 (of 256 rows: 45) of its tokens take.
    const double per = p.tile_rows == 128 ? 32. : 45.;
    if (p.tile_rows >= 128) n = std::min(n, static_cast<long long>(std::sqrt(static_cast<double>(s) / per)));
    return static_cast<int>(std::max(1LL, n));
  };
  static_assert(q4::kMaxCounters >= 256, "a split tile has a counter");
  p.n_split = splits(span);
  p.off_part = q4::kMaxCounters * sizeof(int);
  const int all = splits(max_seq_len);  // longer spans have no fewer: the most of any window
  if (all > 1) {
    const size_t part = static_cast<size_t>(tiles) * all * p.tile_rows * (head_dim + 2) * sizeof(float);
    p.total = p.off_part + ((part + 255) & ~static_cast<size_t>(255));
  }
  return p;
}

hipError_t launch_chunk(const ChunkArgs &a, const ChunkPlan &plan, hipStream_t stream) {
  return plan.tile_rows == 256   ? launch_chunk_wide(a, plan, stream)
         : plan.tile_rows == 128 ? launch_chunk_tile(a, plan, stream)
                                 : launch_few(a, plan, stream);
}

}  // namespace novakv
