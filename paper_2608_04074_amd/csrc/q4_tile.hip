// Attention of many query rows over a cache held in 4 bits (nova_kv_q4_attn with
// bf16 queries and more than 32 rows per KV head: chunks of prompts).
//
// A workgroup of eight (four) waves takes 256 (128) rows, 32 a wave, and 128 (64)
// tokens at a time. The waves unpack the tokens' rows once, between them, to fp16
// keys and values in LDS, in the order in which the matrix cores take them, the
// next ones while these are used. Unpacked, a score needs no more than its
// multiply-add into the exponent: 8 vector instructions each, an exponential
// among them (10.5 with four waves, which unpack for half the rows), where sums over
// the codes, as in q4_attn.hip, took 14.5 (but no LDS, and no rounding of keys and values).
//
// Two sequences' 2048 queries over 8192 tokens (32 query, 8 KV heads of 128): 525 us, 916
// TFLOP/s. Vector (about 320 us) and matrix instructions (192 us) bound it, which add
// on a SIMD. Four waves take 620 us, and the same without the LDS took 1211; with few tiles
// the smaller ones win, by parallelism and by a merge of splits over more workgroups.
//
// Keys and values are divided by 2^7 times a power of two at or above the largest
// magnitude of the 64 tokens (each side its own), which the exponent and the
// output take back: a scale's and an offset's 8 bits then fit fp16, and one
// packed multiply-add unpacks two codes (fp16 denormals as they lie, c * 2^-24)
// with one rounding: half a step of fp16, 2^-12 of the power of two above the number,
// or of the smallest normal one, 2^-18 of the tokens' power, below. Tokens at most 2^5 apart
// keep 2^-12 of their row's largest so; where 64 tokens are further apart, each has a power of its own, so
// that no other token, hidden or of no weight, takes bits of it.
// (2^7 is the least that keeps 15 scales, at most four times the power, in fp16.)
#include <type_traits>

#include "q4_common.h"

namespace novakv {

namespace {

using namespace q4;

constexpr int kRowTiles = 2;
constexpr float kTop = 6.f, kSlack = 8.f;  // log2 of the largest probability after a rescale, and how far it may grow

// The same value in every lane, in a scalar register.
__device__ __forceinline__ int uniform(const int x) { return __builtin_amdgcn_readfirstlane(x); }
// Exponent of a power of two above a magnitude (half of it beyond 2^127) whose biased exponent is e; at least 2^least.
__device__ __forceinline__ int power_above(const int e, const int least) { return min(max(e - 126, least), 127); }
// Of keys, so that 2^17 over it is a float; of values, so that sums of probabilities over it stay in range.
constexpr int kLeastKey = -110, kLeastValue = -90;
// Exponents of 64 tokens this far apart at most share one: the least keeps 2^-12 of its largest.
constexpr int kSpread = 5;
constexpr int kFinite = 0x7f7fffff;  // bits of the largest float
__device__ __forceinline__ float power_of_two(const int e) { return __builtin_amdgcn_ldexpf(1.f, e); }

// W: waves of a workgroup, a multiple of four. ALIGNED: blocks of a multiple of 16 rows.
template <int D, int W, bool ALIGNED>
__global__ __launch_bounds__(64 * W, 2) void q4_tile_kernel(const Q4AttnArgs a) {
  constexpr int kWaves = W, kParts = W / 4, kTokens = 64 * kParts;  // tokens of a round, in parts of 64
  constexpr int kSteps = D / 32, kTiles = D / 16, kKeyWords = D / 32;
  constexpr int kKeys = 4 * kSteps * 64, kBuffer = kKeys + 2 * kTiles * 64;  // fragments of 16 bytes: keys, then values
  using Lds = FinishLds<D, kRowTiles, kWaves, true>;
  static_assert(2 * kParts * kBuffer * 16 >= Lds::kMerge * 4, "the splits' weights take the tokens' place");
  __shared__ half8_t s_tokens[2][kParts * kBuffer];
  __shared__ uint32_t s_rows[ALIGNED ? 1 : kWaves][32];
  __shared__ __align__(16) uint32_t s_pack[kWaves][64];
  // [round mod 3][32 tokens][keys, values]: the largest magnitude, and by how many bits the smallest is below kFinite
  __shared__ __align__(16) float s_mag[3][2 * kParts][2][2];
  __shared__ __align__(16) float s_unit[2][2][kTokens];  // [round mod 2][keys, values]: a token's power of two
  // [round mod 2]: the part's exponents of keys and values, 128 added, or (bit 16) that its tokens have their own
  __shared__ int s_shared[2][kParts];
  __shared__ uint32_t s_valid[3][2 * kParts];
  __shared__ float s_inv[Lds::kRows];
  __shared__ int s_last;

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int lane = threadIdx.x & 63, n = lane & 15, j = lane >> 4;
  // the wave unpacks, of a round's part, 16 keys and half of the coordinates of 32 values
  const int group = wave >> 1, part = wave & 1, own = wave >> 2;
  Tile g;
  place_tile(a, Lds::kRows, g);
  if (!find_span(a, Lds::kRows, kTokens, g)) return;
  const int b = g.b, kv = g.kv;
  const int row0 = g.row0 + 16 * kRowTiles * wave, row1 = min(row0 + 16 * kRowTiles, g.rows_valid);
  const bool idle = row0 >= g.rows_valid;
  const int wave_lo = idle ? 0 : g.first_pos(a, row0), wave_hi = idle ? 0 : g.last_pos(a, row1 - 1) + 1;
  const int inner_lo = idle ? 0 : g.first_pos(a, row1 - 1), inner_hi = idle ? 0 : g.last_pos(a, row0) + 1;

  // Requests of the tokens' codes, scales and offsets: lane l holds row, scale and
  // offset of token l % 32 of the wave's 32 (key: l < 32, value: l >= 32).
  const int bs = a.layout.block_size, bps = a.layout.blocks_per_seq;
  const uint32_t block_rows = static_cast<uint32_t>(a.num_kv_heads) * bs, head_row = static_cast<uint32_t>(kv) * bs;
  const int32_t *table = a.layout.block_table ? a.layout.block_table + static_cast<size_t>(b) * bps : nullptr;
  const uint32_t *sq = reinterpret_cast<const uint32_t *>(lane < 32 ? a.k_sq : a.v_sq);
  int look = g.t0 + 32 * group + (lane & 31);
  int look_blk = look / bs, look_row = look - look_blk * bs;
  const int step_blk = kTokens / bs, step_row = kTokens - step_blk * bs;
  int phys = -1, phys_tok = 0, phys_row = 0;
  auto look_up = [&]() {
    phys = -1;
    phys_tok = look;
    phys_row = look_row;
    if (look_blk < bps) {
      const long long own = static_cast<long long>(b) * bps + look_blk;
      phys = table ? table[look_blk] : own < a.num_blocks ? static_cast<int>(own) : -1;
    }
    look += kTokens;
    look_blk += step_blk;
    look_row += step_row;
    if (look_row >= bs) look_row -= bs, ++look_blk;
  };
  struct Round {
    uint32_t kw[kKeyWords], vw[8], sq;
    bool ok;
  };
  const uint32_t k_lane = n * (D / 2) + 4 * kKeyWords * j, v_lane = 4 * j * (D / 2) + 4 * (n & (D / 8 - 1));
  auto read_key = [&](Round &r, const uint8_t *k) {
    if constexpr (D == 128) {
      const uint4 w = *reinterpret_cast<const uint4 *>(k);
      r.kw[0] = w.x, r.kw[1] = w.y, r.kw[2] = w.z, r.kw[3] = w.w;
    } else {
      const uint2 w = *reinterpret_cast<const uint2 *>(k);
      r.kw[0] = w.x, r.kw[1] = w.y;
    }
  };
  auto request = [&](Round &r) {
    const bool held = static_cast<uint32_t>(phys) < static_cast<uint32_t>(a.num_blocks);
    r.ok = held && phys_tok < g.t1 && phys_tok >= g.lo;
    uint32_t row = static_cast<uint32_t>(phys) * block_rows + head_row + phys_row;
    if constexpr (ALIGNED) {  // 16 tokens' rows follow each other; in the place of a block that holds nothing, the pool's first
      if (!held) row = lane & 15;
      const size_t first[2] = {static_cast<size_t>(static_cast<uint32_t>(__builtin_amdgcn_readlane(row, 0))) * (D / 2),
                               static_cast<size_t>(static_cast<uint32_t>(__builtin_amdgcn_readlane(row, 16))) * (D / 2)};
      read_key(r, a.k_codes + first[part] + k_lane);
      for (int e = 0; e < 8; ++e)
        r.vw[e] = *reinterpret_cast<const uint32_t *>(a.v_codes + first[e >> 2] + (v_lane + (e & 3) * (D / 2)));
    } else {
      if (!r.ok) row = 0;
      s_rows[wave][lane & 31] = row;
      __builtin_amdgcn_wave_barrier();
      read_key(r, a.k_codes + static_cast<size_t>(s_rows[wave][16 * part + n]) * (D / 2) + 4 * kKeyWords * j);
      for (int e = 0; e < 8; ++e)
        r.vw[e] = *reinterpret_cast<const uint32_t *>(
            a.v_codes + static_cast<size_t>(s_rows[wave][16 * (e >> 2) + 4 * j + (e & 3)]) * (D / 2) + 4 * (n & (D / 8 - 1)));
      __builtin_amdgcn_wave_barrier();
    }
    r.sq = sq[row];
  };
  auto biased_of = [](const float mag) { return __builtin_bit_cast(int, mag) >> 23; };  // of mag >= 0
  // scale and offset of the lane's token, 0 for hidden tokens
  auto scale_of = [&](const Round &r, float &scale, float &offset) {
    scale = r.ok ? __uint_as_float(r.sq << 16) : 0.f;
    offset = r.ok ? __uint_as_float(r.sq & 0xffff0000u) : 0.f;
    // the largest magnitude of the row (of code 0 or 15); NaN or infinity where one is
    const float last = __builtin_fmaf(15.f, scale, offset);
    return last - last == 0.f ? fmaxf(fabsf(offset), fabsf(last)) : fabsf(last);
  };
  auto announce = [&](const Round &r, const int slot) {
    float scale, offset;
    const float mag = scale_of(r, scale, offset);
    // of the two waves with these tokens, part 0 seeks the largest, part 1 the smallest that is not 0
    float most = mag > 0.f && mag < __builtin_inff() ? part ? __builtin_bit_cast(float, kFinite - __builtin_bit_cast(int, mag)) : mag : 0.f;
    most = fmaxf(most, lut::row_ror<8>(most));
    most = fmaxf(most, lut::row_ror<4>(most));
    most = fmaxf(most, lut::row_ror<2>(most));
    most = fmaxf(most, lut::row_ror<1>(most));
    most = max_rows16(most);  // over the 32 lanes of a side
    const uint32_t valid = static_cast<uint32_t>(__ballot(r.ok));
    if ((lane & 31) == 0) s_mag[slot][group][lane >> 5][part] = most;
    if (part == 0 && lane == 0) s_valid[slot][group] = valid;
  };
  // the exponents of a round's part, and whether its tokens have their own
  auto exponents = [&](const int slot, const int y, int &ek, int &ev) {
    auto of = [&](const int side, const int least, int &e) {
      const float *const m[2] = {s_mag[slot][2 * y][side], s_mag[slot][2 * y + 1][side]};
      const int most = uniform(__builtin_bit_cast(int, fmaxf(m[0][0], m[1][0]))), left = uniform(__builtin_bit_cast(int, fmaxf(m[0][1], m[1][1])));
      e = power_above(most >> 23, least);
      return e - power_above((kFinite - left) >> 23, least) > kSpread;
    };
    const bool k = of(0, kLeastKey, ek), v = of(1, kLeastValue, ev);
    return k || v;
  };
  auto unpack = [&](const Round &r, const int slot, const int buffer) {
    half8_t *const to = s_tokens[buffer] + own * kBuffer;
    int ek, ev;
    const bool spread = exponents(slot, own, ek, ev);
    float scale, offset;
    const float mag = scale_of(r, scale, offset);
    const bool odd = !(mag < __builtin_inff());
    // A value that is not finite would reach the rows it is hidden from (0 * NaN): its
    // token's key becomes NaN instead, and the value 0.
    const uint64_t odds = __ballot(odd);
    const uint32_t any_odd = static_cast<uint32_t>(odds) | static_cast<uint32_t>(odds >> 32);
    const bool token_odd = (any_odd >> (lane & 31)) & 1u;
    const int shared = lane < 32 ? ek : ev;
    const int e = spread ? min(power_above(odd ? 0 : biased_of(mag), lane < 32 ? kLeastKey : kLeastValue), shared) : shared;
    const float unit = power_of_two(-e);
    if (part == 0 && lane == 0) s_shared[buffer][own] = spread ? 128 | (128 << 8) | (1 << 16) : (ek + 128) | ((ev + 128) << 8);
    if (part == 0) s_unit[buffer][lane >> 5][32 * group + (lane & 31)] = power_of_two(e);
    scale = token_odd ? (lane < 32 ? __builtin_nanf("") : 0.f) : scale * (unit * 0x1p17f);  // s <= 4 / 15 / unit: below 2^15.1
    offset = token_odd ? 0.f : offset * (unit * 0x1p-7f);
    const lut::half2_t both = {static_cast<_Float16>(scale), static_cast<_Float16>(offset)};
    s_pack[wave][lane] = __builtin_bit_cast(uint32_t, both);
    __builtin_amdgcn_wave_barrier();
    // codes k and k + 4 of a word (of two tokens' halves), with their scales and offsets
    auto place = [](auto k, const uint32_t w, const uint32_t scales, const uint32_t offsets) {
      const _Float16 down = k() % 2 ? 0x1p-4f : 1.f;
      return __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(code_pair<k()>(w), __builtin_bit_cast(lut::half2_t, scales) * lut::half2_t{down, down},
                                                                    __builtin_bit_cast(lut::half2_t, offsets)));
    };
    using std::integral_constant;
    constexpr integral_constant<int, 0> c0{};
    constexpr integral_constant<int, 1> c1{};
    constexpr integral_constant<int, 2> c2{};
    constexpr integral_constant<int, 3> c3{};
    {  // key 16 part + n of the 32: fragment (token tile, step) holds eight coordinates of it a lane
      const uint32_t p = s_pack[wave][16 * part + n];
      const uint32_t s2 = __builtin_amdgcn_perm(p, p, 0x01000100u), o2 = __builtin_amdgcn_perm(p, p, 0x03020302u);
      for (int i = 0; i < kKeyWords; ++i) {
        const int word = kKeyWords * j + i;
        const uint32_t w = r.kw[i];
        to[((wave & 3) * kSteps + word / 4) * 64 + 16 * (word % 4) + n] = __builtin_bit_cast(
            half8_t, make_uint4(place(c0, w, s2, o2), place(c1, w, s2, o2), place(c2, w, s2, o2), place(c3, w, s2, o2)));
      }
    }
    // values: fragment (32 tokens, output tile) holds eight tokens of a coordinate a lane
    uint32_t s2[4], o2[4], pair[4];
    const uint32_t pick = D == 128 ? (part ? 0x07060302u : 0x05040100u) : n < 8 ? 0x05040100u : 0x07060302u;
    for (int h = 0; h < 2; ++h) {
      const uint4 p = *reinterpret_cast<const uint4 *>(&s_pack[wave][32 + 16 * h + 4 * j]);
      s2[2 * h] = __builtin_amdgcn_perm(p.y, p.x, 0x05040100u), o2[2 * h] = __builtin_amdgcn_perm(p.y, p.x, 0x07060302u);
      s2[2 * h + 1] = __builtin_amdgcn_perm(p.w, p.z, 0x05040100u), o2[2 * h + 1] = __builtin_amdgcn_perm(p.w, p.z, 0x07060302u);
    }
    __builtin_amdgcn_wave_barrier();
    for (int e = 0; e < 4; ++e) pair[e] = __builtin_amdgcn_perm(r.vw[2 * e + 1], r.vw[2 * e], pick);
    auto put = [&](auto k, const int o) {
      to[kKeys + ((group & 1) * kTiles + o) * 64 + lane] = __builtin_bit_cast(
          half8_t, make_uint4(place(k, pair[0], s2[0], o2[0]), place(k, pair[1], s2[1], o2[1]), place(k, pair[2], s2[2], o2[2]),
                              place(k, pair[3], s2[3], o2[3])));
    };
    if constexpr (D == 128) {
      put(c0, 4 * part);
      put(c1, 4 * part + 1);
      put(c2, 4 * part + 2);
      put(c3, 4 * part + 3);
    } else if (part == 0) {
      put(c0, 0);
      put(c1, 1);
    } else {
      put(c2, 2);
      put(c3, 3);
    }
  };

  const bool any = g.t0 < g.t1;
  Round cur;
  if (any) {
    look_up();
    request(cur);
    look_up();
  }

  // queries, times a power of two that brings the row's largest magnitude to [2^13, 2^14)
  half8_t qf[kRowTiles][kSteps];
  float alpha[kRowTiles], ref[kRowTiles], sum[kRowTiles];
  int row_lo[kRowTiles], row_hi[kRowTiles];
  float4_t acc[kRowTiles][kTiles];
  for (int t = 0; t < kRowTiles; ++t) {
    const int row = row0 + 16 * t + n;
    const bool on = row < g.rows_valid;
    const int i = row / a.gqa, h = row - i * a.gqa;
    row_hi[t] = on ? g.last_pos(a, row) + 1 : 0;
    row_lo[t] = on ? g.first_pos(a, row) : 0;
    const size_t at = ((static_cast<size_t>(b) * a.n_q + i) * a.num_q_heads + kv * a.gqa + h) * D + 8 * j;
    uint4 w[kSteps];
    float top = 0.f;
    bool finite = true;
    for (int s = 0; s < kSteps; ++s) {
      w[s] = make_uint4(0u, 0u, 0u, 0u);
      if (on) w[s] = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(a.q) + at + 32 * s);
      const uint32_t u[4] = {w[s].x, w[s].y, w[s].z, w[s].w};
      for (int e = 0; e < 4; ++e) {
        const float x = fabsf(__uint_as_float(u[e] << 16)), y = fabsf(__uint_as_float(u[e] & 0xffff0000u));
        finite = finite && x < __builtin_inff() && y < __builtin_inff();
        top = fmaxf(top, fmaxf(x, y));
      }
    }
    top = max_rows32(max_rows16(finite ? top : __builtin_inff()));
    const bool usable = top < __builtin_inff();
    const int up = usable && top > 0.f ? min(13 - ilogbf(top), 120) : 0;
    const float unit = ldexpf(1.f, up);
    for (int s = 0; s < kSteps; ++s) {
      const uint32_t u[4] = {w[s].x, w[s].y, w[s].z, w[s].w};
      for (int e = 0; e < 4; ++e) {
        const float x[2] = {__uint_as_float(u[e] << 16), __uint_as_float(u[e] & 0xffff0000u)};
        for (int y = 0; y < 2; ++y) {
          // a row that is not finite: NaN scores, of what it attends
          const int c = 2 * e + y;  // slots as value_pair has the nibbles: 0, 4, 1, 5, 2, 6, 3, 7
          qf[t][s][2 * (c & 3) + (c >> 2)] = static_cast<_Float16>(usable ? x[y] * unit : __builtin_nanf(""));
        }
      }
    }
    alpha[t] = fmaxf(ldexpf(a.qscale, -up), 0x1p-126f);
    ref[t] = kNone;
    sum[t] = 0.f;
    for (int o = 0; o < kTiles; ++o) acc[t][o] = float4_t{0.f, 0.f, 0.f, 0.f};
  }

  int slot = 1;  // of the round behind the one at hand
  if (any) {
    announce(cur, 0);
    __syncthreads();
    unpack(cur, 0, 0);
    request(cur);
    look_up();
    announce(cur, 1);
    __syncthreads();
  }
  for (int tb = g.t0, round = 0; tb < g.t1; tb += kTokens, ++round) {
    const int slot0 = slot == 0 ? 2 : slot - 1, slot2 = slot == 2 ? 0 : slot + 1;
    auto scores = [&](const half8_t *tokens, float4_t (&s)[kRowTiles][4]) {
      for (int x = 0; x < 4; ++x) {
        for (int t = 0; t < kRowTiles; ++t) s[t][x] = float4_t{0.f, 0.f, 0.f, 0.f};
        for (int st = 0; st < kSteps; ++st) {
          const half8_t k = tokens[(x * kSteps + st) * 64 + lane];
          for (int t = 0; t < kRowTiles; ++t) s[t][x] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, qf[t][st], s[t][x], 0, 0, 0);
        }
      }
    };
    auto attend = [&](const half8_t *tokens, float4_t (&s)[kRowTiles][4], const int y) {
      const int tb0 = tb + 64 * y;
      if (idle || tb0 >= wave_hi || tb0 + 64 <= wave_lo) return;
      const int shared = uniform(s_shared[round & 1][y]), ek = (shared & 255) - 128, ev = ((shared >> 8) & 255) - 128;
      const bool spread = shared >> 16;
      const float *const key_units = &s_unit[round & 1][0][64 * y + 4 * j], *const value_units = &s_unit[round & 1][1][64 * y + 4 * j];
      const uint32_t valid[2] = {static_cast<uint32_t>(uniform(s_valid[slot0][2 * y])), static_cast<uint32_t>(uniform(s_valid[slot0][2 * y + 1]))};
      const bool inner = (valid[0] & valid[1]) == 0xffffffffu && tb0 >= inner_lo && tb0 + 64 <= inner_hi;
      const float key_unit = power_of_two(ek), value_exp = static_cast<float>(ev);
      if (spread) {
        for (int t = 0; t < kRowTiles; ++t)
          for (int x = 0; x < 4; ++x)
            for (int i = 0; i < 4; ++i) s[t][x][i] *= key_units[16 * x + i];
      }
      if (!inner) {  // without branches in it the scores stay where they are, and inner rounds copy nothing
        for (int t = 0; t < kRowTiles; ++t)
          for (int x = 0; x < 4; ++x)
            for (int i = 0; i < 4; ++i) {
              const int m = 16 * x + 4 * j + i;
              const bool seen = ((valid[x >> 1] >> (m & 31)) & 1u) & (tb0 + m >= row_lo[t]) & (tb0 + m < row_hi[t]);
              s[t][x][i] = seen ? s[t][x][i] : kNone;
            }
      }
      float by[kRowTiles], bound[kRowTiles];
      bool over = false;
      for (int t = 0; t < kRowTiles; ++t) {
        float top = kNone;
        for (int x = 0; x < 4; ++x)
          for (int i = 0; i < 4; ++i) top = fmaxf(top, s[t][x][i]);
        by[t] = fminf(fmaxf(alpha[t] * 128.f * key_unit, 0x1p-126f), 0x1p127f);
        bound[t] = top * by[t] + value_exp;
        if (spread) {
          bound[t] = kNone;
          for (int x = 0; x < 4; ++x)
            for (int i = 0; i < 4; ++i)
              bound[t] = fmaxf(bound[t], __builtin_fmaf(s[t][x][i], by[t], static_cast<float>(biased_of(value_units[16 * x + i]) - 127)));
        }
        over |= bound[t] > ref[t] + (kTop + kSlack);
      }
      if (__any(over)) {
        for (int t = 0; t < kRowTiles; ++t) {
          const float most = max_rows32(max_rows16(bound[t]));
          const float to = fmaxf(ref[t], most - kTop);
          const float f = to == kNone ? 1.f : half_factor(ref[t] - to);
          ref[t] = to;
          for (int y = 0; y < 2; ++y) {
            sum[t] *= f;
            for (int o = 0; o < kTiles; ++o) acc[t][o] *= f;
          }
        }
      }
      half8_t pf[kRowTiles][2];
      auto probabilities = [&](const int t) {
        const float r = ref[t] == kNone ? 0.f : ref[t];
        // Summed in fp32, in front of the values' power of two and of the rounding to
        // fp16: a weight does not depend on its value, which may be far below others.
        for (int x = 0; x < 4; ++x)
          for (int i = 0; i < 4; ++i) {
            const float p = exp2_raw(__builtin_fmaf(s[t][x][i], by[t], -r));
            sum[t] += p;
            pf[t][x >> 1][4 * (x & 1) + i] = static_cast<_Float16>(p * value_units[16 * x + i]);
          }
      };
      for (int t = 0; t < kRowTiles; ++t) probabilities(t);
      for (int h = 0; h < 2; ++h)
        for (int o = 0; o < kTiles; ++o) {
          const half8_t v = tokens[kKeys + (h * kTiles + o) * 64 + lane];
          for (int t = 0; t < kRowTiles; ++t) acc[t][o] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, pf[t][h], acc[t][o], 0, 0, 0);
        }
    };
    const half8_t *tokens = s_tokens[round & 1];
    float4_t s[kRowTiles][4];
    scores(tokens, s);
    unpack(cur, slot, (round + 1) & 1);
    request(cur);  // past the end: hidden
    look_up();
    attend(tokens, s, 0);
    for (int y = 1; y < kParts; ++y) {
      scores(tokens + y * kBuffer, s);
      attend(tokens + y * kBuffer, s, y);
    }
    announce(cur, slot2);
    __syncthreads();
    slot = slot2;
  }

  for (int t = 0; t < kRowTiles; ++t) {
    sum[t] = add_rows32(add_rows16(sum[t]));
    if (sum[t] != sum[t]) ref[t] = fmaxf(ref[t], 0.f);  // NaN logits move no reference, but attend
    for (int o = 0; o < kTiles; ++o) acc[t][o] *= 128.f;
  }
  finish_rows<D, kRowTiles, kWaves, true>(a, g, {reinterpret_cast<float *>(s_tokens), nullptr, nullptr, s_inv, &s_last}, wave, lane, acc, ref,
                                          sum);
}

}  // namespace

hipError_t launch_q4_tile(const Q4AttnArgs &a, const Q4AttnPlan &plan, hipStream_t stream) {
  const unsigned groups = static_cast<unsigned>(a.batch) * a.num_kv_heads * plan.row_tiles * plan.n_split;
  auto go = [&](auto d, auto w, auto aligned) {
    q4_tile_kernel<d(), w(), aligned()><<<groups, 64 * w(), 0, stream>>>(a);
    return hipGetLastError();
  };
  using std::integral_constant;
  auto by_waves = [&](auto d, auto aligned) {
    return plan.waves == 8 ? go(d, integral_constant<int, 8>{}, aligned) : go(d, integral_constant<int, 4>{}, aligned);
  };
  auto by_size = [&](auto aligned) {
    return a.head_dim == 128 ? by_waves(integral_constant<int, 128>{}, aligned) : by_waves(integral_constant<int, 64>{}, aligned);
  };
  return a.layout.block_size % 16 == 0 ? by_size(std::true_type{}) : by_size(std::false_type{});
}

}  // namespace novakv
