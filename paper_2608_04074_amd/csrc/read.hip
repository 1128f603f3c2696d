// Reading a cache back: tokens of the 2-bit cache (nova_kv_read) and of the 4-bit cache
// (nova_kv_q4_read) as dense rows in fp32 or bf16.
//
// 2 bits: k = rho (r R_K^-1) + k_bar and v = s R_V^T, both a row of codewords times the
// transposed rows of a [D][D] array, on the fp16 matrix cores: a token's codewords, gathered
// from the codebook in LDS, are one operand as they come; the transform's rows stay in
// registers, as two fp16 parts (22 bits; one part where they are stored as bf16). The scalar
// arm's levels enter as level - 1.5, exact, and meet the transform's row sums with the
// token's offset + 1.5 scale.
#include <algorithm>
#include <type_traits>

#include "chunk_common.h"

namespace novakv {

namespace {

using namespace chunk;

// ------------------------------------------------------------------ 2 bits

constexpr int kWaves = 8, kThreads = 64 * kWaves;

// PARTS: fp16 parts of the transform.
template <int D, int PARTS>
__global__ __launch_bounds__(kThreads, 1) void read_kernel(const ReadArgs a) {
  constexpr int L = D / kGroupDim, kSteps = D / 32, kTiles = 4;  // a wave has 64 of the coordinates
  constexpr int kHalves = D / 64, kGroups = kWaves / kHalves;    // waves on tokens of their own
  __shared__ uint2 s_book[L * kCodebookSize];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63, n = lane & 15, j = lane >> 4;
  const int half = wave % kHalves, team = wave / kHalves;
  // (chunk, side, KV head fastest): the heads of a token, whose output rows follow each other, run together
  int wg = lut::xcd_contiguous(blockIdx.x, gridDim.x);
  const int kv = wg % a.num_kv_heads;
  wg /= a.num_kv_heads;
  const int sides = (a.k_out ? 1 : 0) + (a.v_out ? 1 : 0);
  const bool value = !a.k_out || wg % sides == 1;
  wg /= sides;
  const int chunks = (a.n + a.chunk - 1) / a.chunk;
  const int b = wg / chunks, first = (wg - b * chunks) * a.chunk;
  const int count = a.lens ? min(max(a.lens[b], 0), a.n) : a.n;
  const int last = min(first + a.chunk, count);
  if (first >= last) return;
  const long long start = a.start_pos[b];
  const long long cap = static_cast<long long>(a.layout.block_size) * a.layout.blocks_per_seq;
  const long long size = a.seq_lens ? min(max(static_cast<long long>(a.seq_lens[b]), 0LL), cap) : cap;
  const bool levels = value && a.v_sq;

  // the transform's rows: tile o's row m is coordinate 64 half + 16 (m / 4) + 4 o + m % 4, so that a
  // lane's results are 16 that follow each other; the contraction in the codewords' order
  const void *t = transform_of(value ? a.t_v : a.t_k_inv_t, kv, D, a.t_bf16);
  half8_t tr[kTiles][kSteps][PARTS];
  float unscale;
  {
    Eight raw[kTiles][kSteps];
    float top = 0.f;
    for (int o = 0; o < kTiles; ++o) {
      const int c = 64 * half + 16 * (n >> 2) + 4 * o + (n & 3);
      for (int s = 0; s < kSteps; ++s) {
        raw[o][s] = load_eight(t, static_cast<size_t>(c) * D + (D / 4) * j + 8 * s, a.t_bf16);
        for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(raw[o][s].x[e]));
      }
    }
    const int up = up_to_14(wave_max(top));
    const float scale = ldexpf(1.f, up);
    unscale = ldexpf(1.f, -up);
    for (int o = 0; o < kTiles; ++o)
      for (int s = 0; s < kSteps; ++s)
        for (int e = 0; e < 8; ++e) {
          _Float16 hi, lo;
          split_half(raw[o][s].x[e] * scale, hi, lo);
          tr[o][s][0][e] = hi;
          if constexpr (PARTS == 2) tr[o][s][1][e] = lo;
        }
  }
  if (!levels) stage_book<L, kThreads>(s_book, value ? a.cb_v : a.cb_k, a.cb_fp8, kv);
  auto times = [&](const half8_t (&x)[kSteps], float4_t (&acc)[kTiles]) {
    for (int o = 0; o < kTiles; ++o) acc[o] = float4_t{0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < kSteps; ++s)
      for (int p = 0; p < PARTS; ++p)
        for (int o = 0; o < kTiles; ++o) acc[o] = __builtin_amdgcn_mfma_f32_16x16x32_f16(tr[o][s][p], x[s], acc[o], 0, 0, 0);
  };
  // what is added to a lane's 16 coordinates: k_bar, or the transform's row sums
  const int coord = 64 * half + 16 * j;
  float4_t bias[kTiles];
  if (levels) {
    const _Float16 one = 1;
    half8_t ones[kSteps];
    for (int s = 0; s < kSteps; ++s) ones[s] = half8_t{one, one, one, one, one, one, one, one};
    times(ones, bias);
  } else {
    for (int o = 0; o < kTiles; ++o)
      for (int i = 0; i < 4; ++i) bias[o][i] = value ? 0.f : a.kbar[kv * D + coord + 4 * o + i];
  }
  __syncthreads();

  const uint8_t *codes = value ? a.v_codes : a.k_codes;
  const int bs = a.layout.block_size;
  const int32_t *table = a.layout.block_table ? a.layout.block_table + static_cast<size_t>(b) * a.layout.blocks_per_seq : nullptr;
  const long long first_block = static_cast<long long>(b) * a.layout.blocks_per_seq;
  // A lane's token: its place, its row, then its codes, each requested a tile of 16 tokens ahead.
  struct Token {
    int i;          // of the call, -1: none
    int pos;
    bool held;      // in the band
    int phys, row;  // block (read from the table), row in it
    uint32_t w[D / 64];
    uint32_t extra;
  };
  constexpr int kStride = 16 * kGroups;
  int at = first + 16 * team + n;
  auto find = [&](Token &k) {
    k.i = -1, k.held = false, k.phys = 0, k.row = 0, k.pos = 0;
    const long long p = start + at;
    if (at < last && p >= 0 && p < size) {
      k.i = at;
      k.pos = static_cast<int>(p);
      k.held = a.band_k && (k.pos < a.n_sink || k.pos >= size - a.n_rec);
      if (!k.held) {
        const int blk = k.pos / bs;
        k.row = k.pos - blk * bs;
        k.phys = table ? table[blk] : static_cast<int>(first_block + blk);
      }
    }
    at += kStride;
  };
  auto request = [&](Token &k) {  // of tokens that are not there or in the band: the pool's first row
    const size_t row = (static_cast<size_t>(k.phys) * a.num_kv_heads + (k.i < 0 || k.held ? 0 : kv)) * bs + k.row;
    const uint8_t *p = codes + row * L + (L / 4) * j;
    if constexpr (D == 128) {
      const uint2 w = *reinterpret_cast<const uint2 *>(p);
      k.w[0] = w.x, k.w[1] = w.y;
    } else {
      k.w[0] = *reinterpret_cast<const uint32_t *>(p);
    }
    k.extra = 0;
    if (levels) k.extra = reinterpret_cast<const uint32_t *>(a.v_sq)[row];
    else if (!value && a.k_scales) k.extra = a.k_scales[row];
  };
  Token cur, next;
  find(cur);
  request(cur);
  find(next);
  const uint32_t book = (L / 4) * j * kCodebookSize;
  for (int tile = first + 16 * team; tile < last; tile += kStride) {
    half8_t x[kSteps];
    for (int s = 0; s < kSteps; ++s) {
      uint2 w[2];
      for (int y = 0; y < 2; ++y) {
        const int g = 2 * s + y;
        const uint32_t code = (cur.w[g / 4] >> (8 * (g & 3))) & 0xffu;
        w[y] = levels ? centred_levels(code) : s_book[book + g * kCodebookSize + code];
      }
      x[s] = __builtin_bit_cast(half8_t, make_uint4(w[0].x, w[0].y, w[1].x, w[1].y));
    }
    const Token mine = cur;
    cur = next;
    request(cur);
    find(next);
    float4_t acc[kTiles];
    times(x, acc);
    if (mine.i < 0) continue;
    float by = unscale, add = 1.f;
    if (levels) {
      const float scale = bf16_bits_to_float(mine.extra & 0xffffu), offset = bf16_bits_to_float(mine.extra >> 16);
      by = scale, add = __builtin_fmaf(1.5f, scale, offset);
    } else if (!value && a.k_scales) {
      by = bf16_bits_to_float(mine.extra) * unscale;
    }
    float y[16];
    for (int o = 0; o < kTiles; ++o)
      for (int i = 0; i < 4; ++i) {
        if (levels) y[4 * o + i] = __builtin_fmaf(by, acc[o][i] * unscale, add * (bias[o][i] * unscale));
        else y[4 * o + i] = __builtin_fmaf(by, acc[o][i], bias[o][i]);
      }
    const size_t to = ((static_cast<size_t>(b) * a.n + mine.i) * a.num_kv_heads + kv) * D + coord;
    if (mine.held) {
      const int slot = band_slot(mine.pos, a.n_sink, a.n_rec);
      const uint16_t *row = (value ? a.band_v : a.band_k) +
                            ((static_cast<size_t>(b) * a.num_kv_heads + kv) * (a.n_sink + a.n_rec) + slot) * D + coord;
      for (int h = 0; h < 2; ++h) {
        const uint4 w = reinterpret_cast<const uint4 *>(row)[h];
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
        for (int e = 0; e < 4; ++e) {
          y[8 * h + 2 * e] = __uint_as_float(u[e] << 16);
          y[8 * h + 2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
        }
      }
    }
    void *out = value ? a.v_out : a.k_out;
    if (a.bf16) {
      for (int h = 0; h < 2; ++h) {
        bf16x8 v;
        for (int e = 0; e < 8; ++e) v[e] = static_cast<__bf16>(y[8 * h + e]);
        *reinterpret_cast<bf16x8 *>(static_cast<__bf16 *>(out) + to + 8 * h) = v;
      }
    } else {
      for (int h = 0; h < 4; ++h)
        reinterpret_cast<float4 *>(static_cast<float *>(out) + to)[h] = make_float4(y[4 * h], y[4 * h + 1], y[4 * h + 2], y[4 * h + 3]);
    }
  }
}

// ------------------------------------------------------------------ 4 bits

constexpr int kHeads = 4;  // heads of a workgroup, whose rows are requested at once

// D / 8 lanes hold a row, 8 coordinates each; a wave's rows are tokens that follow each
// other, so their codes do too.
template <int D, bool BF16>
__global__ __launch_bounds__(256) void q4_read_kernel(const ReadArgs a) {
  constexpr int kLanes = D / 8, kTokens = 256 / kLanes;
  const int lane = threadIdx.x % kLanes, slot = threadIdx.x / kLanes;
  const int tiles = (a.n + kTokens - 1) / kTokens;
  const int b = blockIdx.x / tiles, i = (blockIdx.x - b * tiles) * kTokens + slot;
  if (i >= (a.lens ? min(a.lens[b], a.n) : a.n)) return;
  const long long pos = static_cast<long long>(a.start_pos[b]) + i;
  if (pos < 0 || pos >= static_cast<long long>(a.layout.block_size) * a.layout.blocks_per_seq) return;
  const int blk = static_cast<int>(pos) / a.layout.block_size;
  const long long logical = static_cast<long long>(b) * a.layout.blocks_per_seq + blk;
  const long long phys = a.layout.block_table ? a.layout.block_table[logical] : logical;
  if (phys < 0 || phys >= a.num_blocks) return;
  const size_t row0 = static_cast<size_t>(phys) * a.num_kv_heads * a.layout.block_size + (static_cast<int>(pos) - blk * a.layout.block_size);
  const int h0 = blockIdx.y * kHeads;
  uint32_t word[2][kHeads], sq[2][kHeads];
#pragma unroll
  for (int y = 0; y < kHeads; ++y) {
    const size_t row = row0 + static_cast<size_t>(min(h0 + y, a.num_kv_heads - 1)) * a.layout.block_size;
    if (a.k_out) {
      word[0][y] = *reinterpret_cast<const uint32_t *>(a.k_codes + row * (D / 2) + 4 * lane);
      sq[0][y] = reinterpret_cast<const uint32_t *>(a.k_sq)[row];
    }
    if (a.v_out) {
      word[1][y] = *reinterpret_cast<const uint32_t *>(a.v_codes + row * (D / 2) + 4 * lane);
      sq[1][y] = reinterpret_cast<const uint32_t *>(a.v_sq)[row];
    }
  }
#pragma unroll
  for (int y = 0; y < kHeads; ++y) {
    if (h0 + y >= a.num_kv_heads) break;
    const size_t to = ((static_cast<size_t>(b) * a.n + i) * a.num_kv_heads + h0 + y) * D + 8 * lane;
    for (int side = 0; side < 2; ++side) {
      void *out = side ? a.v_out : a.k_out;
      if (!out) continue;
      const float scale = bf16_bits_to_float(sq[side][y] & 0xffffu), offset = bf16_bits_to_float(sq[side][y] >> 16);
      float x[8];
      for (int e = 0; e < 8; ++e) x[e] = __builtin_fmaf(scale, static_cast<float>((word[side][y] >> (4 * e)) & 15u), offset);
      if constexpr (BF16) {
        bf16x8 v;
        for (int e = 0; e < 8; ++e) v[e] = static_cast<__bf16>(x[e]);
        *reinterpret_cast<bf16x8 *>(static_cast<__bf16 *>(out) + to) = v;
      } else {
        float4 *p = reinterpret_cast<float4 *>(static_cast<float *>(out) + to);
        p[0] = make_float4(x[0], x[1], x[2], x[3]);
        p[1] = make_float4(x[4], x[5], x[6], x[7]);
      }
    }
  }
}

}  // namespace

hipError_t launch_read(const ReadArgs &args, hipStream_t stream) {
  ReadArgs a = args;
  const int sides = (a.k_out ? 1 : 0) + (a.v_out ? 1 : 0);
  const long long units = static_cast<long long>(a.batch) * a.num_kv_heads * sides;
  const int step = 16 * kWaves / (a.head_dim / 64);
  const long long want = std::max(1LL, 512 / units);  // chunks that fill the CUs with two workgroups each
  a.chunk = static_cast<int>(((a.n + want - 1) / want + step - 1) / step * step);
  const unsigned grid = static_cast<unsigned>(units * ((a.n + a.chunk - 1) / a.chunk));
  using std::integral_constant;
  auto go = [&](auto d, auto parts) {
    read_kernel<d(), parts()><<<grid, kThreads, 0, stream>>>(a);
    return hipGetLastError();
  };
  auto by_parts = [&](auto d) { return a.t_bf16 ? go(d, integral_constant<int, 1>{}) : go(d, integral_constant<int, 2>{}); };
  return a.head_dim == 128 ? by_parts(integral_constant<int, 128>{}) : by_parts(integral_constant<int, 64>{});
}

hipError_t launch_q4_read(const ReadArgs &a, hipStream_t stream) {
  const int tokens = 256 / (a.head_dim / 8);
  const dim3 grid(static_cast<unsigned>(a.batch) * ((a.n + tokens - 1) / tokens), (a.num_kv_heads + kHeads - 1) / kHeads);
  auto go = [&](auto d, auto bf16) {
    q4_read_kernel<d(), bf16()><<<grid, 256, 0, stream>>>(a);
    return hipGetLastError();
  };
  auto by_type = [&](auto d) { return a.bf16 ? go(d, std::true_type{}) : go(d, std::false_type{}); };
  return a.head_dim == 128 ? by_type(std::integral_constant<int, 128>{}) : by_type(std::integral_constant<int, 64>{});
}

}  // namespace novakv
