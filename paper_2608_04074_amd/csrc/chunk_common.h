// Device code shared by the kernels that take 2-bit codes to matrix operands.
#pragma once

#include "chunk_internal.h"
#include "q4_common.h"

namespace novakv {
namespace chunk {

using lut::add_rows16;
using lut::add_rows32;
using lut::float4_t;
using lut::half2_t;
using lut::half8_t;
using lut::max_rows16;
using lut::max_rows32;
using q4::exp2_raw;
using q4::half_factor;
using q4::kNone;
using q4::Tile;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// The physical blocks of a sequence, without a branch: a load that may not have been made would be waited
// for at once. Without a table a place that can be read is, times 0.
struct Blocks {
  const int32_t *table;
  int mapped, first;
  __device__ __forceinline__ Blocks(const CacheLayout &layout, const int b, const int32_t *readable) {
    mapped = __builtin_amdgcn_readfirstlane(layout.block_table ? 1 : 0);
    asm volatile("" : "+s"(mapped));  // not turned back into a branch
    table = layout.block_table ? layout.block_table + static_cast<size_t>(b) * layout.blocks_per_seq : readable;
    first = layout.block_table ? 0 : b * layout.blocks_per_seq;
  }
  __device__ __forceinline__ int entry(const int blk) const { return table[mapped * blk]; }
  __device__ __forceinline__ int phys(const int entry, const int blk) const { return entry * mapped + (1 - mapped) * blk + first; }
};

// log2 of the largest probability (times its value's scale) after a rescale, and how far it may grow
constexpr float kTop = 6.f, kSlack = 8.f;
constexpr int kLeastValue = -70;  // exponent of the smallest value scale that the reference follows

// A KV head's codebook [L][256] into LDS as fp16 codewords.
template <int L, int THREADS>
__device__ __forceinline__ void stage_book(uint2 *to, const void *cb, const int fp8, const int kv) {
  const size_t first = static_cast<size_t>(kv) * L * kCodebookSize;
  if (fp8) {
    const uint4 *from = reinterpret_cast<const uint4 *>(static_cast<const uint32_t *>(cb) + first);  // four codewords
#pragma unroll 4
    for (int i = threadIdx.x; i < L * kCodebookSize / 4; i += THREADS) {
      const uint4 w = from[i];
      const uint2 c[4] = {codeword_f16(make_uint2(w.x, 0u), 1), codeword_f16(make_uint2(w.y, 0u), 1),
                          codeword_f16(make_uint2(w.z, 0u), 1), codeword_f16(make_uint2(w.w, 0u), 1)};
      reinterpret_cast<uint4 *>(to)[2 * i] = make_uint4(c[0].x, c[0].y, c[1].x, c[1].y);
      reinterpret_cast<uint4 *>(to)[2 * i + 1] = make_uint4(c[2].x, c[2].y, c[3].x, c[3].y);
    }
  } else {
    const uint4 *from = reinterpret_cast<const uint4 *>(static_cast<const uint2 *>(cb) + first);  // two codewords
#pragma unroll 8
    for (int i = threadIdx.x; i < L * kCodebookSize / 2; i += THREADS) reinterpret_cast<uint4 *>(to)[i] = from[i];
  }
}

// Eight consecutive elements of a transform, widened.
struct Eight {
  float x[8];
};
__device__ __forceinline__ Eight load_eight(const void *t, const size_t i, const int bf16) {
  Eight r;
  const float4 a = t4_value(load_t4(t, i, bf16), bf16), b = t4_value(load_t4(t, i + 4, bf16), bf16);
  r.x[0] = a.x, r.x[1] = a.y, r.x[2] = a.z, r.x[3] = a.w, r.x[4] = b.x, r.x[5] = b.y, r.x[6] = b.z, r.x[7] = b.w;
  return r;
}

// x in two fp16 parts, x = hi + lo to 2^-22 of it (|x| below fp16's range; parts below 2^-24
// are lost). x is made opaque: a product fused into one of the uses of hi but not the other
// would leave two different roundings of it.
__device__ __forceinline__ void split_half(float x, _Float16 &hi, _Float16 &lo) {
  asm volatile("" : "+v"(x));
  hi = static_cast<_Float16>(x);
  lo = static_cast<_Float16>(x - static_cast<float>(hi));
}

// Largest magnitude of a wave's lanes.
__device__ __forceinline__ float wave_max(float x) {
  x = fmaxf(x, lut::row_ror<8>(x));
  x = fmaxf(x, lut::row_ror<4>(x));
  x = fmaxf(x, lut::row_ror<2>(x));
  x = fmaxf(x, lut::row_ror<1>(x));
  return lut::max_rows32(lut::max_rows16(x));
}

// Exponent that brings a magnitude to [2^13, 2^14); 0 for one that is 0 or not finite.
__device__ __forceinline__ int up_to_14(const float top) {
  return top > 0.f && top < __builtin_inff() ? min(max(13 - ilogbf(top), -120), 120) : 0;
}

// Scalar value arm: a code byte's four levels minus 1.5, exact in fp16.
__device__ __forceinline__ uint2 centred_levels(const uint32_t c) {
  const uint2 q = sq_unpack_f16(c);
  const half2_t mid = {static_cast<_Float16>(1.5f), static_cast<_Float16>(1.5f)};
  return make_uint2(__builtin_bit_cast(uint32_t, __builtin_bit_cast(half2_t, q.x) - mid),
                    __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2_t, q.y) - mid));
}

// Coordinate (in the value transform's order) of output tile o's row m, of sums over codewords.
template <int D>
__device__ __forceinline__ int code_coord(const int o, const int m) {
  return D == 128 ? 16 * (m & 7) + 8 * (m >> 3) + o : 16 * (m & 3) + 4 * (m >> 2) + o;
}
// The value group whose codewords a lane n mod 16 makes tiles 4 p .. 4 p + 3 of.
template <int D>
__device__ __forceinline__ int value_group(const int n, const int p) {
  return D == 128 ? 4 * (n & 7) + 2 * (n >> 3) + p : 4 * (n & 3) + (n >> 2);
}

// Three bf16 parts of an fp32 value: 24 bits.
__device__ __forceinline__ void split_bf16(const float x, __bf16 &a, __bf16 &b, __bf16 &c) {
  float y = x;
  asm volatile("" : "+v"(y));
  a = static_cast<__bf16>(y);
  y -= static_cast<float>(a);
  b = static_cast<__bf16>(y);
  c = static_cast<__bf16>(y - static_cast<float>(b));
}

// Low or high halves of two words.
__device__ __forceinline__ uint32_t half_pair(const uint32_t x, const uint32_t y, const bool high) {
  return __builtin_amdgcn_perm(y, x, high ? 0x07060302u : 0x05040100u);
}

// A wave's sums over NT tiles of 16 rows (lane: row lane mod 16), in front of the division:
// sum_j exp2(z_j - ref) and the same times values.
template <int D, int NT>
struct Sums {
  float ref[NT], sum[NT], off_sum[NT];  // off_sum: of weights times the scalar arm's offsets
  float4_t acc[NT][D / 16];
  __device__ __forceinline__ void clear() {
    for (int t = 0; t < NT; ++t) {
      ref[t] = kNone, sum[t] = 0.f, off_sum[t] = 0.f;
      for (int o = 0; o < D / 16; ++o) acc[t][o] = float4_t{0.f, 0.f, 0.f, 0.f};
    }
  }
  // Raises the references where a weight (times 2^exponent of its value's scale) would leave fp16:
  // bound is this lane's largest log2 of one.
  __device__ __forceinline__ void raise(const float (&bound)[NT]) {
    bool over = false;
    for (int t = 0; t < NT; ++t) over |= bound[t] > ref[t] + (kTop + kSlack);
    if (!__any(over)) return;
    for (int t = 0; t < NT; ++t) {
      const float to = fmaxf(ref[t], max_rows32(max_rows16(bound[t])) - kTop);
      const float f = to == kNone ? 1.f : half_factor(ref[t] - to);
      ref[t] = to;
      for (int y = 0; y < 2; ++y) {
        sum[t] *= f;
        off_sum[t] *= f;
        for (int o = 0; o < D / 16; ++o) acc[t][o] *= f;
      }
    }
  }
};

// A band's exact rows, on the bf16 cores: queries in one part (fp32 ones in three), probabilities
// in two (three). Output tile o's row m is coordinate q4::out_coord.
template <int D, bool WIDE, int NT>
struct Band {
  static constexpr int kQParts = WIDE ? 3 : 1, kPParts = WIDE ? 3 : 2, kSteps = D / 32, kTiles = D / 16;
  const ChunkArgs &a;
  size_t rows;  // of the (sequence, KV head)
  int n, j;
  bf16x8 q[NT][kSteps][kQParts];

  __device__ __forceinline__ Band(const ChunkArgs &args, const int b, const int kv, const int lane)
      : a(args), rows((static_cast<size_t>(b) * args.num_kv_heads + kv) * (args.n_sink + args.n_rec)), n(lane & 15), j(lane >> 4) {}
  // tile t's queries: coordinates 32 s + 8 j + e of row n
  __device__ __forceinline__ void set_queries(const int t, const float (&x)[kSteps][8]) {
    for (int s = 0; s < kSteps; ++s)
      for (int e = 0; e < 8; ++e) {
        if constexpr (WIDE) {
          __bf16 u, v, w;
          split_bf16(x[s][e], u, v, w);
          q[t][s][0][e] = u, q[t][s][1][e] = v, q[t][s][2][e] = w;
        } else {
          q[t][s][0][e] = static_cast<__bf16>(x[s][e]);
        }
      }
  }
  // Positions [from, to) of the 32 from tb on, for rows that attend [row_lo, row_hi).
  __device__ __forceinline__ void attend(const int tb, const int from, const int to, const int (&row_lo)[NT], const int (&row_hi)[NT],
                                         Sums<D, NT> &y) const {
    auto row_of = [&](const int tok) { return (rows + band_slot(min(max(tok, from), to - 1), a.n_sink, a.n_rec)) * D; };
    float4_t s[NT][2];
    for (int x = 0; x < 2; ++x) {
      const uint16_t *k = a.band_k + row_of(tb + 16 * x + n) + 8 * j;
      for (int t = 0; t < NT; ++t) s[t][x] = float4_t{0.f, 0.f, 0.f, 0.f};
      for (int st = 0; st < kSteps; ++st) {
        const bf16x8 kf = *reinterpret_cast<const bf16x8 *>(k + 32 * st);
        for (int t = 0; t < NT; ++t)
          for (int p = 0; p < kQParts; ++p) s[t][x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, q[t][st][p], s[t][x], 0, 0, 0);
      }
    }
    // a lane's eight tokens 16 x + 4 j + i, D / 16 coordinates of each
    uint32_t v[8][D / 32];
    bool odd[8];
    for (int e = 0; e < 8; ++e) {
      const int tok = tb + 16 * (e >> 2) + 4 * j + (e & 3);
      const uint32_t *p = reinterpret_cast<const uint32_t *>(a.band_v + row_of(tok) + (D == 128 ? 8 * n : 8 * (n & 7) + 4 * (n >> 3)));
      bool bad = false;
      for (int w = 0; w < D / 32; ++w) {
        v[e][w] = p[w];
        bad |= (v[e][w] & 0x7f80u) == 0x7f80u || (v[e][w] & 0x7f800000u) == 0x7f800000u;
      }
      // A value that is not finite would reach the rows it is hidden from (0 * NaN): the token's
      // score becomes NaN instead, and the value 0.
      const uint64_t any = __ballot(bad);
      odd[e] = (any >> (16 * j)) & 0xffffu;
      for (int w = 0; w < D / 32; ++w) v[e][w] = odd[e] ? 0u : v[e][w];
    }
    float bound[NT];
    for (int t = 0; t < NT; ++t) {
      bound[t] = kNone;
      for (int e = 0; e < 8; ++e) {
        const int tok = tb + 16 * (e >> 2) + 4 * j + (e & 3);
        const bool seen = tok >= max(from, row_lo[t]) && tok < min(to, row_hi[t]);
        const float z = seen ? (odd[e] ? __builtin_nanf("") : s[t][e >> 2][e & 3] * a.qscale) : kNone;
        s[t][e >> 2][e & 3] = z;
        bound[t] = fmaxf(bound[t], z);
      }
    }
    y.raise(bound);
    bf16x8 pf[NT][kPParts];
    for (int t = 0; t < NT; ++t) {
      const float r = y.ref[t] == kNone ? 0.f : y.ref[t];
      for (int e = 0; e < 8; ++e) {
        const float p = exp2_raw(s[t][e >> 2][e & 3] - r);
        y.sum[t] += p;
        __bf16 u, v, w;
        split_bf16(p, u, v, w);
        pf[t][0][e] = u, pf[t][1][e] = v;
        if constexpr (kPParts == 3) pf[t][2][e] = w;
      }
    }
    for (int o = 0; o < kTiles; ++o) {
      uint32_t w[4];
      for (int x = 0; x < 4; ++x) w[x] = half_pair(v[2 * x][o / 2], v[2 * x + 1][o / 2], o & 1);
      const bf16x8 vf = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
      for (int t = 0; t < NT; ++t)
        for (int p = 0; p < kPParts; ++p) y.acc[t][o] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[t][p], y.acc[t][o], 0, 0, 0);
    }
  }
};

// Eight coordinates of a query row from its 16-byte aligned place.
template <bool WIDE>
__device__ __forceinline__ void load_query(const void *q, const size_t at, float (&x)[8]) {
  if constexpr (WIDE) {
    const float4 *p = reinterpret_cast<const float4 *>(static_cast<const float *>(q) + at);
    const float4 u = p[0], v = p[1];
    x[0] = u.x, x[1] = u.y, x[2] = u.z, x[3] = u.w, x[4] = v.x, x[5] = v.y, x[6] = v.z, x[7] = v.w;
  } else {
    const uint4 w = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(q) + at);
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
    for (int e = 0; e < 4; ++e) x[2 * e] = __uint_as_float(u[e] << 16), x[2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
  }
}

// The scalar arm's token: scale, offset + 1.5 scale (of levels - 1.5), and the exponent above the scale
// or, where that is less, above 2^-8 of the offset. Of a value that is not finite (it would reach
// the rows it is hidden from) the token's key becomes NaN instead, and the value 0; a token that is
// not there has none.
struct Grid {
  float scale, offset, expo;
};
__device__ __forceinline__ Grid grid_of(const uint32_t sq, const bool there, float &rho) {
  Grid g;
  g.scale = there ? __uint_as_float(sq << 16) : 0.f;
  g.offset = there ? __uint_as_float(sq & 0xffff0000u) : 0.f;
  g.offset = __builtin_fmaf(1.5f, g.scale, g.offset);
  if (!(fabsf(g.scale) < __builtin_inff() && fabsf(g.offset) < __builtin_inff())) rho = __builtin_nanf(""), g.scale = g.offset = 0.f;
  const float size = fmaxf(fabsf(g.scale), 0x1p-8f * fabsf(g.offset));
  g.expo = static_cast<float>(max((__builtin_bit_cast(int, size) >> 23) - 126, kLeastValue));
  return g;
}

// What a split attends: codes [c0, c1), and the band's positions [low, sink1) and [rec0, t1).
struct Spans {
  int c0, c1, low, sink1, rec0;
  bool codes, banded;
  __device__ __forceinline__ Spans(const ChunkArgs &a, const Tile &g) {
    low = max(g.t0, g.lo);
    const int rec = a.band_k ? max(g.S - a.n_rec, a.n_sink) : g.t1;
    c0 = max(low, a.n_sink), c1 = min(g.t1, rec);
    sink1 = min(g.t1, a.n_sink), rec0 = max(low, rec);
    codes = c0 < c1;
    banded = a.band_k && (low < sink1 || rec0 < g.t1);
  }
};

}  // namespace chunk
}  // namespace novakv
