// Reading a cache back: tokens of the 2-bit cache (nova_kv_read) and of the 4-bit cache
// (nova_kv_q4_read) as dense rows in fp32 or bf16.
//
// 2 bits: k = rho (r R_K^-1) + k_bar and v = s R_V^T, both a row of codewords times the
// transposed rows of a [D][D] array, on the fp16 matrix cores: a token's codewords, gathered
// from the codebook in LDS, are one operand as they come; the transform's rows stay in
// registers, as two fp16 parts (22 bits; one part where they are stored as bf16). The scalar
// arm's levels enter as level - 1.5, exact, and meet the transform's row sums with the
// token's offset + 1.5 scale.
//
// Bound by its stores and by the products: 16 sequences' 8192 tokens of 8 heads of 128 in bf16 take 159 us; the matrix
// cores work 45% of the cycles, the vector units 43, and a copy of as many bytes would take 123 us. On the way there (241 us at first):
// stores of whole lines of a row instead of 16 bytes, marked as streamed (in halves of lines 180 us, with 753 MB
// written instead of 537); no branch around them; the transform's rows through LDS; one workgroup a CU for the
// whole call.
#include <algorithm>
#include <type_traits>

#include "chunk_common.h"

namespace novakv {

namespace {

using namespace chunk;

// ------------------------------------------------------------------ 2 bits

constexpr int kWaves = 8, kThreads = 64 * kWaves;
// (nt) of stores that are not read again here: 230 -> 198 us when it came; now 183 and 211 alone, with a copy of the rows
// behind the call 381 and 399. Of 17 MB with a copy 25 and 27 us; between, where the caches would have held the rows
// for the copy, 54 and 50 (67 MB).
constexpr int kStream = 2;
typedef float float16_t __attribute__((ext_vector_type(16)));
typedef uint32_t uint4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// One side of a workgroup's tokens [first, last) of a sequence and KV head. LEVELS: the scalar
// value arm. PARTS: fp16 parts of the transform. BAND: some positions are held in the band.
template <int D, int PARTS, bool LEVELS, bool BAND, bool BF16>
__device__ __forceinline__ void read_side(const ReadArgs &a, uint2 *s_book, float *s_rows, const bool value, const int kv, const int b, const int first,
                                          const int last, const int place, const int places) {
  constexpr int L = D / kGroupDim, kSteps = D / 16, kTiles = 2;  // a wave has 64 of the coordinates, 32 tokens at a time
  constexpr int kHalves = D / 64, kTeams = kWaves / kHalves, kStride = 32 * kTeams;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63, n = lane & 31, j = lane >> 5;
  const int half = wave % kHalves, team = wave / kHalves;
  const long long cap = static_cast<long long>(a.layout.block_size) * a.layout.blocks_per_seq;
  const int size = static_cast<int>(a.seq_lens ? min(max(static_cast<long long>(a.seq_lens[b]), 0LL), cap) : min(cap, 0x7fffffffLL));

  // Loads and stores of the loop stand outside branches (a store that may not have been made would
  // be waited for with every load), so lanes whose token is not there, or in the band, read the codes of the
  // nearest that is: code positions [c0, c1); where there are none, the pool's first row.
  const long long start = a.start_pos[b];
  const int sinks = BAND ? a.n_sink : 0, recent = BAND ? min(max(size - a.n_rec, sinks), size) : size;
  const int c0 = static_cast<int>(min(max(start + first, static_cast<long long>(sinks)), static_cast<long long>(size)));
  const int c1 = static_cast<int>(min(max(start + last, 0LL), static_cast<long long>(recent)));
  const bool coded = c0 < c1;
  const uint8_t *codes = value ? a.v_codes : a.k_codes;
  const int bs = a.layout.block_size;
  // without a table (or codes): entries of a place that can be read, times 0
  const bool mapped = a.layout.block_table && coded;
  const int32_t *table = mapped ? a.layout.block_table + static_cast<size_t>(b) * a.layout.blocks_per_seq : a.start_pos + b;
  int by_table = __builtin_amdgcn_readfirstlane(mapped ? 1 : 0);
  asm volatile("" : "+s"(by_table));  // not turned into a branch
  const int first_block = mapped || !coded ? 0 : b * a.layout.blocks_per_seq, by_order = coded ? 1 - by_table : 0;  // blocks are counted in 32 bits
  const uint16_t *const extras = LEVELS ? a.v_sq : value ? nullptr : a.k_scales;
  // Places are looked up two rounds of tokens ahead, codes requested one.
  struct Place {
    int phys, row;
  };
  struct Codes {
    uint32_t w[L / 8], extra;
  };
  // The workgroups start at different rounds of their tokens, and go round: those of a large call would write to
  // the same memory channels at the same time.
  const int rounds = (last - first + kStride - 1) / kStride;
  const int turn0 = static_cast<int>(static_cast<long long>(rounds) * place / places);
  int turn = turn0;  // the next round to look up
  auto find = [&](Place &k) {
    const int pos = static_cast<int>(min(max(start + first + 32 * team + turn * kStride + n, static_cast<long long>(c0)), static_cast<long long>(c1) - 1));
    const int blk = a.block_of(pos);
    k.row = coded ? pos - blk * bs : 0;
    k.phys = table[by_table * blk] * by_table + by_order * blk + first_block;
    turn = turn + 1 == rounds ? 0 : turn + 1;
  };
  auto request = [&](const Place &k, Codes &c) {
    const size_t row = (static_cast<size_t>(k.phys) * a.num_kv_heads + (coded ? kv : 0)) * bs + k.row;
    const uint8_t *p = codes + row * L + (L / 2) * j;
    if constexpr (D == 128) {
      const uint4 w = *reinterpret_cast<const uint4 *>(p);
      c.w[0] = w.x, c.w[1] = w.y, c.w[2] = w.z, c.w[3] = w.w;
    } else {
      const uint2 w = *reinterpret_cast<const uint2 *>(p);
      c.w[0] = w.x, c.w[1] = w.y;
    }
    if constexpr (LEVELS) {
      c.extra = reinterpret_cast<const uint32_t *>(extras)[row];
    } else {
      const uint32_t rho = *(extras ? extras + row : reinterpret_cast<const uint16_t *>(a.start_pos + b));
      c.extra = extras ? rho : 0x3f80u;  // 1
    }
  };
  Place ahead;
  Codes c;
  find(ahead);

  // A lane's results e = 16 o + i (of tile o) are kRun coordinates that follow each other, its other half's (j)
  // beside them: coord_of(e, j). The transform's rows are dealt to the tiles that way; the contraction is in the
  // codewords' order.
  constexpr int kRun = BF16 ? 8 : 4;
  auto coord_of = [](const int e, const int j) { return 2 * kRun * (e / kRun) + kRun * j + e % kRun; };
  {
    // through LDS, where rows are apart by an odd number of 16 bytes: a wave's loads of 64 rows' parts would
    // otherwise be 64 requests each (12 us of a workgroup's time at head_dim 128)
    constexpr int kPieces = D * D / 4 / kThreads;
    const void *t = transform_of(value ? a.t_v : a.t_k_inv_t, kv, D, a.t_bf16);
    T4 piece[kPieces];
    for (int i = 0; i < kPieces; ++i) piece[i] = load_t4(t, 4 * (static_cast<size_t>(i) * kThreads + threadIdx.x), a.t_bf16);
    if constexpr (!LEVELS) stage_book<L, kThreads>(s_book, value ? a.cb_v : a.cb_k, a.cb_fp8, kv);
    for (int i = 0; i < kPieces; ++i) {
      const int x = 4 * (i * kThreads + threadIdx.x);
      *reinterpret_cast<float4 *>(s_rows + (x / D) * (D + 4) + x % D) = t4_value(piece[i], a.t_bf16);
    }
  }
  __syncthreads();
  half8_t tr[kTiles][kSteps][PARTS];
  float unscale[kTiles];
#pragma unroll
  for (int o = 0; o < kTiles; ++o) {
    const int row = 64 * half + coord_of(16 * o + 4 * (n >> 3) + (n & 3), (n >> 2) & 1);
    Eight raw[kSteps];
    float top = 0.f;
    for (int s = 0; s < kSteps; ++s) {
      const float4 *p = reinterpret_cast<const float4 *>(s_rows + row * (D + 4) + (D / 2) * j + 8 * s);
      const float4 u = p[0], v = p[1];
      raw[s] = {{u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w}};
      for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(raw[s].x[e]));
    }
    const int up = up_to_14(wave_max(top));
    const float scale = ldexpf(1.f, up);
    unscale[o] = ldexpf(1.f, -up);
    for (int s = 0; s < kSteps; ++s)
      for (int e = 0; e < 8; ++e) {
        _Float16 hi, lo;
        split_half(raw[s].x[e] * scale, hi, lo);
        tr[o][s][0][e] = hi;
        if constexpr (PARTS == 2) tr[o][s][1][e] = lo;
      }
  }
  request(ahead, c);
  find(ahead);
  auto times = [&](const half8_t (&x)[kSteps], float16_t (&acc)[kTiles]) {
    for (int o = 0; o < kTiles; ++o)
      for (int i = 0; i < 16; ++i) acc[o][i] = 0.f;
    for (int s = 0; s < kSteps; ++s)
      for (int p = 0; p < PARTS; ++p)
        for (int o = 0; o < kTiles; ++o) acc[o] = __builtin_amdgcn_mfma_f32_32x32x16_f16(tr[o][s][p], x[s], acc[o], 0, 0, 0);
  };
  // what is added to a lane's 32 coordinates: k_bar, or the transform's row sums
  float16_t bias[kTiles];
  if constexpr (LEVELS) {
    const _Float16 one = 1;
    half8_t ones[kSteps];
    for (int s = 0; s < kSteps; ++s) ones[s] = half8_t{one, one, one, one, one, one, one, one};
    times(ones, bias);
    for (int o = 0; o < kTiles; ++o) bias[o] *= unscale[o];
  } else {
    const float *kbar = a.kbar + kv * D + 64 * half;
    for (int o = 0; o < kTiles; ++o)
      for (int i = 0; i < 16; ++i) bias[o][i] = kbar[coord_of(16 * o + i, j)];
    if (value)
      for (int o = 0; o < kTiles; ++o)
        for (int i = 0; i < 16; ++i) bias[o][i] = 0.f;
  }

  // the chunk's rows of the output; stores of lanes that have no token fall behind their end
  constexpr int kBytes = BF16 ? 2 : 4;
  const size_t row_bytes = static_cast<size_t>(a.num_kv_heads) * D * kBytes;
  uint8_t *const out = static_cast<uint8_t *>(value ? a.v_out : a.k_out) + (static_cast<size_t>(b) * a.n + first) * row_bytes;
  const __amdgpu_buffer_rsrc_t rows = __builtin_amdgcn_make_buffer_rsrc(out, 0, static_cast<int>((last - first) * row_bytes), 0x00020000);
  constexpr int kOutside = -0x7fffffff - 1;  // 2^31, above any chunk's bytes, and some more stays so
  const uint32_t book = (L / 2) * j * kCodebookSize;
  for (int r = 0; r < rounds; ++r) {
    const int at = r + turn0 < rounds ? r + turn0 : r + turn0 - rounds, tile = first + 32 * team + at * kStride;
    half8_t x[kSteps];
    for (int s = 0; s < kSteps; ++s) {
      uint2 w[2];
      for (int y = 0; y < 2; ++y) {
        const int g = 2 * s + y;
        const uint32_t code = (c.w[g / 4] >> (8 * (g & 3))) & 0xffu;
        if constexpr (LEVELS) w[y] = centred_levels(code);
        else w[y] = s_book[book + g * kCodebookSize + code];
      }
      x[s] = __builtin_bit_cast(half8_t, make_uint4(w[0].x, w[0].y, w[1].x, w[1].y));
    }
    const uint32_t extra = c.extra;
    request(ahead, c);
    find(ahead);
    float16_t acc[kTiles];
    times(x, acc);
    float y[32];
    if constexpr (LEVELS) {
      const float scale = bf16_bits_to_float(extra & 0xffffu), offset = bf16_bits_to_float(extra >> 16);
      const float add = __builtin_fmaf(1.5f, scale, offset);
      for (int e = 0; e < 32; ++e) y[e] = __builtin_fmaf(scale, acc[e >> 4][e & 15] * unscale[e >> 4], add * bias[e >> 4][e & 15]);
    } else {
      const float rho = bf16_bits_to_float(extra), by[kTiles] = {rho * unscale[0], rho * unscale[1]};
      for (int e = 0; e < 32; ++e) y[e] = __builtin_fmaf(by[e >> 4], acc[e >> 4][e & 15], bias[e >> 4][e & 15]);
    }
    auto there = [&](const int i) { return static_cast<int>(i < last) & static_cast<int>(start + i >= 0) & static_cast<int>(start + i < size); };
    if constexpr (BAND) {
      const long long pos = start + tile + n;
      if (there(tile + n) && (pos < sinks || pos >= size - a.n_rec)) {
        const int slot = band_slot(static_cast<int>(pos), a.n_sink, a.n_rec);
        const uint16_t *row = (value ? a.band_v : a.band_k) +
                              ((static_cast<size_t>(b) * a.num_kv_heads + kv) * (a.n_sink + a.n_rec) + slot) * D + 64 * half;
        for (int e = 0; e < 32; e += 4) {
          const uint2 w = *reinterpret_cast<const uint2 *>(row + coord_of(e, j));
          y[e] = __uint_as_float(w.x << 16), y[e + 1] = __uint_as_float(w.x & 0xffff0000u);
          y[e + 2] = __uint_as_float(w.y << 16), y[e + 3] = __uint_as_float(w.y & 0xffff0000u);
        }
      }
    }
    // Runs of two tokens 16 apart change places, then those of two that are 8 apart, so that a store has 128
    // bytes of a row (whole lines) from eight lanes.
    int to[2][2];  // tokens 16 x + 8 z + n % 8
    for (int x = 0; x < 2; ++x)
      for (int z = 0; z < 2; ++z) {
        const int i = tile + 16 * x + 8 * z + (n & 7);
        const int at = kv * D + 64 * half + 4 * kRun * ((n >> 3) & 1) + 2 * kRun * (n >> 4) + kRun * j;
        to[x][z] = there(i) ? static_cast<int>((i - first) * row_bytes) + at * kBytes : kOutside;
      }
    for (int h = 0; h < 32 / kRun; h += 4) {
      uint32_t w[4][4];
      for (int x = 0; x < 4; ++x)
        for (int u = 0; u < 4; ++u) {
          const float *from = y + kRun * (h + x) + (BF16 ? 2 * u : u);
          if constexpr (BF16) w[x][u] = __builtin_bit_cast(uint32_t, bf16x2{static_cast<__bf16>(from[0]), static_cast<__bf16>(from[1])});
          else w[x][u] = __float_as_uint(from[0]);
        }
      for (int u = 0; u < 4; ++u) {
        for (int x = 0; x < 4; x += 2) {
          const auto s = __builtin_amdgcn_permlane16_swap(w[x][u], w[x + 1][u], false, false);
          w[x][u] = s[0], w[x + 1][u] = s[1];
        }
        for (int x = 0; x < 2; ++x) {  // lanes 8 .. 15 of a row for 0 .. 7 of the other (DPP row_ror:8)
          const int low = w[x][u], high = w[x + 2][u];
          w[x][u] = __builtin_amdgcn_update_dpp(low, high, 0x128, 0xf, 0xc, false);
          w[x + 2][u] = __builtin_amdgcn_update_dpp(high, low, 0x128, 0xf, 0x3, false);
        }
      }
      for (int x = 0; x < 2; ++x)
        for (int z = 0; z < 2; ++z) {
          const uint32_t(&v)[4] = w[x + 2 * z];
          __builtin_amdgcn_raw_buffer_store_b128(uint4_t{v[0], v[1], v[2], v[3]}, rows, to[x][z], 2 * kRun * kBytes * h, kStream);
        }
    }
  }
}

// SQ: values are the scalar arm's levels.
template <int D, int PARTS, bool SQ, bool BAND, bool BF16>
__global__ __launch_bounds__(kThreads, 2) void read_kernel(const ReadArgs a) {
  __shared__ __align__(16) uint2 s_book[D / kGroupDim * kCodebookSize];
  __shared__ __align__(16) float s_rows[D * (D + 4)];
  // (chunk, side, KV head fastest): the heads of a token, whose output rows follow each other, run together
  int wg = lut::xcd_contiguous(blockIdx.x, gridDim.x);
  const int kv = wg % a.num_kv_heads;
  wg /= a.num_kv_heads;
  const int sides = (a.k_out ? 1 : 0) + (a.v_out ? 1 : 0);
  const bool value = !a.k_out || wg % sides == 1;
  wg /= sides;
  const int chunks = (a.n + a.chunk - 1) / a.chunk;
  const int places = a.batch * chunks * sides, place = wg * sides + (value ? sides - 1 : 0);
  const int b = wg / chunks, first = (wg - b * chunks) * a.chunk;
  const int count = a.lens ? min(max(a.lens[b], 0), a.n) : a.n;
  const int last = min(first + a.chunk, count);
  if (first >= last) return;
  if constexpr (SQ) {
    if (value) read_side<D, PARTS, true, BAND, BF16>(a, s_book, s_rows, true, kv, b, first, last, place, places);
    else read_side<D, PARTS, false, BAND, BF16>(a, s_book, s_rows, false, kv, b, first, last, place, places);
  } else {
    read_side<D, PARTS, false, BAND, BF16>(a, s_book, s_rows, value, kv, b, first, last, place, places);
  }
}

// ------------------------------------------------------------------ 4 bits

constexpr int kHeads = 4;  // heads of a workgroup, whose rows are requested at once

// D / 8 lanes hold a row, 8 coordinates each; a wave's rows are tokens that follow each
// other, so their codes do too. Bound by HBM: 16 sequences' 8192 tokens of 8 heads of 128 in bf16 127 us, 5.3 TB/s (132
// without streamed stores).
// STREAMED: large bf16 outputs. A lane's 16 bytes of bf16 are parts of whole lines; the two 16 bytes of its fp32
// coordinates lie apart, and streamed they leave as parts of lines (16 sequences' 8192 tokens of 8 heads of 64: 246 us,
// 167 through the caches). What fits the caches is left there for the next call: 4 sequences' 4096 tokens with a copy of
// them 32 us, 41 streamed; 8 x 4096 67 and 76, 8 x 8192 (256 MiB) 174 and 171.
template <int D, bool BF16, bool STREAMED>
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
        bf16x8 *p = reinterpret_cast<bf16x8 *>(static_cast<__bf16 *>(out) + to);
        if constexpr (STREAMED) __builtin_nontemporal_store(v, p);
        else *p = v;
      } else {
        float4_t *p = reinterpret_cast<float4_t *>(static_cast<float *>(out) + to);
        p[0] = float4_t{x[0], x[1], x[2], x[3]};
        p[1] = float4_t{x[4], x[5], x[6], x[7]};
      }
    }
  }
}

}  // namespace

hipError_t launch_read(const ReadArgs &args, hipStream_t stream) {
  ReadArgs a = args;
  const int sides = (a.k_out ? 1 : 0) + (a.v_out ? 1 : 0);
  const long long units = static_cast<long long>(a.batch) * a.num_kv_heads * sides;
  const int step = 32 * kWaves / (a.head_dim / 64);
  // Chunks: their number c that takes the least time, a workgroup's set-up being worth about 128 tokens; a CU holds
  // one workgroup (two at head_dim 64 spilled: 15.5 us for parts of six sequences in the deployed format, 13.2 so).
  const long long seats = 256, rounds = (a.n + step - 1) / step;
  long long best = 0;
  for (int k = 0; k < 8; ++k) {
    const long long c = std::max(1LL, k < 4 ? k + 1 : (k - 3) * seats / units);
    const long long size = (rounds + c - 1) / c * step, time = (units * ((a.n + size - 1) / size) + seats - 1) / seats * (size + 128);
    if (best == 0 || time < best) best = time, a.chunk = static_cast<int>(size);
  }
  a.block_of.set(static_cast<uint32_t>(a.layout.block_size));
  // its rows' bytes are counted in 31 bits
  const long long row_bytes = static_cast<long long>(a.num_kv_heads) * a.head_dim * (a.bf16 ? 2 : 4);
  a.chunk = static_cast<int>(std::min<long long>(a.chunk, std::max(1LL, ((1LL << 31) - 1) / row_bytes / step) * step));
  const unsigned grid = static_cast<unsigned>(units * ((a.n + a.chunk - 1) / a.chunk));
  using std::false_type;
  using std::integral_constant;
  using std::true_type;
  auto go = [&](auto d, auto parts, auto sq, auto band, auto bf16) {
    read_kernel<d(), parts(), sq(), band(), bf16()><<<grid, kThreads, 0, stream>>>(a);
    return hipGetLastError();
  };
  auto by_type = [&](auto d, auto parts, auto sq, auto band) {
    return a.bf16 ? go(d, parts, sq, band, true_type{}) : go(d, parts, sq, band, false_type{});
  };
  auto by_band = [&](auto d, auto parts, auto sq) { return a.band_k ? by_type(d, parts, sq, true_type{}) : by_type(d, parts, sq, false_type{}); };
  auto by_values = [&](auto d, auto parts) {
    return a.v_out && a.v_sq ? by_band(d, parts, true_type{}) : by_band(d, parts, false_type{});
  };
  auto by_parts = [&](auto d) { return a.t_bf16 ? by_values(d, integral_constant<int, 1>{}) : by_values(d, integral_constant<int, 2>{}); };
  return a.head_dim == 128 ? by_parts(integral_constant<int, 128>{}) : by_parts(integral_constant<int, 64>{});
}

hipError_t launch_q4_read(const ReadArgs &a, hipStream_t stream) {
  const int tokens = 256 / (a.head_dim / 8);
  const dim3 grid(static_cast<unsigned>(a.batch) * ((a.n + tokens - 1) / tokens), (a.num_kv_heads + kHeads - 1) / kHeads);
  const long long sides = (a.k_out ? 1 : 0) + (a.v_out ? 1 : 0);
  const bool streamed = sides * a.batch * a.n * a.num_kv_heads * a.head_dim * 2 >= 256LL << 20;  // bytes of bf16
  auto go = [&](auto d, auto bf16, auto nt) {
    q4_read_kernel<d(), bf16(), nt()><<<grid, 256, 0, stream>>>(a);
    return hipGetLastError();
  };
  using std::false_type;
  using std::true_type;
  auto by_type = [&](auto d) {
    if (!a.bf16) return go(d, false_type{}, false_type{});
    return streamed ? go(d, true_type{}, true_type{}) : go(d, true_type{}, false_type{});
  };
  return a.head_dim == 128 ? by_type(std::integral_constant<int, 128>{}) : by_type(std::integral_constant<int, 64>{});
}

}  // namespace novakv
