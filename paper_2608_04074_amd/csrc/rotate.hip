// Norm and rotation of a layer's query and key heads, in one pass from the
// projection's rows to dense tensors (nova_kv_rotate_qkv) or, for keys and
// values, to a cache held in 4 bits (nova_kv_q4_append).
//
// A row is one head of one token.  D / 8 lanes hold it, 8 coordinates each, as
// two chunks of four; a lane's chunks are the two ends of its rotated pairs, so
// the rotation needs no other lane: with pairs (j, j + r/2) lane i < r/8 holds
// [4i, 4i + 4) and [4i + r/2, 4i + r/2 + 4), elsewhere and with neighbouring pairs
// [8i, 8i + 8).  Both ways its angles are 4i .. 4i + 3.
//
// Memory bounds it: 32 x 4096 tokens of 32 query and 8 + 8 KV heads of 128 in bf16 are
// rotated in 566 us, 3.22 GB read and written at 5.7 TB/s; to a cache (3.37 GB) 716 us, where
// the vector instructions of the codes take about 580 us beside it. One token: 3.8 to 4.7 us,
// 64 sequences' to a cache 5.0 us, launch and latency.
#include <type_traits>

#include "q4_internal.h"
#include "rotate_layout.h"

namespace novakv {

namespace {

constexpr int kThreads = 256;

// Value of another lane of the 16-lane row (DPP).
template <int CTRL>
__device__ __forceinline__ float dpp(const float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
template <int CTRL>
__device__ __forceinline__ double dpp(const double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_mov_dpp(static_cast<int>(u), CTRL, 0xf, 0xf, true);
  const uint32_t hi = __builtin_amdgcn_mov_dpp(static_cast<int>(u >> 32), CTRL, 0xf, 0xf, true);
  return __builtin_bit_cast(double, (static_cast<uint64_t>(hi) << 32) | lo);
}

// Reduction over the LANES lanes of a row: neighbours, pairs, then mirrored
// within 8 and within 16 lanes (every lane gets the same result).
template <int LANES, typename T, typename F>
__device__ __forceinline__ T reduce_row(T x, F f) {
  x = f(x, dpp<0xB1>(x));   // quad_perm [1, 0, 3, 2]
  x = f(x, dpp<0x4E>(x));   // quad_perm [2, 3, 0, 1]
  x = f(x, dpp<0x141>(x));  // row_half_mirror
  if constexpr (LANES == 16) x = f(x, dpp<0x140>(x));  // row_mirror
  return x;
}

__device__ __forceinline__ uint32_t bf16_rne(const float x) {  // finite x (or overflow to infinity)
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  return (u + 0x7fffu + ((u >> 16) & 1u)) >> 16;
}

// Four consecutive elements as they lie (VEC: aligned to their 8 or 16 bytes),
// converted where they are used, so that a load issued early is not waited for.
template <bool BF16>
using Raw4 = std::conditional_t<BF16, uint2, float4>;
template <bool BF16, bool VEC>
__device__ __forceinline__ Raw4<BF16> load4(const void *p) {
  if constexpr (VEC) return *static_cast<const Raw4<BF16> *>(p);
  if constexpr (BF16) {
    const uint16_t *h = static_cast<const uint16_t *>(p);
    return make_uint2(h[0] | (static_cast<uint32_t>(h[1]) << 16), h[2] | (static_cast<uint32_t>(h[3]) << 16));
  } else {
    const float *f = static_cast<const float *>(p);
    return make_float4(f[0], f[1], f[2], f[3]);
  }
}
__device__ __forceinline__ void to_floats(const uint2 w, float *x) {
  x[0] = __uint_as_float(w.x << 16), x[1] = __uint_as_float(w.x & 0xffff0000u);
  x[2] = __uint_as_float(w.y << 16), x[3] = __uint_as_float(w.y & 0xffff0000u);
}
__device__ __forceinline__ void to_floats(const float4 w, float *x) { x[0] = w.x, x[1] = w.y, x[2] = w.z, x[3] = w.w; }
template <bool BF16>
__device__ __forceinline__ void store4(char *p, const float *x) {
  if constexpr (BF16) {
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    *reinterpret_cast<bf16x4 *>(p) =
        bf16x4{static_cast<__bf16>(x[0]), static_cast<__bf16>(x[1]), static_cast<__bf16>(x[2]), static_cast<__bf16>(x[3])};
  } else {
    *reinterpret_cast<float4 *>(p) = make_float4(x[0], x[1], x[2], x[3]);
  }
}

// Norm and rotation of a lane's 8 coordinates, in T; the mean square with eps (1 without a norm).
template <int D, bool IL, typename T>
__device__ __forceinline__ T norm_rotate(T *y, const float *w, const bool norm, const float eps, const float *cs,
                                         const float *sn, const bool turns) {
  T v = 1;
  if (norm) {
    T ss = 0;
    for (int j = 0; j < 8; ++j) ss += y[j] * y[j];
    ss = reduce_row<D / 8>(ss, [](T a, T b) { return a + b; });
    v = ss * static_cast<T>(1. / D) + static_cast<T>(eps);
    T r;
    if constexpr (std::is_same_v<T, float>) r = v > 0x1p-100f ? __builtin_amdgcn_rsqf(v) : 1.f / sqrtf(v);  // within 2 u
    else r = 1 / sqrt(v);
    for (int j = 0; j < 8; ++j) y[j] *= r * static_cast<T>(w[j]);
  }
  if (turns) {
    for (int j = 0; j < 4; ++j) {
      T &a = IL ? y[2 * j] : y[j];
      T &b = IL ? y[2 * j + 1] : y[4 + j];
      const T c = cs[j], s = sn[j], a0 = a;
      a = a0 * c - b * s;
      b = b * c + a0 * s;
    }
  }
  return v;
}

// A row's 4-bit codes (clamped by the caller) and its scale and offset in a word, everything that decides
// them in fp64, so that they do not depend on how a sum is ordered.
template <int D, bool IL>
__device__ __forceinline__ void quantize_wide(const float *x, const float *w, const bool norm, const float eps, const float *cs,
                                              const float *sn, const bool turns, float *code, uint32_t &sq) {
  double y[8];
  bool odd = false;
  for (int j = 0; j < 8; ++j) y[j] = x[j];
  norm_rotate<D, IL, double>(y, w, norm, eps, cs, sn, turns);
  double lo = y[0], hi = y[0];
  for (int j = 0; j < 8; ++j) {
    odd |= !(fabs(y[j]) < __builtin_inf());
    lo = fmin(lo, y[j]);
    hi = fmax(hi, y[j]);
  }
  lo = reduce_row<D / 8>(lo, [](double p, double q) { return fmin(p, q); });
  hi = reduce_row<D / 8>(hi, [](double p, double q) { return fmax(p, q); });
  const float any_odd = reduce_row<D / 8>(odd ? 1.f : 0.f, [](float p, float q) { return fmaxf(p, q); });
  uint32_t sc = bf16_rne(static_cast<float>((hi - lo) / 15)), of = bf16_rne(static_cast<float>(lo));
  const bool nan = any_odd != 0.f || (sc & 0x7f80u) == 0x7f80u || (of & 0x7f80u) == 0x7f80u;
  if (nan) sc = of = 0x7fc0u;
  const float offset = bf16_bits_to_float(of);
  const double step = bf16_bits_to_float(sc), inv = 1 / step;
  for (int j = 0; j < 8; ++j) {
    // the quotient rounded half to even: from an approximate quotient, then
    // by the remainder, which is exact
    const double u = y[j] - offset;
    double c = rint(u * inv);
    const double rem = __builtin_fma(-c, step, u);
    const bool c_odd = (static_cast<int>(fmin(fmax(c, -1.), 16.)) & 1) != 0;
    if (rem > 0.5 * step || (rem == 0.5 * step && c_odd)) c += 1;
    if (rem < -0.5 * step || (rem == -0.5 * step && c_odd)) c -= 1;
    code[j] = nan || step == 0 ? 0.f : static_cast<float>(fmin(fmax(c, 0.), 15.));
  }
  sq = sc | (of << 16);
}

// Whether a value known to within `off` might round to another bf16 number:
// fp32 bits next to the middle of two. (Zero, denormals and what overflows: yes.)
__device__ __forceinline__ bool near_bf16_border(const float v, const float off) {
  const uint32_t u = __builtin_bit_cast(uint32_t, v);
  const float middle = __builtin_bit_cast(float, (u & 0xffff0000u) | 0x8000u);
  const uint32_t e = u & 0x7f800000u;
  return !(fabsf(v - middle) > off) || e == 0 || e >= 0x7f000000u;
}

// The same codes from fp32 arithmetic, where its rounding cannot have decided one:
// returns whether the row is sure. The error of y = norm and rotation, u = 2^-24 and
// m the row's largest |y|: 13 u of the sum of squares (all positive: 8 + 4 additions),
// half of it in the reciprocal root, with eps, the root's 2 u and two products below
// 13 u of a coordinate; the rotation's two products and sum below 15 u (|a| + |b|) <=
// 30 u m. Below 32 u m = 2^-19 m all told; values are exact.
template <int D, bool IL>
__device__ __forceinline__ bool quantize_fast(const float *x, const float *w, const bool norm, const float eps, const float *cs,
                                              const float *sn, const bool turns, float *code, uint32_t &sq) {
  float y[8];
  for (int j = 0; j < 8; ++j) y[j] = x[j];
  const float square = norm_rotate<D, IL, float>(y, w, norm, eps, cs, sn, turns);
  float lo = y[0], hi = y[0], all = y[0];  // all: not finite where a coordinate is not (or the sum overflows)
  for (int j = 1; j < 8; ++j) {
    lo = fminf(lo, y[j]);
    hi = fmaxf(hi, y[j]);
    all += y[j];
  }
  lo = reduce_row<D / 8>(lo, [](float p, float q) { return fminf(p, q); });
  hi = reduce_row<D / 8>(hi, [](float p, float q) { return fmaxf(p, q); });
  const float m = fmaxf(fabsf(lo), fabsf(hi));
  const float off = norm || turns ? m * 0x1p-19f : 0.f;
  const float range = hi - lo, scale32 = range * (1.f / 15.f);
  // the roundings of the range, of 1/15 and of their product: below 4 u
  bool sure = all - all == 0.f && !near_bf16_border(scale32, 2.f / 15.f * off + scale32 * 0x1p-22f);
  // squares, or the root's product with a weight, that left the normal numbers have lost more
  sure = sure && (!norm || (square > 0x1p-100f && m > 0x1p-60f));
  sure = sure && (off == 0.f ? (__builtin_bit_cast(uint32_t, lo) & 0x7f800000u) < 0x7f000000u : !near_bf16_border(lo, off));
  const uint32_t sc = bf16_rne(scale32), of = bf16_rne(lo);
  const float step = bf16_bits_to_float(sc), offset = bf16_bits_to_float(of);
  const float inv = __builtin_amdgcn_rcpf(step);
  sq = sc | (of << 16);
  float u[8], worst = 0.f;
  for (int j = 0; j < 8; ++j) {
    u[j] = y[j] - offset;
    code[j] = rintf(u[j] * inv);
    worst = fmaxf(worst, fabsf(__builtin_fmaf(-code[j], step, u[j])));
  }
  // a remainder so near half a step that y's error, or the subtraction's (of at
  // most 16 steps), may have decided
  const float near = off + 0x1p-20f * step;
  if (!(worst < 0.5f * step - near)) {
    for (int j = 0; j < 8; ++j) {
      const float c = code[j], rem = __builtin_fmaf(-c, step, u[j]), beyond = fabsf(rem) - 0.5f * step;
      if (beyond < -near || c < -1.f || c > 16.f) continue;
      // exact where the subtraction was (and y is): then a tie goes to the even code
      const float bb = u[j] - y[j], lost = (y[j] - (u[j] - bb)) - (offset + bb);
      sure = sure && off == 0.f && lost == 0.f && beyond <= near;
      if (beyond > 0.f || (beyond == 0.f && (static_cast<int>(c) & 1))) code[j] += rem > 0.f ? 1.f : -1.f;
    }
  }
  return sure;
}

// A row's codes: in fp32, and again in fp64 where any of the wave's rows needs it
// (the other rows' results are the same). 32 x 4096 tokens: 716 us, 1568 us all in fp64.
template <int D, bool IL>
__device__ __forceinline__ void quantize(const float *x, const float *w, const bool norm, const float eps, const float *cs,
                                         const float *sn, const bool turns, float *code, uint32_t &sq) {
  const bool sure = quantize_fast<D, IL>(x, w, norm, eps, cs, sn, turns, code, sq);
  // every lane of a row takes the same way: its codes and its scale belong together
  if (reduce_row<D / 8>(sure ? 0.f : 1.f, [](float p, float q) { return fmaxf(p, q); }) != 0.f)
    quantize_wide<D, IL>(x, w, norm, eps, cs, sn, turns, code, sq);
}

// VEC: the rows' base and strides are multiples of 16 bytes. AHEAD: rows of a
// lane requested at once. FAST: quantize in fp32 where that decides the codes.
template <int D, bool BF16, bool IL, bool Q4, bool VEC, int AHEAD, bool FAST>
__global__ __launch_bounds__(kThreads) void rotate_kernel(const RotateArgs a) {
  constexpr int kLanes = D / 8, kSlots = kThreads / kLanes, kElem = BF16 ? 2 : 4;
  const int tok = blockIdx.x;
  const int b = tok / a.n_new, i = tok - b * a.n_new;
  if (a.new_lens && i >= a.new_lens[b]) return;
  const int lane = threadIdx.x % kLanes, slot = threadIdx.x / kLanes;
  const int heads = a.nq + a.nk + a.nv;
  const rotate::LaneChunks chunks = rotate::lane_chunks(lane, a.rotary_dim, IL);
  const bool turns = chunks.turns;
  const int c0 = chunks.c0, c1 = chunks.c1;
  // the token's rows on each side (addresses in scalar registers)
  auto rows_of = [&](const HeadRows &r) {
    return static_cast<const char *>(r.data) + (b * r.batch_stride + i * r.token_stride) * kElem;
  };
  const char *const q_rows = rows_of(a.q), *const k_rows = rows_of(a.k), *const v_rows = rows_of(a.v);
  auto outs_of = [&](void *out, const int n_heads) {
    return out ? static_cast<char *>(out) + static_cast<long long>(tok) * n_heads * (D * kElem) : nullptr;
  };
  char *const q_out = outs_of(a.q_out, a.nq), *const k_out = outs_of(a.k_out, a.nk), *const v_out = outs_of(a.v_out, a.nv);
  struct Row {
    int side, head;  // 0: query, 1: key, 2: value; -1: none
    Raw4<BF16> x[2];
  };
  const int first = (blockIdx.y * kSlots * AHEAD) + slot;
  Row rows[AHEAD];
#pragma unroll
  for (int y = 0; y < AHEAD; ++y) {
    const int h = first + y * kSlots;
    Row &r = rows[y];
    r.side = h < a.nq ? 0 : h < a.nq + a.nk ? 1 : h < heads ? 2 : -1;
    r.head = r.side == 0 ? h : r.side == 1 ? h - a.nq : h - a.nq - a.nk;
    if (r.side < 0) continue;
    const char *p = (r.side == 0 ? q_rows : r.side == 1 ? k_rows : v_rows) + r.head * (D * kElem);
    r.x[0] = load4<BF16, VEC>(p + c0 * kElem);
    r.x[1] = load4<BF16, VEC>(p + c1 * kElem);
  }
  const long long pos = a.start_pos ? static_cast<long long>(a.start_pos[b]) + i : i;
  if (a.rotary_dim && (pos < 0 || pos >= a.num_positions)) return;
  size_t row0 = 0;  // the cache row of KV head 0
  if constexpr (Q4) {
    const long long cap = static_cast<long long>(a.layout.block_size) * a.layout.blocks_per_seq;
    if (pos < 0 || pos >= cap) return;
    const int blk = static_cast<int>(pos) / a.layout.block_size;
    const long long logical = static_cast<long long>(b) * a.layout.blocks_per_seq + blk;
    const long long phys = a.layout.block_table ? a.layout.block_table[logical] : logical;
    if (phys < 0 || phys >= a.num_blocks) return;
    row0 = static_cast<size_t>(phys) * a.nk * a.layout.block_size + (static_cast<int>(pos) - blk * a.layout.block_size);
  }
  float cs[4], sn[4];
  if (turns) {
    const float *t = a.cos_sin + pos * a.rotary_dim + 4 * lane;
    to_floats(load4<false, true>(t), cs);
    to_floats(load4<false, true>(t + a.rotary_dim / 2), sn);
  }

#pragma unroll
  for (int y = 0; y < AHEAD; ++y) {
    const int side = rows[y].side, hh = rows[y].head;
    if (side < 0) continue;
    float x[8], w[8];
    to_floats(rows[y].x[0], x);
    to_floats(rows[y].x[1], x + 4);
    const float *weight = side == 0 ? a.q_norm : side == 1 ? a.k_norm : nullptr;
    if (weight) {
      weight += hh * (side == 0 ? a.q_norm_stride : a.k_norm_stride);
      to_floats(load4<false, true>(weight + c0), w);
      to_floats(load4<false, true>(weight + c1), w + 4);
    }
    char *out = side == 0 ? q_out : side == 1 ? k_out : v_out;
    const int to0 = (hh * D + c0) * kElem, to1 = (hh * D + c1) * kElem;
    if (!Q4 || side == 0) {
      norm_rotate<D, IL, float>(x, w, weight != nullptr, a.eps, cs, sn, turns && side < 2);
      store4<BF16>(out + to0, x);
      store4<BF16>(out + to1, x + 4);
      continue;
    }
    float code[8];
    uint32_t sq;
    if constexpr (FAST) quantize<D, IL>(x, w, weight != nullptr, a.eps, cs, sn, turns && side == 1, code, sq);
    else quantize_wide<D, IL>(x, w, weight != nullptr, a.eps, cs, sn, turns && side == 1, code, sq);
    const size_t row = row0 + static_cast<size_t>(hh) * a.layout.block_size;
    uint8_t *dst = (side == 1 ? a.k_codes : a.v_codes) + row * (D / 2);
    for (int j = 0; j < 8; ++j) code[j] = __builtin_amdgcn_fmed3f(code[j], 0.f, 15.f);
    auto four = [](const float *c) {  // 16 bits, exact in fp32
      return static_cast<uint32_t>(__builtin_fmaf(__builtin_fmaf(__builtin_fmaf(c[3], 16.f, c[2]), 16.f, c[1]), 16.f, c[0]));
    };
    const uint32_t packed = four(code) | (four(code + 4) << 16);
    const rotate::CodeStore how = rotate::code_store(chunks, a.rotary_dim, IL);
    if (how == rotate::CodeStore::kApart) {
      *reinterpret_cast<uint16_t *>(dst + c0 / 2) = packed;
      *reinterpret_cast<uint16_t *>(dst + c1 / 2) = packed >> 16;
    } else {
      uint32_t word = packed;
      if (how == rotate::CodeStore::kExchange) {
        const uint32_t other = __builtin_amdgcn_update_dpp(0, static_cast<int>(packed), 0xB1, 0xf, 0xf, false);  // lane ^ 1
        word = lane & 1 ? (other >> 16) | (packed & 0xffff0000u) : (packed & 0xffffu) | (other << 16);
      }
      *reinterpret_cast<uint32_t *>(dst + rotate::word_at(chunks, how, lane)) = word;
    }
    if (lane == 0) *reinterpret_cast<uint32_t *>((side == 1 ? a.k_sq : a.v_sq) + 2 * row) = sq;
    if (out) {
      const float scale = bf16_bits_to_float(sq & 0xffffu), offset = bf16_bits_to_float(sq >> 16);
      for (int j = 0; j < 8; ++j) x[j] = __builtin_fmaf(scale, code[j], offset);
      store4<BF16>(out + to0, x);
      store4<BF16>(out + to1, x + 4);
    }
  }
}

// Whether a side's rows can be read 16 bytes at a time from any multiple of
// four elements.
bool vector_rows(const HeadRows &r, const int elem) {
  return !r.data || (reinterpret_cast<uintptr_t>(r.data) % 16 == 0 && r.batch_stride * elem % 16 == 0 &&
                     r.token_stride * elem % 16 == 0);
}

}  // namespace

hipError_t launch_rotate(const RotateArgs &a, hipStream_t stream) {
  const int elem = a.bf16 ? 2 : 4;
  const bool vec = vector_rows(a.q, elem) && vector_rows(a.k, elem) && vector_rows(a.v, elem);
  const int slots = kThreads / (a.head_dim / 8), heads = a.nq + a.nk + a.nv;
  const unsigned tokens = static_cast<unsigned>(a.batch) * a.n_new;
  // Many tokens: a lane requests three rows at once (32 x 4096 tokens rotated in
  // 566 us, one row at a time 693 us; with few, more workgroups share them: 1839
  // tokens 11.9 us against 12.8 us), and quantizes in fp32 with a second look in fp64
  // (716 us against 1568 us; of 64 tokens some wave always takes both ways: 5.5 us
  // against 4.9 us in fp64 alone).
  auto go = [&](auto d, auto bf16, auto il, auto q4, auto vec) {
    const auto launch = [&](auto ahead, auto fast) {
      const dim3 grid(tokens, (heads + slots * ahead() - 1) / (slots * ahead()));
      rotate_kernel<d(), bf16(), il(), q4(), vec(), ahead(), fast()><<<grid, kThreads, 0, stream>>>(a);
      return hipGetLastError();
    };
    constexpr std::integral_constant<int, 1> one{};
    constexpr std::integral_constant<int, 3> three{};
    if (tokens >= 8192) return launch(three, std::bool_constant<q4()>{});
    if constexpr (q4())
      if (tokens >= 512) return launch(one, std::true_type{});
    return launch(one, std::false_type{});
  };
  using std::false_type;
  using std::true_type;
  auto by_rows = [&](auto d, auto bf16, auto il, auto q4) { return vec ? go(d, bf16, il, q4, true_type{}) : go(d, bf16, il, q4, false_type{}); };
  auto by_cache = [&](auto d, auto bf16, auto il) { return a.q4 ? by_rows(d, bf16, il, true_type{}) : by_rows(d, bf16, il, false_type{}); };
  auto by_pairs = [&](auto d, auto bf16) { return a.interleaved ? by_cache(d, bf16, true_type{}) : by_cache(d, bf16, false_type{}); };
  auto by_type = [&](auto d) { return a.bf16 ? by_pairs(d, true_type{}) : by_pairs(d, false_type{}); };
  return a.head_dim == 128 ? by_type(std::integral_constant<int, 128>{}) : by_type(std::integral_constant<int, 64>{});
}

}  // namespace novakv
