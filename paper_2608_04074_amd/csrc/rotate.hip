// Norm and rotation of a layer's query and key heads, in one pass from the
// projection's rows to dense tensors (nova_kv_rotate_qkv) or, for keys and
// values, to a cache held in 4 bits (nova_kv_q4_append).
//
// A row is one head of one token.  D / 8 lanes hold it, 8 coordinates each, as
// two chunks of four; a lane's chunks are the two ends of its rotated pairs, so
// the rotation needs no other lane: with pairs (j, j + r/2) lane i < r/8 holds
// [4i, 4i + 4) and [4i + r/2, 4i + r/2 + 4), elsewhere and with neighbouring pairs
// [8i, 8i + 8).  Both ways its angles are 4i .. 4i + 3.
#include <type_traits>

#include "q4_internal.h"

namespace novakv {

namespace {

constexpr int kThreads = 256;

// Value of another lane of the 16-lane row (DPP).
template <int CTRL>
__device__ __forceinline__ float dpp(const float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, false));
}
template <int CTRL>
__device__ __forceinline__ double dpp(const double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, static_cast<int>(u), CTRL, 0xf, 0xf, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, static_cast<int>(u >> 32), CTRL, 0xf, 0xf, false);
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
__device__ __forceinline__ uint32_t bf16_any(const float x) {
  return x != x ? 0x7fc0u : bf16_rne(x);
}

// Four consecutive elements.
template <bool BF16>
__device__ __forceinline__ void load4(const void *p, const long long i, const bool vec, float *x) {
  if constexpr (BF16) {
    const uint16_t *h = static_cast<const uint16_t *>(p) + i;
    if (vec) {
      const uint2 w = *reinterpret_cast<const uint2 *>(h);
      x[0] = __uint_as_float(w.x << 16), x[1] = __uint_as_float(w.x & 0xffff0000u);
      x[2] = __uint_as_float(w.y << 16), x[3] = __uint_as_float(w.y & 0xffff0000u);
    } else {
      for (int j = 0; j < 4; ++j) x[j] = bf16_bits_to_float(h[j]);
    }
  } else {
    const float *f = static_cast<const float *>(p) + i;
    if (vec) {
      const float4 w = *reinterpret_cast<const float4 *>(f);
      x[0] = w.x, x[1] = w.y, x[2] = w.z, x[3] = w.w;
    } else {
      for (int j = 0; j < 4; ++j) x[j] = f[j];
    }
  }
}
template <bool BF16>
__device__ __forceinline__ void store4(void *p, const long long i, const float *x) {
  if constexpr (BF16) {
    *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(p) + i) =
        make_uint2(bf16_any(x[0]) | (bf16_any(x[1]) << 16), bf16_any(x[2]) | (bf16_any(x[3]) << 16));
  } else {
    *reinterpret_cast<float4 *>(static_cast<float *>(p) + i) = make_float4(x[0], x[1], x[2], x[3]);
  }
}

// Norm and rotation of a lane's 8 coordinates, in T.
template <int D, bool IL, typename T>
__device__ __forceinline__ void norm_rotate(T *y, const float *w, const bool norm, const float eps, const float *cs,
                                            const float *sn, const bool turns) {
  if (norm) {
    T ss = 0;
    for (int j = 0; j < 8; ++j) ss += y[j] * y[j];
    ss = reduce_row<D / 8>(ss, [](T a, T b) { return a + b; });
    const T r = static_cast<T>(1) / sqrt(ss / D + static_cast<T>(eps));
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
}

template <int D, bool BF16, bool IL, bool Q4>
__global__ __launch_bounds__(kThreads) void rotate_kernel(const RotateArgs a, const bool vec) {
  constexpr int kLanes = D / 8, kSlots = kThreads / kLanes;
  const int tok = blockIdx.x;
  const int b = tok / a.n_new, i = tok - b * a.n_new;
  if (a.new_lens && i >= a.new_lens[b]) return;
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

  const int lane = threadIdx.x % kLanes, slot = threadIdx.x / kLanes;
  const bool turns = lane < a.rotary_dim / 8;
  const int c0 = !IL && turns ? 4 * lane : 8 * lane;
  const int c1 = !IL && turns ? c0 + a.rotary_dim / 2 : c0 + 4;
  float cs[4], sn[4];
  if (turns) {
    const float *t = a.cos_sin + pos * a.rotary_dim + 4 * lane;
    load4<false>(t, 0, true, cs);
    load4<false>(t, a.rotary_dim / 2, true, sn);
  }

  const int heads = a.nq + a.nk + a.nv;
  for (int h = blockIdx.y * kSlots + slot; h < heads; h += gridDim.y * kSlots) {
    const int side = h < a.nq ? 0 : h < a.nq + a.nk ? 1 : 2;
    const HeadRows &src = side == 0 ? a.q : side == 1 ? a.k : a.v;
    const int hh = side == 0 ? h : side == 1 ? h - a.nq : h - a.nq - a.nk;
    const int n_heads = side == 0 ? a.nq : side == 1 ? a.nk : a.nv;
    const long long at = b * src.batch_stride + i * src.token_stride + static_cast<long long>(hh) * D;
    float x[8], w[8];
    load4<BF16>(src.data, at + c0, vec, x);
    load4<BF16>(src.data, at + c1, vec, x + 4);
    const float *weight = side == 0 ? a.q_norm : side == 1 ? a.k_norm : nullptr;
    if (weight) {
      weight += hh * (side == 0 ? a.q_norm_stride : a.k_norm_stride);
      load4<false>(weight, c0, true, w);
      load4<false>(weight, c1, true, w + 4);
    }
    void *out = side == 0 ? a.q_out : side == 1 ? a.k_out : a.v_out;
    const long long to = (static_cast<long long>(tok) * n_heads + hh) * D;
    if (!Q4 || side == 0) {
      norm_rotate<D, IL, float>(x, w, weight != nullptr, a.eps, cs, sn, turns && side < 2);
      store4<BF16>(out, to + c0, x);
      store4<BF16>(out, to + c1, x + 4);
      continue;
    }
    // 4 bits: everything that decides a code in fp64, so that the codes do not
    // depend on how a sum is ordered
    double y[8];
    bool odd = false;
    for (int j = 0; j < 8; ++j) y[j] = x[j];
    norm_rotate<D, IL, double>(y, w, weight != nullptr, a.eps, cs, sn, turns && side < 2);
    double lo = y[0], hi = y[0];
    for (int j = 0; j < 8; ++j) {
      odd |= !(fabs(y[j]) < __builtin_inf());
      lo = fmin(lo, y[j]);
      hi = fmax(hi, y[j]);
    }
    lo = reduce_row<kLanes>(lo, [](double p, double q) { return fmin(p, q); });
    hi = reduce_row<kLanes>(hi, [](double p, double q) { return fmax(p, q); });
    const float any_odd = reduce_row<kLanes>(odd ? 1.f : 0.f, [](float p, float q) { return fmaxf(p, q); });
    uint32_t sc = bf16_rne(static_cast<float>((hi - lo) / 15)), of = bf16_rne(static_cast<float>(lo));
    const bool nan = any_odd != 0.f || (sc & 0x7f80u) == 0x7f80u || (of & 0x7f80u) == 0x7f80u;
    if (nan) sc = of = 0x7fc0u;
    const float scale = bf16_bits_to_float(sc), offset = bf16_bits_to_float(of);
    const double step = scale, inv = 1 / step;
    uint32_t code[8];
    for (int j = 0; j < 8; ++j) {
      // the quotient rounded half to even: from an approximate quotient, then
      // by the remainder, which is exact
      const double u = y[j] - offset;
      double c = rint(u * inv);
      const double rem = __builtin_fma(-c, step, u);
      const bool c_odd = (static_cast<int>(fmin(fmax(c, -1.), 16.)) & 1) != 0;
      if (rem > 0.5 * step || (rem == 0.5 * step && c_odd)) c += 1;
      if (rem < -0.5 * step || (rem == -0.5 * step && c_odd)) c -= 1;
      code[j] = nan || step == 0 ? 0u : static_cast<uint32_t>(fmin(fmax(c, 0.), 15.));
    }
    const size_t row = row0 + static_cast<size_t>(hh) * a.layout.block_size;
    uint8_t *dst = (side == 1 ? a.k_codes : a.v_codes) + row * (D / 2);
    *reinterpret_cast<uint16_t *>(dst + c0 / 2) = code[0] | (code[1] << 4) | (code[2] << 8) | (code[3] << 12);
    *reinterpret_cast<uint16_t *>(dst + c1 / 2) = code[4] | (code[5] << 4) | (code[6] << 8) | (code[7] << 12);
    if (lane == 0) *reinterpret_cast<uint32_t *>((side == 1 ? a.k_sq : a.v_sq) + 2 * row) = sc | (of << 16);
    if (out) {
      for (int j = 0; j < 8; ++j) x[j] = scale * static_cast<float>(code[j]) + offset;
      store4<BF16>(out, to + c0, x);
      store4<BF16>(out, to + c1, x + 4);
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
  const dim3 grid(static_cast<unsigned>(a.batch) * a.n_new, (heads + slots - 1) / slots);
  auto go = [&](auto kernel) {
    kernel<<<grid, kThreads, 0, stream>>>(a, vec);
    return hipGetLastError();
  };
  auto by_cache = [&](auto d, auto bf16, auto il) {
    return a.q4 ? go(rotate_kernel<d(), bf16(), il(), true>) : go(rotate_kernel<d(), bf16(), il(), false>);
  };
  auto by_pairs = [&](auto d, auto bf16) {
    return a.interleaved ? by_cache(d, bf16, std::true_type{}) : by_cache(d, bf16, std::false_type{});
  };
  auto by_type = [&](auto d) { return a.bf16 ? by_pairs(d, std::true_type{}) : by_pairs(d, std::false_type{}); };
  return a.head_dim == 128 ? by_type(std::integral_constant<int, 128>{}) : by_type(std::integral_constant<int, 64>{});
}

}  // namespace novakv
