// Device code shared by the kernels that take 2-bit codes to matrix operands.
#pragma once

#include "chunk_internal.h"
#include "lut_common.h"

namespace novakv {
namespace chunk {

using lut::float4_t;
using lut::half2_t;
using lut::half8_t;

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

}  // namespace chunk
}  // namespace novakv
