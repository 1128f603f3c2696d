// Device code shared by the kernels of attention over a 4-bit cache.
#pragma once

#include "lut_common.h"
#include "q4_internal.h"

namespace novakv {
namespace q4 {

using lut::add_rows16;
using lut::add_rows32;
using lut::float4_t;
using lut::half8_t;
using lut::max_rows16;
using lut::max_rows32;

// The fp16 cores add the products of eight slots after cutting them about 24 bits
// below the largest, then round to nearest (measured). A sum of small multiples of
// one unit is therefore exact; one of products far apart loses what lies below
// the cut, towards one side, which fp32 outputs would show. So with fp32
// queries a probability is split into two fixed-point parts of 11 bits and the rest.
constexpr float kNone = -__builtin_inff();
// Most splits of a tile's span: their weights lie in LDS (up to 32 rows a tile; 128 or 256).
constexpr int kMaxSplits = 96, kMaxSplitsTiled = 32;
// Arrival counters of a workspace: a span is split only where at most this many
// workgroups run, so no call's partials lie on another shape's counters.
constexpr int kMaxCounters = 1024;

__device__ __forceinline__ float exp2_raw(const float x) { return __builtin_amdgcn_exp2f(x); }

// 2^(d / 2), to be multiplied twice: a sum of weights beside small values reaches
// 2^110, and one factor 2^d below 2^-126 would take it to zero.
__device__ __forceinline__ float half_factor(const float d) { return exp2_raw(0.5f * d); }

typedef int int4_t __attribute__((ext_vector_type(4)));

// Codes k and k + 4 of a word as fp16 denormals in a word: c * 2^-24, times 16 for odd k.
template <int K>
__device__ __forceinline__ lut::half2_t code_pair(const uint32_t w) {
  return __builtin_bit_cast(lut::half2_t, (K < 2 ? w : w >> 8) & (K % 2 ? 0x00f000f0u : 0x000f000fu));
}
// The same as (c - 8) * 2^-9.
template <int K>
__device__ __forceinline__ uint32_t value_pair(const uint32_t w) {
  const _Float16 up = K % 2 ? 0x1p11f : 0x1p15f, centre = -0x1p-6f;
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(code_pair<K>(w), lut::half2_t{up, up}, lut::half2_t{centre, centre}));
}

// Coordinate of a lane's output value: tile t, accumulator register i, lane row j.
template <int D>
__device__ __forceinline__ int out_coord(const int t, const int i, const int j) {
  const int m = 4 * j + i;
  return D == 128 ? 8 * m + t : 8 * (m & 7) + 4 * (m >> 3) + t;
}

// Split partials meet through memory as device-coherent words (lut_common.h).
__device__ __forceinline__ void publish4(float *p, const float4 v) {
  uint64_t *w = reinterpret_cast<uint64_t *>(p);
  const uint64_t lo = (static_cast<uint64_t>(__float_as_uint(v.y)) << 32) | __float_as_uint(v.x);
  const uint64_t hi = (static_cast<uint64_t>(__float_as_uint(v.w)) << 32) | __float_as_uint(v.z);
  __hip_atomic_store(w, lo, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __hip_atomic_store(w + 1, hi, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void publish2(float *p, const float x, const float y) {
  __hip_atomic_store(reinterpret_cast<uint64_t *>(p), (static_cast<uint64_t>(__float_as_uint(y)) << 32) | __float_as_uint(x),
                     __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 fetch2(const float *p) {
  const uint64_t w = __hip_atomic_load(reinterpret_cast<uint64_t *>(const_cast<float *>(p)), __ATOMIC_RELAXED,
                                       __HIP_MEMORY_SCOPE_AGENT);
  return make_float2(__uint_as_float(static_cast<uint32_t>(w)), __uint_as_float(static_cast<uint32_t>(w >> 32)));
}

__device__ __forceinline__ void store_out(const Q4AttnArgs &a, const size_t at, const float4 v) {
  if (a.q_bf16) {
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    const bf16x4 o = {static_cast<__bf16>(v.x), static_cast<__bf16>(v.y), static_cast<__bf16>(v.z), static_cast<__bf16>(v.w)};
    *reinterpret_cast<bf16x4 *>(static_cast<__bf16 *>(a.out) + at) = o;
  } else {
    *reinterpret_cast<float4 *>(static_cast<float *>(a.out) + at) = v;
  }
}

// A workgroup's tile of rows (query tokens times query heads of a KV head) and
// its split of their span.
struct Tile {
  int unit, b, kv, tile, split;
  int S, nb, rows_valid;  // cached tokens, the sequence's queries, its rows
  int row0, row1;         // rows of the tile
  int lo, base, t0, t1;   // first attended position; the split's tokens [t0, t1) from a multiple of 32 on
  // attended positions of a row: [first_pos, last_pos]
  __device__ __forceinline__ int last_pos(const Q4AttnArgs &a, const int row) const { return S - nb + row / a.gqa; }
  __device__ __forceinline__ int first_pos(const Q4AttnArgs &a, const int row) const {
    return a.window > 0 ? max(0, last_pos(a, row) + 1 - a.window) : 0;
  }
};

// The workgroup's place. Consecutive tiles, which read the same rows and pages,
// run on one XCD.
__device__ __forceinline__ void place_tile(const Q4AttnArgs &a, const int rows, Tile &g) {
  int wg = lut::xcd_contiguous(blockIdx.x, gridDim.x);
  g.split = wg % a.n_split;
  wg /= a.n_split;
  g.tile = a.row_tiles - 1 - wg % a.row_tiles;  // the last queries, which attend most, first
  g.unit = wg / a.row_tiles;
  g.b = g.unit / a.num_kv_heads;
  g.kv = g.unit - g.b * a.num_kv_heads;
  g.row0 = g.tile * rows;
}
// Its rows and tokens; false: the tile has no rows. `step`: tokens that a split is
// a multiple of.
__device__ __forceinline__ bool find_span(const Q4AttnArgs &a, const int rows, const int step, Tile &g) {
  g.S = min(max(a.seq_lens[g.b], 0), a.max_seq_len);
  g.nb = a.q_lens ? min(max(a.q_lens[g.b], 0), a.n_q) : a.n_q;
  g.rows_valid = g.nb * a.gqa;
  if (g.row0 >= g.rows_valid) return false;
  g.row1 = min(g.row0 + rows, g.rows_valid);
  g.lo = g.first_pos(a, g.row0);
  g.base = g.lo & ~31;
  const int span = max(0, g.last_pos(a, g.row1 - 1) + 1 - g.base);
  const int per = ((span + a.n_split - 1) / a.n_split + step - 1) / step * step;
  g.t0 = min(g.base + g.split * per, g.base + span);
  g.t1 = min(g.t0 + per, g.base + span);
  return true;
}

// LDS of finish_rows.
template <int D, int NT, int W, bool TILED>
struct FinishLds {
  static constexpr int kRows = 16 * NT * (TILED ? W : 1), kStride = D + 4;
  // the merge over waves, then the splits' weights and sums
  static constexpr int kMerge = TILED ? 2 * kRows * kMaxSplitsTiled : W * 16 * NT * kStride;
  float *merge;             // [kMerge], 16-byte aligned
  float (*ref)[16 * NT], (*sum)[16 * NT];  // [W]
  float *inv;               // [kRows]
  int *last;
};

// Where a tile's rows and partials lie, and what makes outputs of them.
template <int D, int kRows>
struct TileRows {
  const Q4AttnArgs &a;
  const Tile &g;
  static constexpr size_t kSlot = static_cast<size_t>(kRows) * (D + 2);  // floats of a split's partials
  __device__ __forceinline__ int rows_here() const { return g.row1 - g.row0; }
  __device__ __forceinline__ int head_of(const int r) const { return g.kv * a.gqa + (g.row0 + r) % a.gqa; }
  __device__ __forceinline__ size_t out_at(const int r) const {
    return ((static_cast<size_t>(g.b) * a.n_q + (g.row0 + r) / a.gqa) * a.num_q_heads + head_of(r)) * D;
  }
  // the split's own partials (nullptr: the tile has one split)
  __device__ __forceinline__ float *part() const {
    return a.n_split > 1 ? a.part + ((static_cast<size_t>(g.unit) * a.row_tiles + g.tile) * a.n_split + g.split) * kSlot : nullptr;
  }
  // 1 / the sum of a row's weights with its sink; 0 where nothing is attended
  __device__ __forceinline__ float inverse(const int r, const float most, float l) const {
    if (a.sinks && most != kNone) l += exp2_raw(a.sinks[head_of(r)] * 1.44269504088896341f - most);
    return most == kNone ? 0.f : 1.f / l;
  }
  static __device__ __forceinline__ float4 scaled(const float4 v, const float f) { return make_float4(v.x * f, v.y * f, v.z * f, v.w * f); }
};

// Over the splits, once a workgroup has published its partials: the last one to arrive
// merges them, in their order. n: the thread's lane modulo 16.
template <int D, int NT, int W, bool TILED>
__device__ __forceinline__ void merge_splits(const Q4AttnArgs &a, const Tile &g, const FinishLds<D, NT, W, TILED> &lds, const int n) {
  constexpr int kThreads = 64 * W, kRows = FinishLds<D, NT, W, TILED>::kRows;
  const TileRows<D, kRows> place{a, g};
  const int rows_here = place.rows_here();
  const size_t slot = place.kSlot;
  float *const s_merge = lds.merge, *const s_inv = lds.inv;
  int &s_last = *lds.last;
  auto out_at = [&](const int r) { return place.out_at(r); };
  auto inverse = [&](const int r, const float most, const float l) { return place.inverse(r, most, l); };
  auto scaled = [&](const float4 v, const float f) { return place.scaled(v, f); };
  __builtin_amdgcn_s_waitcnt(0);  // this thread's words have landed
  __syncthreads();
  int *counter = a.counters + static_cast<size_t>(g.unit) * a.row_tiles + g.tile;
  if (threadIdx.x == 0)
    s_last = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == a.n_split - 1;
  __syncthreads();
  if (!s_last) return;
  if (threadIdx.x == 0) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  const float *parts = place.part() - g.split * slot;
  float2 *weight = reinterpret_cast<float2 *>(s_merge);
  // All words are requested before any is used: the statistics, and each
  // thread's first values (in groups that share the splits where there are fewer
  // chunks than threads).
  const int items = rows_here * (D / 4);
  const int groups = min(8, max(1, kThreads / items));
  const int group = groups > 1 ? static_cast<int>(threadIdx.x) / items : 0;
  const int item = groups > 1 ? static_cast<int>(threadIdx.x) % items : static_cast<int>(threadIdx.x);
  constexpr int kAhead = 8;
  float4 v[kAhead];
  auto fetch_values = [&](const int x, const int first) {
    const float *src = parts + (x / (D / 4)) * D + 4 * (x % (D / 4));
    for (int y = 0; y < kAhead; ++y) {
      const int u = min(first + y * groups, a.n_split - 1);
      const float2 lo2 = fetch2(src + u * slot), hi2 = fetch2(src + u * slot + 2);
      v[y] = make_float4(lo2.x, lo2.y, hi2.x, hi2.y);
    }
  };
  const bool mine = group < groups && item < items;
  for (int x = threadIdx.x; x < rows_here * a.n_split; x += kThreads) {
    const int r = x / a.n_split, u = x - r * a.n_split;
    weight[x] = fetch2(parts + u * slot + kRows * D + 2 * r);
  }
  if (mine) fetch_values(item, group);
  __syncthreads();
  for (int r = threadIdx.x / 16; r < rows_here; r += kThreads / 16) {  // 16 lanes a row
    float most = kNone, l = 0.f;
    for (int x = n; x < a.n_split; x += 16) most = fmaxf(most, weight[r * a.n_split + x].x);
    most = fmaxf(most, lut::row_ror<1>(most));
    most = fmaxf(most, lut::row_ror<2>(most));
    most = fmaxf(most, lut::row_ror<4>(most));
    most = fmaxf(most, lut::row_ror<8>(most));
    for (int x = n; x < a.n_split; x += 16) {
      const float2 ml = weight[r * a.n_split + x];
      // A split of no weight counts all the same: it may hold a NaN. One that attends nothing has weight -1.
      const float f = ml.x == kNone ? -1.f : half_factor(ml.x - most);
      if (ml.x != kNone) l += f * ml.y * f;
      weight[r * a.n_split + x].x = f;
    }
    l += lut::row_ror<1>(l);
    l += lut::row_ror<2>(l);
    l += lut::row_ror<4>(l);
    l += lut::row_ror<8>(l);
    if (n == 0) s_inv[r] = inverse(r, most, l);
  }
  __syncthreads();
  float4 *sums = reinterpret_cast<float4 *>(weight + rows_here * a.n_split + (rows_here * a.n_split & 1));
  for (int x = item; mine && x < items; x += kThreads) {
    const int r = x / (D / 4), c = 4 * (x % (D / 4));
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int first = group; first < a.n_split; first += kAhead * groups) {
      if (x != item || first != group) fetch_values(x, first);
      for (int y = 0; y < kAhead; ++y) {
        const int u = first + y * groups;
        const float f = u < a.n_split ? weight[r * a.n_split + u].x : -1.f;
        if (f != -1.f) o.x += f * v[y].x * f, o.y += f * v[y].y * f, o.z += f * v[y].z * f, o.w += f * v[y].w * f;
      }
    }
    if (groups > 1) {
      sums[group * items + x] = o;
      break;
    }
    store_out(a, out_at(r) + c, scaled(o, s_inv[r]));
  }
  if (groups > 1) {
    __syncthreads();
    if (static_cast<int>(threadIdx.x) < items) {
      const int r = threadIdx.x / (D / 4), c = 4 * (threadIdx.x % (D / 4));
      float4 o = sums[threadIdx.x];
      for (int g = 1; g < groups; ++g) {
        const float4 y = sums[g * items + threadIdx.x];
        o.x += y.x, o.y += y.y, o.z += y.z, o.w += y.w;
      }
      store_out(a, out_at(r) + c, scaled(o, s_inv[r]));
    }
  }
}

// Writes a tile's outputs from its waves' partials: out = acc / sum of a row's
// weights exp2(z - ref). The waves share the rows, or (TILED) have 16 NT each.
template <int D, int NT, int W, bool TILED>
__device__ __forceinline__ void finish_rows(const Q4AttnArgs &a, const Tile &g, const FinishLds<D, NT, W, TILED> &lds,
                                            const int wave, const int lane, const float4_t (&acc)[NT][D / 16],
                                            const float (&ref)[NT], const float (&sum)[NT]) {
  using Lds = FinishLds<D, NT, W, TILED>;
  constexpr int kThreads = 64 * W, kWaves = W, kTiles = D / 16, kRows = Lds::kRows, kStride = Lds::kStride;
  const int n = lane & 15, j = lane >> 4;
  const int wg_row0 = g.row0;
  const int row0 = g.row0 + (TILED ? wave * 16 * NT : 0);
  float *const s_merge = lds.merge;
  auto s_ref = lds.ref, s_sum = lds.sum;
  const TileRows<D, kRows> place{a, g};
  const int rows_here = place.rows_here();
  float *const part = place.part();
  auto out_at = [&](const int r) { return place.out_at(r); };
  auto inverse = [&](const int r, const float most, const float l) { return place.inverse(r, most, l); };
  auto scaled = [&](const float4 v, const float f) { return place.scaled(v, f); };
  // a lane's values in chunks of four coordinates
  auto chunk = [&](const int t, const int x) {
    const int o = 4 * (x / 4), i = x % 4;
    return make_float4(acc[t][o][i], acc[t][o + 1][i], acc[t][o + 2][i], acc[t][o + 3][i]);
  };
  auto chunk_coord = [&](const int x) { return out_coord<D>(4 * (x / 4), x % 4, j); };
  if constexpr (!TILED) {  // over the waves, which hold the same rows
    for (int t = 0; t < NT; ++t) {
      float *row = s_merge + (wave * 16 * NT + 16 * t + n) * kStride;
      for (int x = 0; x < kTiles; ++x) *reinterpret_cast<float4 *>(row + chunk_coord(x)) = chunk(t, x);
      if (j == 0) s_ref[wave][16 * t + n] = ref[t], s_sum[wave][16 * t + n] = sum[t];
    }
    __syncthreads();
    for (int x = threadIdx.x; x < rows_here * (D / 4); x += kThreads) {
      const int r = x / (D / 4), c = 4 * (x % (D / 4));
      float most = kNone, l = 0.f;
      for (int u = 0; u < kWaves; ++u) most = fmaxf(most, s_ref[u][r]);
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int u = 0; u < kWaves; ++u) {
        if (s_ref[u][r] == kNone) continue;
        const float f = half_factor(s_ref[u][r] - most);
        const float4 y = *reinterpret_cast<const float4 *>(s_merge + (u * 16 * NT + r) * kStride + c);
        l += f * s_sum[u][r] * f;
        v.x += f * y.x * f, v.y += f * y.y * f, v.z += f * y.z * f, v.w += f * y.w * f;
      }
      if (part) {
        publish4(part + r * D + c, v);
        if (c == 0) publish2(part + kRows * D + 2 * r, most, l);
      } else {
        store_out(a, out_at(r) + c, scaled(v, inverse(r, most, l)));
      }
    }
  } else {
    for (int t = 0; t < NT; ++t) {
      const int r = row0 + 16 * t + n - wg_row0;
      if (r >= rows_here) continue;
      const float f = part ? 1.f : inverse(r, ref[t], sum[t]);
      for (int x = 0; x < kTiles; ++x) {
        if (part) publish4(part + r * D + chunk_coord(x), chunk(t, x));
        else store_out(a, out_at(r) + chunk_coord(x), scaled(chunk(t, x), f));
      }
      if (part && j == 0) publish2(part + kRows * D + 2 * r, ref[t], sum[t]);
    }
  }
  if (part) merge_splits<D, NT, W, TILED>(a, g, lds, n);
}

}  // namespace q4
}  // namespace novakv
