// Internal declarations of the attention of several query tokens over the 2-bit cache
// and of reading the caches back (chunk_rows.hip, chunk_tile.hip, read.hip, chunk_api.hip).
#pragma once

#include "q4_internal.h"

namespace novakv {

// position / block_size without a division or a branch: with 2^(l - 1) < d <= 2^l, ceil(2^(31 + l) / d) d lies
// less than 2^l above 2^(31 + l), so the products of positions below 2^31 are cut to their quotients.
struct BlockDivisor {
  uint32_t factor;
  int shift;
  __host__ void set(const uint32_t d) {
    shift = 31;
    while ((1ull << (shift - 31)) < d) ++shift;
    factor = static_cast<uint32_t>(((1ull << shift) + d - 1) / d);
  }
  __host__ __device__ __forceinline__ int operator()(const int pos) const {
    return static_cast<int>((static_cast<uint64_t>(static_cast<uint32_t>(pos)) * factor) >> shift);
  }
};

// Tokens of a cache to be read as dense rows. k_out, v_out: [B][n][Hkv][D], nullptr: left out.
struct ReadArgs {
  int batch, n, num_kv_heads, head_dim;
  CacheLayout layout;
  const int32_t *lens, *start_pos, *seq_lens;  // lens, seq_lens: or nullptr
  void *k_out, *v_out;
  int bf16;  // outputs: bf16, else fp32
  const uint8_t *k_codes, *v_codes;
  // 2-bit cache
  const float *kbar;
  const void *t_k_inv_t, *t_v, *cb_k, *cb_v;
  int t_bf16, cb_fp8;
  const uint16_t *k_scales, *v_sq;  // of the formats that have them, else nullptr
  int n_sink, n_rec;
  const uint16_t *band_k, *band_v;
  int chunk;  // tokens of a workgroup
  BlockDivisor block_of;
  // 4-bit cache
  int num_blocks;
  const uint16_t *k_sq;  // and v_sq above
};
hipError_t launch_read(const ReadArgs &a, hipStream_t stream);
hipError_t launch_q4_read(const ReadArgs &a, hipStream_t stream);

// Attention of several query tokens over the 2-bit cache. The rows, their splits and outputs as
// in the attention over a 4-bit cache (k_sq and num_blocks are unused).
struct ChunkArgs : Q4AttnArgs {
  const float *kbar;
  const void *t_k_inv_t, *t_v, *cb_k, *cb_v;
  int t_bf16, cb_fp8;
  const uint16_t *k_scales;  // key-scale format, else nullptr (v_sq: the scalar value arm, else nullptr)
  int n_sink, n_rec;
  const uint16_t *band_k, *band_v;
  BlockDivisor block_of;
};

// Plan of a nova_kv_chunk_attn call: rows (query tokens * query heads per KV head) in tiles
// of tile_rows, each tile's span in n_split splits.
struct ChunkPlan {
  int tile_rows, row_tiles, n_split;
  size_t off_part, total;  // workspace: arrival counters, then the split partials (needed when n_split > 1)
};
ChunkPlan plan_chunk(int batch, int n_q, int num_q_heads, int num_kv_heads, int head_dim, int max_seq_len, int window);
hipError_t launch_chunk_tile(const ChunkArgs &a, const ChunkPlan &plan, hipStream_t stream);  // tiles of 128 rows; launch_chunk calls it
hipError_t launch_chunk_wide(const ChunkArgs &a, const ChunkPlan &plan, hipStream_t stream);  // of 256
hipError_t launch_chunk(const ChunkArgs &a, const ChunkPlan &plan, hipStream_t stream);

}  // namespace novakv
