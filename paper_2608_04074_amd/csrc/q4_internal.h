// Internal declarations of the 4-bit cache's calls and of the norm and
// rotation in front of them (rotate.hip, q4_attn.hip, q4_api.hip).
#pragma once

#include "nova_kv_internal.h"

namespace novakv {

// Rows of heads in the caller's memory (nova_kv_rows), data == nullptr: absent.
struct HeadRows {
  const void *data;
  long long batch_stride, token_stride;  // elements
};

struct RotateArgs {
  int batch, n_new, head_dim;
  int nq, nk, nv;  // heads of the sides that are present (0: absent)
  int bf16;        // inputs and dense outputs: bf16, else fp32
  HeadRows q, k, v;
  const int32_t *new_lens, *start_pos;
  const float *cos_sin;  // [num_positions][rotary_dim], or nullptr when rotary_dim == 0
  int rotary_dim, interleaved, num_positions;
  const float *q_norm, *k_norm;  // weights, or nullptr
  int q_norm_stride, k_norm_stride;  // elements from one head's weights to the next one's: 0 or head_dim
  float eps;
  void *q_out, *k_out, *v_out;  // dense [B][n_new][heads][D]; k_out, v_out of an append: the held values, or nullptr
  // append to a 4-bit cache (q4 != 0)
  int q4;
  CacheLayout layout;
  int num_blocks;
  uint8_t *k_codes, *v_codes;
  uint16_t *k_sq, *v_sq;
};
hipError_t launch_rotate(const RotateArgs &a, hipStream_t stream);

struct Q4AttnArgs {
  int batch, n_q, num_q_heads, num_kv_heads, head_dim, gqa;
  CacheLayout layout;
  int num_blocks;
  const uint8_t *k_codes, *v_codes;
  const uint16_t *k_sq, *v_sq;
  const void *q;
  int q_bf16;
  const int32_t *q_lens, *seq_lens;
  int max_seq_len, window;
  const float *sinks;
  float qscale;  // softmax scale * log2(e)
  void *out;
  int n_split, row_tiles;
  float *part;  // split partials [unit][n_split][rows of a tile][D + 2]
  int *counters;
};

// Plan of a nova_kv_q4_attn call: rows (query tokens * query heads per KV
// head) in tiles of tile_rows, each tile's span in n_split splits.
struct Q4AttnPlan {
  int tile_rows, row_tiles, n_split;
  int waves;    // of a workgroup
  double cost;  // estimated time, ns
  size_t off_part, total;  // workspace: arrival counters, then the split partials (needed when n_split > 1)
};
Q4AttnPlan plan_q4_attn(int batch, int n_q, int num_q_heads, int num_kv_heads, int head_dim, int q_bf16,
                        int max_seq_len, int window);
// bf16 queries, tiles of 128 or 256 rows (q4_tile.hip); launch_q4_attn calls it.
hipError_t launch_q4_tile(const Q4AttnArgs &a, const Q4AttnPlan &plan, hipStream_t stream);
hipError_t launch_q4_attn(const Q4AttnArgs &a, const Q4AttnPlan &plan, hipStream_t stream);

}  // namespace novakv
