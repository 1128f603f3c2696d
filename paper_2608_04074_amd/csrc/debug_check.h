// Debug mode's check of a call's metadata (api.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/nova_kv.h"

namespace novakv {

// With debug mode on (nova_kv_set_debug): waits for the stream, copies a call's metadata
// to the host and checks it.  new_lens: tokens that each sequence writes
// (nullptr: n_new); num_blocks > 0: the pool's size, of a cache that knows it (one
// held in 4 bits), where negative block-table entries hold nothing.
nova_kv_status debug_check(const nova_kv_layout *lay, int32_t batch, const int32_t *seq_lens, int32_t max_seq_len,
                           const int32_t *start_pos, int32_t n_new, hipStream_t stream,
                           const int32_t *new_lens = nullptr, int32_t num_blocks = 0);

}  // namespace novakv
