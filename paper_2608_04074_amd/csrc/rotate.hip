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
// rotated in 556 us, 3.22 GB read and written at 5.8 TB/s; to a cache (3.37 GB) 702 us, where
// the vector instructions of the codes take about 580 us beside it. One token: 3.8 to 4.7 us,
// 64 sequences' to a cache 5.0 us, launch and latency.
#include "rotate_kernel.h"

namespace novakv {

hipError_t launch_rotate(const RotateArgs &a, hipStream_t stream) {
  return a.num_axes ? launch_rotate_axes(a, stream) : launch_rows<false>(a, stream);
}

}  // namespace novakv
