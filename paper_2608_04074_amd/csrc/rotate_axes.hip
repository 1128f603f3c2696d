// The norm and rotation of heads at positions of several axes (nova_kv_rotate_qkv_axes,
// nova_kv_q4_append_axes): rotate_kernel.h, whose other instantiations are in rotate.hip.
#include "rotate_kernel.h"

namespace novakv {

hipError_t launch_rotate_axes(const RotateArgs &a, hipStream_t stream) { return launch_rows<true>(a, stream); }

}  // namespace novakv
