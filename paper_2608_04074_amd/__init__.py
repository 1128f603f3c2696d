"""NOVA-KV hot path for MI355X (gfx950): 2-bit VQ KV-cache encode and decode attention.

Beside it: attention of several query tokens over that cache, and reading it back (chunk.py); norm and
rotation of heads, and a cache held in 4 bits with its attention (q4.py).

The compute lives in ``libnovakv.so`` (hand-written HIP, C ABI in
``include/nova_kv.h``); this package is its Python binding.
"""

from .api import (NOALLOC_SCRATCH_BYTES, Band, CacheLayout, NovaKVParams, append_decode_attn,  # noqa: F401
                  append_decode_attn_noalloc, band_shape, check_metadata, set_debug,
                  code_pool_shape, decode_attn, decode_workspace_bytes, encode, prepare_append_decode,
                  prepare_decode, prepare_encode, scale_pool_shape)
from .chunk import chunk_attn, chunk_attn_workspace_bytes, prepare_chunk_attn, prepare_read, read  # noqa: F401
from .q4 import (Q4Cache, Rotary, RotaryAxes, prepare_q4_append, prepare_q4_append_axes, prepare_q4_attn,  # noqa: F401
                 prepare_q4_read, prepare_rotate_qkv, prepare_rotate_qkv_axes, q4_append, q4_append_axes, q4_attn,
                 q4_attn_workspace_bytes, q4_code_shape, q4_read, q4_sq_shape, rotate_qkv, rotate_qkv_axes)
from ._native import NovaKVError  # noqa: F401
