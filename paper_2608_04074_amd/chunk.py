"""Python binding of the attention of several query tokens over the 2-bit cache and of reading
that cache back.

As in api.py, every step runs in the HIP kernels of libnovakv.so; this module checks dtypes,
shapes and devices and hands over raw device pointers and the stream.  The calls run on the
device of their tensors, whichever is current.
"""

from __future__ import annotations

import ctypes
from typing import Optional

import torch

from . import _native as nat
from .api import (Band, CacheLayout, NovaKVParams, PreparedCall, _band_ref, _dtype_code, _require, _scales_ptr,
                  _sq_ptr)
from .q4 import _DTYPES, _dense, _DeviceCall, _first, _fresh, _lens, _one_device, _read_shape, _stream_of

__all__ = ["chunk_attn", "chunk_attn_workspace_bytes", "prepare_chunk_attn", "read", "prepare_read"]


def _param_tensors(params: NovaKVParams):
    return (params.kbar, params.t_k, params.t_k_inv_t, params.t_v, params.cb_k, params.cb_v)


def _check_pool(params: NovaKVParams, layout: CacheLayout, codes: torch.Tensor, name: str, batch: int) -> None:
    """A code pool [num_blocks][Hkv][block_size][L] that holds the sequences' blocks."""
    _require(codes, name, (torch.uint8,))
    if codes.dim() != 4 or tuple(codes.shape[1:]) != (params.num_kv_heads, layout.block_size, params.groups):
        raise ValueError(f"{name} must be [num_blocks][{params.num_kv_heads}][{layout.block_size}][{params.groups}], "
                         f"got {tuple(codes.shape)}")
    table, per_seq = layout.block_table, layout.blocks_per_seq
    have = codes.shape[0] if table is None else table.numel()
    if have < batch * per_seq:
        raise ValueError(f"{batch} sequences of {per_seq} blocks need {batch * per_seq} "
                         f"{'blocks' if table is None else 'block-table entries'}, there are {have}")


def chunk_attn_workspace_bytes(params: NovaKVParams, batch: int, n_q: int, num_q_heads: int, max_seq_len: int) -> int:
    return int(nat.lib().nova_kv_chunk_attn_workspace_bytes(ctypes.byref(params.c), batch, n_q, num_q_heads, max_seq_len))


def _chunk_call(params, layout, q, k_codes, v_codes, seq_lens, max_seq_len, out, workspace, q_lens, window, sinks,
                softmax_scale, k_scales, band, v_sq, stream):
    if not isinstance(q, torch.Tensor) or q.dim() != 4 or q.shape[3] != params.head_dim:
        raise ValueError(f"q must be [B][n_q][Hq][{params.head_dim}]")
    b, n, hq, d = q.shape
    _require(q, "q", _DTYPES)
    _require(seq_lens, "seq_lens", (torch.int32,), b)
    if sinks is not None:
        _require(sinks, "sinks", (torch.float32,), hq)
    if workspace is not None:
        _require(workspace, "workspace", (torch.uint8,))
    _check_pool(params, layout, k_codes, "k_codes", b)
    _check_pool(params, layout, v_codes, "v_codes", b)
    if v_codes.shape != k_codes.shape:
        raise ValueError("code pools must be alike")
    tensors = (q, seq_lens, out, workspace, q_lens, sinks, k_codes, v_codes, k_scales, v_sq, layout.block_table) + \
        (() if band is None else (band.k, band.v)) + _param_tensors(params)
    device = _one_device(tensors)
    vp = ctypes.c_void_p
    args = (ctypes.byref(params.c), ctypes.byref(layout.c), vp(q.data_ptr()), ctypes.c_int(_dtype_code(q)),
            ctypes.c_int32(b), ctypes.c_int32(n), ctypes.c_int32(hq), vp(_lens(q_lens, "q_lens", b)),
            vp(k_codes.data_ptr()), vp(v_codes.data_ptr()), vp(_scales_ptr(params, k_scales, k_codes)),
            vp(_sq_ptr(params, v_sq, k_codes)), _band_ref(band, params, b), vp(seq_lens.data_ptr()),
            ctypes.c_int32(max_seq_len), ctypes.c_int32(window), vp(None if sinks is None else sinks.data_ptr()),
            ctypes.c_float(softmax_scale), vp(_dense(out, "out", (b, n, hq, d), q.dtype)),
            vp(None if workspace is None else workspace.data_ptr()),
            ctypes.c_size_t(0 if workspace is None else workspace.numel()), vp(_stream_of(stream, device)))
    return _DeviceCall(nat.lib().nova_kv_chunk_attn, args, (params, layout, band, tensors), device)


def chunk_attn(params: NovaKVParams, layout: CacheLayout, q: torch.Tensor, k_codes: torch.Tensor, v_codes: torch.Tensor,
               seq_lens: torch.Tensor, max_seq_len: int, q_lens: Optional[torch.Tensor] = None, window: int = 0,
               sinks: Optional[torch.Tensor] = None, softmax_scale: float = 0.0, out: Optional[torch.Tensor] = None,
               workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None,
               k_scales: Optional[torch.Tensor] = None, band: Optional[Band] = None,
               v_sq: Optional[torch.Tensor] = None) -> torch.Tensor:
    """nova_kv_chunk_attn: q [B][n_q][Hq][D] (fp32 or bf16) over the 2-bit cache -> out [B][n_q][Hq][D] in
    q's dtype; query i of sequence b sits at position seq_lens[b] - q_lens[b] + i (q_lens None: n_q) and
    attends what is at or before it.

    Rows i >= q_lens[b] are padding: they stay as they were (zeros in an output that the call makes
    itself).  A caller-provided workspace must be zero-filled before its first use; each call leaves it
    ready for the next.  When omitted, a zeroed one is allocated."""
    if out is None:
        out = _fresh(q, q_lens is None, stream)
    if workspace is None and q.dim() == 4:
        need = chunk_attn_workspace_bytes(params, q.shape[0], q.shape[1], q.shape[2], max_seq_len)
        if need:
            with torch.cuda.stream(stream):
                workspace = torch.zeros(need, dtype=torch.uint8, device=q.device)
    _chunk_call(params, layout, q, k_codes, v_codes, seq_lens, max_seq_len, out, workspace, q_lens, window, sinks,
                softmax_scale, k_scales, band, v_sq, stream)()
    return out


def prepare_chunk_attn(params: NovaKVParams, layout: CacheLayout, q, k_codes, v_codes, seq_lens, max_seq_len: int, out,
                       workspace, q_lens=None, window: int = 0, sinks=None, softmax_scale: float = 0.0, k_scales=None,
                       band: Optional[Band] = None, v_sq=None,
                       stream: Optional[torch.cuda.Stream] = None) -> PreparedCall:
    """nova_kv_chunk_attn with the arguments of chunk_attn(), marshalled once (out and, where
    chunk_attn_workspace_bytes is not 0, a zero-filled workspace are required)."""
    return _chunk_call(params, layout, q, k_codes, v_codes, seq_lens, max_seq_len, out, workspace, q_lens, window, sinks,
                       softmax_scale, k_scales, band, v_sq, stream)


def _read_call(params, layout, k_codes, v_codes, start_pos, k_out, v_out, lens, seq_lens, k_scales, band, v_sq, stream):
    b, n, x = _read_shape(k_out, v_out, params.num_kv_heads, params.head_dim)
    outs = [_dense(t, name, tuple(x.shape), x.dtype) for t, name in ((k_out, "k_out"), (v_out, "v_out"))]
    for codes, name, to in ((k_codes, "k_codes", k_out), (v_codes, "v_codes", v_out)):
        if to is not None:
            _check_pool(params, layout, codes, name, b)
    tensors = (start_pos, k_out, v_out, lens, seq_lens, k_codes, v_codes, k_scales, v_sq, layout.block_table) + \
        (() if band is None else (band.k, band.v)) + _param_tensors(params)
    device = _one_device(tensors)
    vp = ctypes.c_void_p
    ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    args = (ctypes.byref(params.c), ctypes.byref(layout.c), vp(ptr(k_codes)), vp(ptr(v_codes)),
            vp(None if k_out is None else _scales_ptr(params, k_scales, k_codes)),
            vp(None if v_out is None else _sq_ptr(params, v_sq, v_codes)), _band_ref(band, params, b),
            vp(_lens(seq_lens, "seq_lens", b)), ctypes.c_int(_dtype_code(x)), ctypes.c_int32(b), ctypes.c_int32(n),
            vp(_lens(start_pos, "start_pos", b)), vp(_lens(lens, "lens", b)), *map(vp, outs),
            vp(_stream_of(stream, device)))
    return _DeviceCall(nat.lib().nova_kv_read, args, (params, layout, band, tensors), device)


def read(params: NovaKVParams, layout: CacheLayout, k_codes: Optional[torch.Tensor], v_codes: Optional[torch.Tensor],
         start_pos: torch.Tensor, n: int, lens: Optional[torch.Tensor] = None, seq_lens: Optional[torch.Tensor] = None,
         dtype: torch.dtype = torch.bfloat16, k_out: Optional[torch.Tensor] = None, v_out: Optional[torch.Tensor] = None,
         k_scales: Optional[torch.Tensor] = None, band: Optional[Band] = None, v_sq: Optional[torch.Tensor] = None,
         stream: Optional[torch.cuda.Stream] = None):
    """nova_kv_read: the tokens start_pos[b] + i, i < n, of the 2-bit cache as dense rows (k, v)
    [B][n][Hkv][D] of `dtype` (of k_out and v_out, when given), in the domain of the keys and values
    that were appended.

    Rows i >= lens[b] and of positions outside [0, seq_lens[b]) (seq_lens None: the capacity; a band
    needs them) stay as they were: zeros in outputs that the call makes itself."""
    if k_out is None and v_out is None:
        shape = (start_pos.numel(), n, params.num_kv_heads, params.head_dim)
        with torch.cuda.stream(stream):
            k_out, v_out = (torch.zeros(shape, dtype=dtype, device=start_pos.device) for _ in range(2))
    elif _first(k_out, v_out).shape[1] != n:
        raise ValueError(f"outputs of {_first(k_out, v_out).shape[1]} tokens, {n} are read")
    _read_call(params, layout, k_codes, v_codes, start_pos, k_out, v_out, lens, seq_lens, k_scales, band, v_sq, stream)()
    return k_out, v_out


def prepare_read(params: NovaKVParams, layout: CacheLayout, k_codes, v_codes, start_pos, k_out, v_out, lens=None,
                 seq_lens=None, k_scales=None, band: Optional[Band] = None, v_sq=None,
                 stream: Optional[torch.cuda.Stream] = None) -> PreparedCall:
    """nova_kv_read to k_out and v_out [B][n][Hkv][D] (either may be None), marshalled once."""
    return _read_call(params, layout, k_codes, v_codes, start_pos, k_out, v_out, lens, seq_lens, k_scales, band, v_sq,
                      stream)
