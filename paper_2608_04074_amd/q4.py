"""Python binding of the norm and rotation of heads and of the cache held in 4 bits.

As in api.py, every step runs in the HIP kernels of libnovakv.so; this module
checks dtypes, shapes and devices and hands over raw device pointers and the
stream.  The calls run on the device of their tensors, whichever is current.
"""

from __future__ import annotations

import ctypes
from typing import Optional

import torch

from . import _native as nat
from .api import CacheLayout, PreparedCall, _dtype_code, _require

__all__ = ["Rotary", "Q4Cache", "q4_code_shape", "q4_sq_shape", "rotate_qkv", "q4_append", "q4_attn",
           "q4_attn_workspace_bytes", "prepare_rotate_qkv", "prepare_q4_append", "prepare_q4_attn"]

_DTYPES = (torch.float32, torch.bfloat16)
_SQ_DTYPES = (torch.bfloat16, torch.int16, torch.uint16)


def _one_device(tensors) -> torch.device:
    """The device that all given tensors (None: absent) live on."""
    devices = {t.device for t in tensors if t is not None}
    if len(devices) != 1:
        raise ValueError(f"tensors on several devices: {sorted(map(str, devices))}")
    return devices.pop()


def _stream_of(stream: Optional[torch.cuda.Stream], device: torch.device) -> int:
    s = stream if stream is not None else torch.cuda.current_stream(device)
    if s.device != device:
        raise ValueError(f"a stream of {s.device} for tensors on {device}")
    return int(s.cuda_stream)


class _DeviceCall(PreparedCall):
    """A PreparedCall that runs with its tensors' device current."""

    def __init__(self, fn, args, keep, device):
        super().__init__(fn, args, keep)
        self._device = device.index

    def __call__(self) -> None:
        if torch.cuda.current_device() == self._device:
            nat.check(self._fn(*self._args))
        else:
            with torch.cuda.device(self._device):
                nat.check(self._fn(*self._args))


class Rotary:
    """A layer's norms and rotation of its heads (see nova_kv_rotary).

    ``cos_sin`` is a device fp32 tensor [num_positions][rotary_dim] (the cosines
    of a position's rotary_dim / 2 angles, then their sines; ``Rotary.table``
    makes the usual one), or None for no rotation.  Pairs are (j, j + rotary_dim/2),
    or (2j, 2j + 1) when ``interleaved``.  ``q_norm`` and ``k_norm`` are fp32 weights
    [D] or, with weights of each head, [H][D]; None for no norm.
    """

    def __init__(self, num_q_heads: int, num_kv_heads: int, head_dim: int, cos_sin: Optional[torch.Tensor] = None,
                 interleaved: bool = False, q_norm: Optional[torch.Tensor] = None,
                 k_norm: Optional[torch.Tensor] = None, eps: float = 1e-6):
        if cos_sin is not None:
            _require(cos_sin, "cos_sin", (torch.float32,))
            if cos_sin.dim() != 2:
                raise ValueError("cos_sin must be [num_positions][rotary_dim]")
        for name, w, heads in (("q_norm", q_norm, num_q_heads), ("k_norm", k_norm, num_kv_heads)):
            if w is None:
                continue
            _require(w, name, (torch.float32,))
            if tuple(w.shape) not in ((head_dim,), (heads, head_dim)):
                raise ValueError(f"{name} must be [{head_dim}] or [{heads}][{head_dim}]")
        self.num_q_heads, self.num_kv_heads, self.head_dim = num_q_heads, num_kv_heads, head_dim
        self.cos_sin, self.interleaved, self.q_norm, self.k_norm, self.eps = cos_sin, bool(interleaved), q_norm, k_norm, eps
        ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
        per_head = lambda t: int(t is not None and t.dim() == 2)  # noqa: E731
        self._c = nat.Rotary(num_q_heads, num_kv_heads, head_dim, 0 if cos_sin is None else cos_sin.shape[1],
                             int(self.interleaved), 0 if cos_sin is None else cos_sin.shape[0], ptr(cos_sin),
                             ptr(q_norm), ptr(k_norm), per_head(q_norm), per_head(k_norm), eps)

    @staticmethod
    def table(num_positions: int, rotary_dim: int, theta: float = 10000.0, device="cuda") -> torch.Tensor:
        """cos_sin of the angles p * theta^(-2j / rotary_dim), evaluated in fp64."""
        j = torch.arange(0, rotary_dim, 2, dtype=torch.float64)
        angle = torch.arange(num_positions, dtype=torch.float64)[:, None] * theta ** (-j / rotary_dim)
        return torch.cat([angle.cos(), angle.sin()], 1).float().to(device)

    @property
    def c(self) -> nat.Rotary:
        return self._c

    @property
    def tensors(self):
        return (self.cos_sin, self.q_norm, self.k_norm)


def q4_code_shape(num_kv_heads: int, head_dim: int, layout: CacheLayout, batch: int, num_blocks: Optional[int] = None):
    """Shape of one code pool of a 4-bit cache: [num_blocks][Hkv][block_size][D / 2] (uint8)."""
    nb = batch * layout.blocks_per_seq if num_blocks is None else num_blocks
    return (nb, num_kv_heads, layout.block_size, head_dim // 2)


def q4_sq_shape(num_kv_heads: int, layout: CacheLayout, batch: int, num_blocks: Optional[int] = None):
    """Shape of a 4-bit cache's (scale, offset) pool: [num_blocks][Hkv][block_size][2] (bf16)."""
    return q4_code_shape(num_kv_heads, 0, layout, batch, num_blocks)[:3] + (2,)


class Q4Cache:
    """A cache held in 4 bits (see nova_kv_q4_cache): uint8 code pools
    [num_blocks][Hkv][block_size][D / 2] and bf16 (scale, offset) pools
    [num_blocks][Hkv][block_size][2], addressed through ``layout``."""

    def __init__(self, layout: CacheLayout, k_codes: torch.Tensor, v_codes: torch.Tensor, k_sq: torch.Tensor,
                 v_sq: torch.Tensor):
        for name, t in (("k_codes", k_codes), ("v_codes", v_codes)):
            _require(t, name, (torch.uint8,))
        if k_codes.dim() != 4 or k_codes.shape[2] != layout.block_size or v_codes.shape != k_codes.shape:
            raise ValueError("code pools must be [num_blocks][Hkv][block_size][D / 2], both alike")
        for name, t in (("k_sq", k_sq), ("v_sq", v_sq)):
            _require(t, name, _SQ_DTYPES)
            if tuple(t.shape) != tuple(k_codes.shape[:3]) + (2,):
                raise ValueError(f"{name} must be [num_blocks][Hkv][block_size][2]")
        self.layout, self.k_codes, self.v_codes, self.k_sq, self.v_sq = layout, k_codes, v_codes, k_sq, v_sq
        self.device = _one_device(self.tensors)
        self._c = nat.Q4Cache(self.num_kv_heads, self.head_dim, self.num_blocks, layout.c, k_codes.data_ptr(),
                              v_codes.data_ptr(), k_sq.data_ptr(), v_sq.data_ptr())

    @classmethod
    def zeros(cls, layout: CacheLayout, batch: int, num_kv_heads: int, head_dim: int,
              num_blocks: Optional[int] = None, device="cuda") -> "Q4Cache":
        """An empty cache for `batch` sequences, or of `num_blocks` blocks."""
        codes = q4_code_shape(num_kv_heads, head_dim, layout, batch, num_blocks)
        sq = q4_sq_shape(num_kv_heads, layout, batch, num_blocks)
        make = lambda shape, dt: torch.zeros(shape, dtype=dt, device=device)  # noqa: E731
        return cls(layout, make(codes, torch.uint8), make(codes, torch.uint8), make(sq, torch.bfloat16),
                   make(sq, torch.bfloat16))

    @property
    def tensors(self):
        return (self.layout.block_table, self.k_codes, self.v_codes, self.k_sq, self.v_sq)

    @property
    def num_blocks(self) -> int:
        return self.k_codes.shape[0]

    @property
    def num_kv_heads(self) -> int:
        return self.k_codes.shape[1]

    @property
    def head_dim(self) -> int:
        return 2 * self.k_codes.shape[3]

    @property
    def c(self) -> nat.Q4Cache:
        return self._c

    def check_batch(self, batch: int) -> None:
        """Whether the layout reaches `batch` sequences."""
        table, per_seq = self.layout.block_table, self.layout.blocks_per_seq
        if table is not None and table.numel() < batch * per_seq:
            raise ValueError(f"block_table has {table.numel()} entries, {batch} sequences of {per_seq} blocks need "
                             f"{batch * per_seq}")


def _rows(t: Optional[torch.Tensor], name: str, batch: int, n_new: int, heads: int, head_dim: int, dtype):
    """nova_kv_rows of a tensor [B][n_new][H][D] whose heads are dense; tokens and sequences may be strided."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} has dtype {t.dtype}, expected {dtype}")
    if tuple(t.shape) != (batch, n_new, heads, head_dim):
        raise ValueError(f"{name} must be [{batch}][{n_new}][{heads}][{head_dim}], got {tuple(t.shape)}")
    if t.numel() and (t.stride(3) != 1 or (heads > 1 and t.stride(2) != head_dim)):
        raise ValueError(f"the heads of a token must be contiguous in {name}")
    return nat.Rows(t.data_ptr(), t.stride(0), t.stride(1))


def _lens(t: Optional[torch.Tensor], name: str, batch: int):
    if t is None:
        return None
    _require(t, name, (torch.int32,), batch)
    return t.data_ptr()


def _dense(t: Optional[torch.Tensor], name: str, shape, dtype):
    if t is None:
        return None
    _require(t, name, (dtype,))
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")
    return t.data_ptr()


def _ref(c):
    return None if c is None else ctypes.byref(c)


def _first(*tensors):
    for t in tensors:
        if t is not None:
            if not isinstance(t, torch.Tensor) or t.dim() != 4:
                raise ValueError("q, k and v must be tensors [B][n_new][heads][D]")
            return t
    raise ValueError("none of q, k and v is given")


def _rotate_call(rotary, q, k, v, start_pos, q_out, k_out, v_out, new_lens, stream):
    x = _first(q, k, v)
    b, n, d, dt = x.shape[0], x.shape[1], rotary.head_dim, x.dtype
    hq, hkv = rotary.num_q_heads, rotary.num_kv_heads
    rows = [_rows(t, name, b, n, h, d, dt) for t, name, h in ((q, "q", hq), (k, "k", hkv), (v, "v", hkv))]
    outs = [_dense(t, name, (b, n, h, d), dt) for t, name, h in ((q_out, "q_out", hq), (k_out, "k_out", hkv), (v_out, "v_out", hkv))]
    tensors = (q, k, v, start_pos, q_out, k_out, v_out, new_lens) + rotary.tensors
    device = _one_device(tensors)
    vp = ctypes.c_void_p
    args = (ctypes.byref(rotary.c), *map(_ref, rows), ctypes.c_int(_dtype_code(x)), ctypes.c_int32(b),
            ctypes.c_int32(n), vp(_lens(new_lens, "new_lens", b)), vp(_lens(start_pos, "start_pos", b)),
            *map(vp, outs), vp(_stream_of(stream, device)))
    return _DeviceCall(nat.lib().nova_kv_rotate_qkv, args, (rotary, tensors, rows), device)


def _fresh(t, whole, stream):
    """An output for rows like t: zeros, but where the call writes the whole of it."""
    make = torch.empty if whole else torch.zeros
    with torch.cuda.stream(stream):
        return make(t.shape, dtype=t.dtype, device=t.device)


def rotate_qkv(rotary: Rotary, q: Optional[torch.Tensor], k: Optional[torch.Tensor], v: Optional[torch.Tensor],
               start_pos: Optional[torch.Tensor], new_lens: Optional[torch.Tensor] = None,
               q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None,
               v_out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
    """nova_kv_rotate_qkv: q [B][n_new][Hq][D], k, v [B][n_new][Hkv][D] (fp32 or bf16;
    heads contiguous, tokens and sequences strided as they come, any of the three
    may be None) -> dense (q, k, v) for encode, decode_attn and the step, queries
    and keys normed and rotated at the positions start_pos[b] + i.

    Tokens i >= new_lens[b] and, with a rotation, those at positions outside the table
    are left out: their output rows stay as they were (zeros in outputs that
    the call makes itself)."""
    whole = new_lens is None and rotary.cos_sin is None
    q_out, k_out, v_out = (o if o is not None or t is None else _fresh(t, whole, stream)
                           for t, o in ((q, q_out), (k, k_out), (v, v_out)))
    _rotate_call(rotary, q, k, v, start_pos, q_out, k_out, v_out, new_lens, stream)()
    return q_out, k_out, v_out


def prepare_rotate_qkv(rotary: Rotary, q, k, v, start_pos, q_out, k_out, v_out, new_lens=None,
                       stream: Optional[torch.cuda.Stream] = None) -> PreparedCall:
    """nova_kv_rotate_qkv with the arguments of rotate_qkv(), marshalled once."""
    return _rotate_call(rotary, q, k, v, start_pos, q_out, k_out, v_out, new_lens, stream)


def _append_call(rotary, cache, q, k, v, start_pos, q_out, new_lens, k_held, v_held, stream):
    x = _first(k)
    b, n, d, dt = x.shape[0], x.shape[1], rotary.head_dim, x.dtype
    hq, hkv = rotary.num_q_heads, rotary.num_kv_heads
    rows = [_rows(t, name, b, n, h, d, dt) for t, name, h in ((q, "q", hq), (k, "k", hkv), (v, "v", hkv))]
    outs = [_dense(t, name, (b, n, h, d), dt) for t, name, h in ((q_out, "q_out", hq), (k_held, "k_held", hkv), (v_held, "v_held", hkv))]
    cache.check_batch(b)
    tensors = (q, k, v, start_pos, q_out, k_held, v_held, new_lens) + rotary.tensors + cache.tensors
    device = _one_device(tensors)
    vp = ctypes.c_void_p
    args = (ctypes.byref(rotary.c), ctypes.byref(cache.c), *map(_ref, rows), ctypes.c_int(_dtype_code(x)),
            ctypes.c_int32(b), ctypes.c_int32(n), vp(_lens(new_lens, "new_lens", b)),
            vp(_lens(start_pos, "start_pos", b)), *map(vp, outs), vp(_stream_of(stream, device)))
    return _DeviceCall(nat.lib().nova_kv_q4_append, args, (rotary, cache, tensors, rows), device)


def q4_append(rotary: Rotary, cache: Q4Cache, q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor,
              start_pos: torch.Tensor, new_lens: Optional[torch.Tensor] = None,
              q_out: Optional[torch.Tensor] = None, k_held: Optional[torch.Tensor] = None,
              v_held: Optional[torch.Tensor] = None,
              stream: Optional[torch.cuda.Stream] = None) -> Optional[torch.Tensor]:
    """nova_kv_q4_append: k, v [B][n_new][Hkv][D] (as in rotate_qkv) to the positions
    start_pos[b] + i of the 4-bit cache, keys normed and rotated -> the queries q
    [B][n_new][Hq][D] normed and rotated, dense (None without q).  Rows of tokens that
    are left out (padding, positions outside the table or the cache, blocks that
    hold nothing) stay as they were: zeros in an output that the call makes itself.

    k_held and v_held, when given, receive the values that the cache now stands
    for, as dense tensors [B][n_new][Hkv][D]."""
    if q is not None and q_out is None:
        q_out = _fresh(q, False, stream)
    _append_call(rotary, cache, q, k, v, start_pos, q_out, new_lens, k_held, v_held, stream)()
    return q_out


def prepare_q4_append(rotary: Rotary, cache: Q4Cache, q, k, v, start_pos, q_out, new_lens=None, k_held=None,
                      v_held=None, stream: Optional[torch.cuda.Stream] = None) -> PreparedCall:
    """nova_kv_q4_append with the arguments of q4_append(), marshalled once."""
    return _append_call(rotary, cache, q, k, v, start_pos, q_out, new_lens, k_held, v_held, stream)


def q4_attn_workspace_bytes(cache: Q4Cache, batch: int, n_q: int, num_q_heads: int, max_seq_len: int) -> int:
    return int(nat.lib().nova_kv_q4_attn_workspace_bytes(ctypes.byref(cache.c), batch, n_q, num_q_heads, max_seq_len))


def _attn_call(cache, q, seq_lens, max_seq_len, out, workspace, q_lens, window, sinks, softmax_scale, stream):
    if not isinstance(q, torch.Tensor) or q.dim() != 4 or q.shape[3] != cache.head_dim:
        raise ValueError(f"q must be [B][n_q][Hq][{cache.head_dim}]")
    b, n, hq, d = q.shape
    _require(q, "q", _DTYPES)
    _require(seq_lens, "seq_lens", (torch.int32,), b)
    if sinks is not None:
        _require(sinks, "sinks", (torch.float32,), hq)
    if workspace is not None:
        _require(workspace, "workspace", (torch.uint8,))
    cache.check_batch(b)
    tensors = (q, seq_lens, out, workspace, q_lens, sinks) + cache.tensors
    device = _one_device(tensors)
    vp = ctypes.c_void_p
    args = (ctypes.byref(cache.c), vp(q.data_ptr()), ctypes.c_int(_dtype_code(q)), ctypes.c_int32(b),
            ctypes.c_int32(n), ctypes.c_int32(hq), vp(_lens(q_lens, "q_lens", b)), vp(seq_lens.data_ptr()),
            ctypes.c_int32(max_seq_len), ctypes.c_int32(window), vp(None if sinks is None else sinks.data_ptr()),
            ctypes.c_float(softmax_scale), vp(_dense(out, "out", (b, n, hq, d), q.dtype)),
            vp(None if workspace is None else workspace.data_ptr()),
            ctypes.c_size_t(0 if workspace is None else workspace.numel()), vp(_stream_of(stream, device)))
    return _DeviceCall(nat.lib().nova_kv_q4_attn, args, (cache, tensors), device)


def q4_attn(cache: Q4Cache, q: torch.Tensor, seq_lens: torch.Tensor, max_seq_len: int,
            q_lens: Optional[torch.Tensor] = None, window: int = 0, sinks: Optional[torch.Tensor] = None,
            softmax_scale: float = 0.0, out: Optional[torch.Tensor] = None,
            workspace: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """nova_kv_q4_attn: q [B][n_q][Hq][D] (fp32 or bf16) over the 4-bit cache -> out
    [B][n_q][Hq][D] in q's dtype; query i of sequence b sits at position
    seq_lens[b] - q_lens[b] + i (q_lens None: n_q) and attends what is at or
    before it.

    Rows i >= q_lens[b] are padding: they stay as they were (zeros in an output
    that the call makes itself).  A caller-provided workspace must be zero-filled
    before its first use; each call leaves it ready for the next.  When omitted,
    a zeroed one is allocated."""
    if out is None:
        out = _fresh(q, q_lens is None, stream)
    if workspace is None and q.dim() == 4:
        need = q4_attn_workspace_bytes(cache, q.shape[0], q.shape[1], q.shape[2], max_seq_len)
        if need:
            with torch.cuda.stream(stream):
                workspace = torch.zeros(need, dtype=torch.uint8, device=q.device)
    _attn_call(cache, q, seq_lens, max_seq_len, out, workspace, q_lens, window, sinks, softmax_scale, stream)()
    return out


def prepare_q4_attn(cache: Q4Cache, q, seq_lens, max_seq_len: int, out, workspace, q_lens=None, window: int = 0,
                    sinks=None, softmax_scale: float = 0.0,
                    stream: Optional[torch.cuda.Stream] = None) -> PreparedCall:
    """nova_kv_q4_attn with the arguments of q4_attn(), marshalled once (out and,
    where q4_attn_workspace_bytes is not 0, a zero-filled workspace are required)."""
    return _attn_call(cache, q, seq_lens, max_seq_len, out, workspace, q_lens, window, sinks, softmax_scale, stream)
