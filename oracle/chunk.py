"""The 2-bit cache read back, and causal attention of several query tokens over it, in fp64 from the
formulas (see nova_kv_read and nova_kv_chunk_attn in include/nova_kv.h)."""

from __future__ import annotations

import numpy as np

__all__ = ["codewords", "levels", "cached_rows", "attend", "axis_angles"]


def codewords(book, codes):
    """Coefficients [S][D] of code rows [S][L] in one head's codebook [L][256][4]."""
    book = np.asarray(book, dtype=np.float64)
    S, L = codes.shape
    return book[np.arange(L), codes.astype(np.int64)].reshape(S, 4 * L)


def levels(codes):
    """The 2-bit levels [S][D] of the scalar arm's code rows [S][L]."""
    return ((codes[..., None] >> np.array([0, 2, 4, 6], dtype=np.uint8)) & 3).reshape(len(codes), 4 * codes.shape[1]).astype(np.float64)


def cached_rows(head, k_codes, v_codes, rho=None, grid=None):
    """One head's keys and values [S][D] in the domain of what was appended, and their coefficients
    r [S][D] and s [S][D].  head: kbar [D], t_k_inv_t, t_v [D][D], cb_k, cb_v [L][256][4]; rho [S] of the
    key-scale format; grid [S][2] (scale, offset) of the scalar value arm."""
    r = codewords(head["cb_k"], k_codes)
    if rho is not None:
        r = r * rho[:, None]
    s = codewords(head["cb_v"], v_codes) if grid is None else grid[:, 1:] + grid[:, :1] * levels(v_codes)
    back = lambda x, t: x @ np.asarray(t, dtype=np.float64).T  # noqa: E731
    return back(r, head["t_k_inv_t"]) + np.asarray(head["kbar"], dtype=np.float64), back(s, head["t_v"]), r, s


def attend(q, k, v, pos, window=0, sinks=None, scale=None):
    """q [m][G][D] at positions pos [m] over keys and values [S][D] -> out [m][G][D]; rows that attend
    nothing are zeros."""
    q = np.asarray(q, dtype=np.float64)
    m, G, D = q.shape
    scale = 1 / np.sqrt(D) if scale is None else scale
    j = np.arange(len(k))
    out = np.zeros_like(q)
    for i in range(m):
        seen = (j <= pos[i]) & ((window == 0) | (j > pos[i] - window))
        if not seen.any():
            continue
        z = (q[i] @ k[seen].T) * scale
        sink = np.full(G, -np.inf) if sinks is None else np.asarray(sinks, dtype=np.float64)
        top = np.maximum(z.max(1), sink)
        e = np.exp(z - top[:, None])
        out[i] = (e @ v[seen]) / (e.sum(1) + np.exp(sink - top))[:, None]
    return out


def axis_angles(cos_sin, pair_axis, positions):
    """The rows [..., rotary_dim] of cosines and sines of tokens at positions [axes][...]: column j (and
    rotary_dim / 2 + j) from the row of pair j's axis."""
    cos_sin = np.asarray(cos_sin)
    half = cos_sin.shape[1] // 2
    cols = [cos_sin[positions[a], j] for j, a in enumerate(pair_axis)]
    cols += [cos_sin[positions[a], half + j] for j, a in enumerate(pair_axis)]
    return np.stack(cols, -1)
