"""Norm, rotation and the 4-bit cache in fp64, written from their formulas (see
nova_kv_rotary, nova_kv_q4_cache and nova_kv_q4_attn in include/nova_kv.h)."""

from __future__ import annotations

import numpy as np

__all__ = ["norm_rotate", "to_bf16_bits", "from_bf16_bits", "quantize_rows", "pack_codes", "unpack_codes", "attend"]


def norm_rotate(x, weight=None, eps=0.0, cos_sin=None, interleaved=False, pos=None):
    """Heads x [..., H, D]: RMS norm with weight ([D] or [H][D]), then the rotation of the
    first rotary_dim coordinates by row pos [...] of cos_sin [P][rotary_dim]."""
    x = np.asarray(x, dtype=np.float64)
    if weight is not None:
        x = x * np.asarray(weight, dtype=np.float64) / np.sqrt((x * x).mean(-1, keepdims=True) + np.float64(np.float32(eps)))
    if cos_sin is None:
        return x
    r = cos_sin.shape[1]
    row = np.asarray(cos_sin, dtype=np.float64)[pos][..., None, :]
    c, s = row[..., : r // 2], row[..., r // 2:]
    ia, ib = (np.arange(0, r, 2), np.arange(1, r, 2)) if interleaved else (np.arange(r // 2), np.arange(r // 2, r))
    y = x.copy()
    y[..., ia] = x[..., ia] * c - x[..., ib] * s
    y[..., ib] = x[..., ib] * c + x[..., ia] * s
    return y


def to_bf16_bits(x):
    """fp64 -> fp32 -> bf16 bit patterns, each to nearest even; NaN becomes 0x7fc0."""
    x = np.asarray(x, dtype=np.float64).astype(np.float32)
    u = x.view(np.uint32).astype(np.uint64)
    h = ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)
    return np.where(np.isnan(x), np.uint16(0x7FC0), h)


def from_bf16_bits(h):
    return (np.asarray(h).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def quantize_rows(x):
    """Rows [..., D] -> codes uint8 [..., D] (0..15), sq uint16 [..., 2] (scale, offset), and the
    distance of each quotient from its nearest border (0: a tie)."""
    x = np.asarray(x, dtype=np.float64)
    with np.errstate(all="ignore"):
        lo, hi = x.min(-1), x.max(-1)
        sq = np.stack([to_bf16_bits((hi - lo) / 15), to_bf16_bits(lo)], -1)
        scale, offset = from_bf16_bits(sq[..., 0]), from_bf16_bits(sq[..., 1])
        bad = ~(np.isfinite(x).all(-1) & np.isfinite(scale) & np.isfinite(offset))
        t = np.where((scale == 0)[..., None], 0.0, (x - offset[..., None]) / scale[..., None])
        codes = np.clip(np.rint(t), 0, 15)
        codes = np.where(bad[..., None], 0, codes).astype(np.uint8)
    sq[bad] = 0x7FC0
    t = np.where(bad[..., None], 0.0, t)
    gap = np.where((t > -0.5) & (t < 15.5), np.abs(np.abs(t - np.floor(t)) - 0.5), 1.0)
    return codes, sq, gap


def pack_codes(codes):
    return codes[..., ::2] | (codes[..., 1::2] << 4)


def unpack_codes(packed):
    return np.stack([packed & 15, packed >> 4], -1).reshape(*packed.shape[:-1], 2 * packed.shape[-1])


def attend(q, kc, ksq, vc, vsq, pos, window=0, sinks=None, scale=None):
    """One KV head of one sequence: q [m][G][D] at positions pos [m] over codes kc, vc [S][D]
    and (scale, offset) values ksq, vsq [S][2] -> (out [m][G][D], and what a bound of the error is
    made of: sum_j p_j s_j c_j; the largest sum of a logit's magnitudes; max |q_i| times the
    largest norm of a key times the scale; the norm of q, and |sum q|, times the largest
    magnitude of a key's parts and the scale; the largest magnitude of a value's parts)."""
    q = np.asarray(q, dtype=np.float64)
    m, G, D = q.shape
    S = kc.shape[0]
    scale = 1 / np.sqrt(D) if scale is None else scale
    j = np.arange(S)
    seen = (j <= pos[:, None]) & ((window == 0) | (j > pos[:, None] - window))
    out, coded = np.zeros_like(q), np.zeros_like(q)
    mags, norms, key_mags, key_sums = (np.zeros((m, G)) for _ in range(4))
    vmax = np.zeros(m)
    for i in range(m):
        at = np.flatnonzero(seen[i])
        if at.size == 0:
            continue
        c, (ks, ko) = kc[at].astype(np.float64), ksq[at].T
        z = (q[i] @ (ko[:, None] + ks[:, None] * c).T) * scale                     # [G][n]
        mags[i] = (np.abs(q[i]) @ (np.abs(ko)[:, None] + ks[:, None] * c).T).max(1) * scale
        norms[i] = np.abs(q[i]).max(-1) * np.linalg.norm(ko[:, None] + ks[:, None] * c, axis=1).max() * scale
        part = (15 * ks + np.abs(ko)).max() * scale
        key_mags[i], key_sums[i] = part * np.linalg.norm(q[i], axis=-1), part * np.abs(q[i].sum(-1))
        sink = -np.inf * np.ones(G) if sinks is None else np.asarray(sinks, dtype=np.float64)
        top = np.maximum(z.max(1), sink)
        e = np.exp(z - top[:, None])
        p = e / (e.sum(1) + np.exp(sink - top))[:, None]
        sc = vsq[at, 0][:, None] * vc[at].astype(np.float64)
        out[i] = p @ (sc + vsq[at, 1][:, None])
        coded[i] = p @ sc
        vmax[i] = (15 * vsq[at, 0] + np.abs(vsq[at, 1])).max()
    return out, coded, mags, norms, key_mags, key_sums, vmax
