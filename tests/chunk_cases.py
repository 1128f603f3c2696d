"""Layers and filled 2-bit caches for the tests of the calls that read them (numpy and torch, seeded)."""

import numpy as np
import torch

from oracle import chunk
from oracle.q4 import from_bf16_bits, to_bf16_bits

FORMATS = {
    "plain": {},
    "key_scale": {"key_scale": True},
    "fp8": {"fp8": True},
    "sq": {"sq": True},
    "bf16t": {"bf16t": True},
    "band": {"band": (5, 40)},
    "deployed": {"key_scale": True, "sq": True, "fp8": True, "bf16t": True, "band": (16, 70)},
    "scaled": {"key_scale": True, "sq": True},
}


def bf16(x):
    return from_bf16_bits(to_bf16_bits(x))


class Cache:
    """A layer's parameters and a cache of sequences `seqs` on the GPU, and what they stand for in fp64.

    Rows that hold no token have random codes, NaN scales and grids and NaN band rows, block-table
    entries of blocks that no token is in point far outside the pool, so a call that reads what it
    must not shows it."""

    def __init__(self, nk, seed, seqs, H, D, block, fmt="plain", k_size=1.0, v_size=1.0, kbar_size=0.3, extra_blocks=3):
        f = FORMATS[fmt]
        rng = np.random.default_rng(seed)
        B, L, top = len(seqs), D // 4, max(max(seqs), 1)
        self.nk, self.seqs, self.H, self.D, self.fmt, self.rng = nk, seqs, H, D, f, rng
        q, qv = (np.linalg.qr(rng.standard_normal((H, D, D)))[0] for _ in range(2))
        lam = np.arange(1, D + 1) ** -0.6
        sigma = np.sqrt(lam * (D / lam.sum()))
        even = sigma ** -0.25
        tdt = torch.bfloat16 if f.get("bf16t") else torch.float32
        dev = lambda x, dt: torch.as_tensor(np.ascontiguousarray(x)).float().to(dt).cuda()  # noqa: E731
        t = {"kbar": dev(kbar_size * rng.standard_normal((H, D)), torch.float32), "t_k": dev(q * even, tdt),
             "t_k_inv_t": dev(q / even, tdt), "t_v": dev(qv, tdt)}
        for name, size, std in (("cb_k", k_size, sigma * even), ("cb_v", v_size, sigma)):
            book = torch.as_tensor(0.92 * size * rng.standard_normal((H, L, 256, 4)) * std.reshape(1, L, 1, 4)).float()
            t[name] = (book.to(torch.float8_e4m3fn).view(torch.uint8) if f.get("fp8") else book.half()).cuda()
        book64 = lambda x: (x.cpu().view(torch.float8_e4m3fn) if x.dtype == torch.uint8 else x.cpu()).double().numpy()  # noqa: E731
        self.arrays = {n: book64(x) if n.startswith("cb") else x.double().cpu().numpy() for n, x in t.items()}
        self.params = nk.NovaKVParams(t["kbar"], t["t_k"], t["t_k_inv_t"], t["t_v"], t["cb_k"],
                                      None if f.get("sq") else t["cb_v"], key_scale=f.get("key_scale", False),
                                      sq_values=f.get("sq", False))
        if block:
            bps = -(-top // block) + 1
            nblk = B * bps + extra_blocks
            order = rng.permutation(nblk)[:B * bps].astype(np.int32).reshape(B, bps)
            table = order.copy()
            for b, S in enumerate(seqs):
                table[b, -(-S // block):] = 2 ** 30 + 7
            rows = block
        else:
            bps, rows, nblk, order, table = 1, top + 5, B, None, None
        self.block, self.order = block, order
        kc, vc = (rng.integers(0, 256, (nblk, H, rows, L)).astype(np.uint8) for _ in range(2))
        ks = np.full((nblk, H, rows), 0x7FC0, dtype=np.uint16)
        vs = np.full((nblk, H, rows, 2), 0x7FC0, dtype=np.uint16)
        self.where = []
        for b, S in enumerate(seqs):
            at = np.arange(S)
            phys = order[b][at // rows] if order is not None else np.full(S, b)
            self.where.append((phys, at % rows))
            ks[phys, :, at % rows] = to_bf16_bits(np.exp(0.25 * rng.standard_normal((S, H))))
            step = v_size * (1.2 + 0.4 * rng.random((S, H)))
            vs[phys, :, at % rows] = to_bf16_bits(np.stack([step, -1.5 * step + 0.1 * v_size * rng.standard_normal((S, H))], -1))
        self.kc, self.vc, self.ks, self.vs = kc, vc, ks, vs
        self.band = self.bk = self.bv = None
        if f.get("band"):
            n_sink, n_rec = f["band"]
            self.bk, self.bv = np.full((2, B, H, n_sink + n_rec, D), np.nan)
            for b, S in enumerate(seqs):
                for p in range(S):
                    if p < n_sink or p >= S - n_rec:
                        slot = p if p < n_sink else n_sink + p % n_rec
                        self.bk[b, :, slot] = bf16(k_size * rng.standard_normal((H, D)) + self.arrays["kbar"])
                        self.bv[b, :, slot] = bf16(v_size * rng.standard_normal((H, D)))
            self.band = nk.Band(n_sink, n_rec, *(torch.as_tensor(x).to(torch.bfloat16).cuda() for x in (self.bk, self.bv)))
        bits = lambda x: torch.as_tensor(x.view(np.int16)).cuda().view(torch.bfloat16)  # noqa: E731
        self.layout = nk.CacheLayout(rows, bps, None if table is None else torch.as_tensor(table).cuda())
        self.k_codes, self.v_codes = torch.as_tensor(kc).cuda(), torch.as_tensor(vc).cuda()
        self.k_scales = bits(ks) if f.get("key_scale") else None
        self.v_sq = bits(vs) if f.get("sq") else None
        self.seq_lens = torch.tensor(seqs, dtype=torch.int32, device="cuda")
        self.top = top

    @property
    def more(self):
        return {"k_scales": self.k_scales, "v_sq": self.v_sq, "band": self.band}

    def banded(self, b):
        """Whether each of sequence b's tokens is the band's."""
        S, at = self.seqs[b], np.arange(self.seqs[b])
        return np.zeros(S, dtype=bool) if self.band is None else (at < self.band.n_sink) | (at >= S - self.band.n_rec)

    def rows(self, b, h):
        """Keys, values [S][D] of one head of a sequence, their coefficients r, s, and the scalar arm's grid."""
        phys, row = self.where[b]
        head = {n: x[h] for n, x in self.arrays.items()}
        rho = from_bf16_bits(self.ks[phys, h, row]) if self.k_scales is not None else None
        grid = from_bf16_bits(self.vs[phys, h, row]) if self.v_sq is not None else None
        k, v, r, s = chunk.cached_rows(head, self.kc[phys, h, row], self.vc[phys, h, row], rho, grid)
        held = self.banded(b)
        if held.any():
            at = np.flatnonzero(held)
            slot = np.where(at < self.band.n_sink, at, self.band.n_sink + at % max(self.band.n_rec, 1))
            k[at], v[at] = self.bk[b, h, slot], self.bv[b, h, slot]
        return k, v, r, s, grid

    def attend(self, q, lens, window=0, sinks=None, scale=None, bf16=True):
        """Outputs [B][n][Hq][D] in fp64 of queries q (numpy), and the bound of their error: see
        test_gpu_chunk_attn.py."""
        B, n, Hq, D = q.shape
        G = Hq // self.H
        scale = scale or 1 / np.sqrt(D)
        out, tol = np.zeros(q.shape), np.zeros(q.shape)
        for b in range(B):
            m, S = lens[b], self.seqs[b]
            if m == 0 or S == 0:
                continue
            held = self.banded(b)
            for h in range(self.H):
                hs = slice(h * G, (h + 1) * G)
                k, v, r, s, grid = self.rows(b, h)
                x = q[b, :m, hs]
                o = chunk.attend(x, k, v, S - m + np.arange(m), window, None if sinks is None else sinks[hs], scale)
                size = np.linalg.norm(v, axis=1)
                if grid is not None:
                    mid = np.abs(grid[:, 1] + 1.5 * grid[:, 0])
                    size = np.where(held, size, np.sqrt(D) * (1.5 * np.abs(grid[:, 0]) + mid))
                U = size.max()
                kbar = np.abs(x) @ np.abs(self.arrays["kbar"][h]) * scale                          # [m][G]
                turned = np.abs(x @ self.arrays["t_k_inv_t"][h]) @ np.abs(r[~held]).T if not held.all() else np.zeros((m, G, 1))
                exact = np.abs(x) @ np.abs(k[held]).T if held.any() else np.zeros((m, G, 1))
                coded = turned.max(-1) * scale
                logit = np.maximum(coded, exact.max(-1) * scale) + kbar
                dz = (2.0 ** -11 * coded if bf16 else 0) + 2.0 ** -20 * logit
                out[b, :m, hs] = o
                tol[b, :m, hs] = np.abs(o) * 2.0 ** (-8 if bf16 else -24) + \
                    ((2 * dz + 2.0 ** -18 + S * 2.0 ** -30 + (2.0 ** -11 if bf16 else 0)) * U)[..., None]
        return out, tol
