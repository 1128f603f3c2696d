"""4-bit attention over values whose magnitudes rise or fall along the cache: a token's weight in
the softmax does not depend on its value, on what comes before it or on what comes after it.

Tolerances are those of test_gpu_q4_attn.py, at sampled queries and heads."""

import math

import numpy as np
import pytest
import torch

from oracle import q4
from test_gpu_q4_attn import BF, F32, bound, make_cache, nk, say  # noqa: F401

pytestmark = pytest.mark.gpu


def put_sizes(cache, host, sizes):
    """Values of sequence b's token t in every KV head: size * (c - 6) / 4 for its codes c."""
    vsq, where = host[3], host[4]
    for (phys, row), size in zip(where, sizes):
        vsq[phys, :, row] = q4.to_bf16_bits(np.stack([0.25 * size, -1.5 * size], -1))[:, None]
    cache.v_sq.copy_(torch.as_tensor(vsq.view(np.int16)).cuda().view(torch.bfloat16))


def check_sampled(nk, cache, host, q, seqs, rng, window=0):  # noqa: F811
    kc, vc, ksq, vsq, where = host
    B, n, Hq, D = q.shape
    H = kc.shape[1]
    G = Hq // H
    out = nk.q4_attn(cache, q, torch.tensor(seqs, dtype=torch.int32, device="cuda"), max(seqs), window=window)
    got, qd = out.double().cpu().numpy(), q.double().cpu().numpy()
    assert np.isfinite(got).all()
    for b, S in enumerate(seqs):
        i = np.unique(np.r_[max(0, n - S), n - 1, rng.integers(max(0, n - S), n, 4)])
        for h in rng.choice(H, min(2, H), replace=False):
            phys, row = where[b]
            k, ks, v, vs = (x[phys, h, row] for x in (kc, ksq, vc, vsq))
            hs = slice(h * G, (h + 1) * G)
            o, *parts = q4.attend(qd[b, i][:, hs], q4.unpack_codes(k), q4.from_bf16_bits(ks), q4.unpack_codes(v),
                                  q4.from_bf16_bits(vs), S - n + i, window, None, 1 / math.sqrt(D))
            bf16 = q.dtype == BF
            off = np.abs(got[b, i][:, hs] - o) - bound(o, *parts, S, bf16, bf16 and n * G > 32)
            assert off.max() <= 0, f"sequence {b} head {h}: {off.max():.3e} over the bound"


SIZES = {
    "ordinary, then zero": lambda t, S: np.where(t < S // 2, 1.0, 0.0),
    "zero, then ordinary": lambda t, S: np.where(t < S // 2, 0.0, 1.0),
    "ordinary, the last zero": lambda t, S: np.where(t < S - 1, 1.0, 0.0),
    "1, then 2^-31": lambda t, S: np.where(t < S // 2, 1.0, 2.0 ** -31),
    "2^31, then 1": lambda t, S: np.where(t < S // 4, 2.0 ** 31, 1.0),
    "zero, then 2^40": lambda t, S: np.where(t < S // 2, 0.0, 2.0 ** 40),
    "zero, then 2^60": lambda t, S: np.where(t < S // 2, 0.0, 2.0 ** 60),
    "2^-100, then 2^100": lambda t, S: np.where(t < S // 2, 2.0 ** -100, 2.0 ** 100),
    "2^100, then 2^-100": lambda t, S: np.where(t < S // 2, 2.0 ** 100, 2.0 ** -100),
}


@pytest.mark.parametrize("seqs,n,Hq,H,D,dtype,block", (
    ([64], 1, 4, 1, 64, BF, 0),              # the waves of one workgroup
    ([3000, 65], 1, 8, 2, 128, BF, 16),      # splits
    ([3000, 65], 5, 8, 2, 64, BF, 16),
    ([3000, 65], 4, 8, 2, 128, F32, 7),
    ([257, 700], 40, 8, 2, 64, F32, 16),     # rows of a wave's own
    ([257, 700], 40, 8, 2, 128, BF, 16),     # tiles of 128 rows, in splits
    ([129], 40, 8, 2, 64, BF, 0),
    ([641, 650, 300] * 5, 300, 8, 8, 64, BF, 16),    # tiles of 256 rows
    ([641, 650, 300] * 5, 300, 8, 8, 128, BF, 24),
))
@pytest.mark.parametrize("sizes", SIZES)
def test_values_that_rise_or_fall(nk, sizes, seqs, n, Hq, H, D, dtype, block):  # noqa: F811
    say(f"{sizes}: seqs={seqs[:3]}x{len(seqs)} n={n} heads={Hq}/{H} D={D} {dtype} block={block}")
    rng = np.random.default_rng(31)
    cache, host = make_cache(nk, rng, seqs, H, D, block)
    put_sizes(cache, host, [SIZES[sizes](np.arange(S), S) for S in seqs])
    q = torch.as_tensor(0.3 * rng.standard_normal((len(seqs), n, Hq, D))).to(dtype).cuda()
    check_sampled(nk, cache, host, q, seqs, rng)
