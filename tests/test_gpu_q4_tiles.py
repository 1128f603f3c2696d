"""nova_kv_q4_attn of many query rows: calls whose rows fill tiles of either size, whole and in
splits, checked at sampled queries with the tolerances of test_gpu_q4_attn.py."""

import math

import numpy as np
import pytest
import torch

from oracle import q4
from test_gpu_q4_attn import BF, bound, make_cache, nk, say  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,block", ((64, 0), (128, 16), (128, 7), (64, 24)))
@pytest.mark.parametrize("seqs,n,Hq,H,window", (
    ([700, 650, 300] * 5, 300, 8, 8, 0),     # tiles of 256 rows, whole
    ([12000], 512, 32, 8, 0),                # many rows over a long cache: splits
    ([12000], 512, 32, 8, 3000),
    ([2000, 1], 70, 8, 2, 0),                # few tiles of 128 rows, in splits
    ([4000, 333], 16, 16, 4, 0),             # tiles whose last waves have no rows
))
def test_tiles(nk, seqs, n, Hq, H, window, D, block):  # noqa: F811
    say(f"tiles seqs={seqs[:3]}x{len(seqs)} n={n} heads={Hq}/{H} D={D} block={block} window={window}")
    rng = np.random.default_rng(21)
    B, G = len(seqs), Hq // H
    cache, (kc, vc, ksq, vsq, where) = make_cache(nk, rng, seqs, H, D, block)
    q = torch.as_tensor(rng.standard_normal((B, n, Hq, D))).to(BF).cuda()
    got = nk.q4_attn(cache, q, torch.tensor(seqs, dtype=torch.int32, device="cuda"), max(seqs), window=window)
    got, qd = got.double().cpu().numpy(), q.double().cpu().numpy()
    assert np.isfinite(got).all()
    for b, S in enumerate(seqs):
        for h in rng.choice(H, 2, replace=False):
            phys, row = where[b]
            k, ks, v, vs = (x[phys, h, row] for x in (kc, ksq, vc, vsq))
            i = np.unique(np.r_[0, n - 1, rng.integers(0, n, 4)])
            hs = slice(h * G, (h + 1) * G)
            o, *parts = q4.attend(qd[b, i][:, hs], q4.unpack_codes(k), q4.from_bf16_bits(ks), q4.unpack_codes(v),
                                  q4.from_bf16_bits(vs), S - n + i, window, None, 1 / math.sqrt(D))
            off = np.abs(got[b, i][:, hs] - o) - bound(o, *parts, S, True, n * G > 32)
            assert off.max() <= 0, f"sequence {b} head {h}: {off.max():.3e} over the bound"
