"""4-bit attention of queries with a coordinate far above the others (a projection's bias makes such rows): the
others keep their bits.

Tolerance: as in test_gpu_q4_attn.py but for the query itself. bf16: exact in fp16 (a coordinate 2^-29 of the largest
and more), and a logit's sums lose below 2^-22 of its sum of magnitudes M. fp32: a multiple of its row's largest magnitude /
8323072, each coordinate off by at most half of it: a logit, as six deviations of D independent errors, by
1.74 / 8323072 N <= 2^-22 N with N = max |q_i| * |k| * scale.
"""

import math

import numpy as np
import pytest
import torch

from oracle import q4
from test_gpu_q4_attn import BF, F32, make_cache, nk, say  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("size", (30.0, 300.0, 1000.0, 5000.0))
@pytest.mark.parametrize("n,Hq,D,dtype", ((1, 8, 128, BF), (1, 8, 64, BF), (6, 8, 128, BF), (6, 8, 64, BF), (3, 8, 128, F32), (40, 8, 64, F32)))
def test_outlying_coordinates(nk, n, Hq, D, dtype, size):  # noqa: F811
    say(f"outlying coordinate {size} n={n} D={D} {dtype}")
    rng = np.random.default_rng(51)
    H, S = 2, 45
    cache, (kc, vc, ksq, vsq, ((phys, row),)) = make_cache(nk, rng, [S], H, D, 16)
    # keys of the outlying coordinate are 0 (code 8 of offset -8 scale), so that it leaves the logits alone
    kc[..., 5] = (kc[..., 5] & 0xF0) | 8
    scale = q4.from_bf16_bits(ksq[phys, :, row, 0])
    ksq[phys, :, row, 1] = q4.to_bf16_bits(-8 * scale)
    cache.k_codes.copy_(torch.as_tensor(kc).cuda())
    cache.k_sq.copy_(torch.as_tensor(ksq.view(np.int16)).cuda().view(torch.bfloat16))
    x = rng.standard_normal((1, n, Hq, D))
    x[..., 10] = size
    q = torch.as_tensor(x).to(dtype).cuda()
    got = nk.q4_attn(cache, q, torch.tensor([S], dtype=torch.int32, device="cuda"), S).double().cpu().numpy()
    qd = q.double().cpu().numpy()
    for h in range(H):
        hs = slice(4 * h, 4 * h + 4)
        k, ks, v, vs = (t[phys, h, row] for t in (kc, ksq, vc, vsq))
        o, coded, M, N, _, _, V = q4.attend(qd[0][:, hs], q4.unpack_codes(k), q4.from_bf16_bits(ks), q4.unpack_codes(v),
                                            q4.from_bf16_bits(vs), S - n + np.arange(n), 0, None, 1 / math.sqrt(D))
        V, M, N = V[:, None, None], M[..., None], N[..., None]
        dz = 2.0 ** -22 * N + 2.0 ** -22 * M
        tol = np.abs(o) * 2.0 ** (-8 if dtype == BF else -24) + ((coded + 8 * V / 15) * 2.0 ** -11 if dtype == BF else 0) + \
            (2 * dz + 2.0 ** -18 + S * 2.0 ** -30) * V
        off = np.abs(got[0][:, hs] - o) - tol
        assert off.max() <= 0, f"head {h}: {off.max():.3e} over the bound"
