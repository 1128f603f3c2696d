"""4-bit attention of rows that are not finite: a cached row that is NaN shows in every output that attends it,
however small its weight and wherever a split ends, and in no other."""

import numpy as np
import pytest
import torch

from test_gpu_q4_attn import BF, F32, make_cache, nk, say  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,dtype", ((1, BF), (1, F32), (5, BF), (5, F32), (40, BF), (40, F32)))
@pytest.mark.parametrize("side", ("k", "v"))
@pytest.mark.parametrize("D,S", ((64, 300), (128, 4000)))
def test_nan_rows_of_no_weight(nk, D, S, side, n, dtype):  # noqa: F811
    """Every token of the first half has a weight of e^-200 and less beside the second half's."""
    say(f"nan {side} row of no weight D={D} S={S} n={n} {dtype}")
    rng = np.random.default_rng(41)
    cache, (kc, vc, ksq, vsq, ((phys, row),)) = make_cache(nk, rng, [S], 1, D, 16)
    seen = torch.as_tensor(phys).cuda().long(), torch.as_tensor(row).cuda().long()
    half = torch.arange(S, device="cuda") < S // 2
    cache.k_sq[seen[0], 0, seen[1], 0] = 0
    cache.k_sq[seen[0], 0, seen[1], 1] = torch.where(half, 0.0, 32.0).bfloat16()   # logits 0 and 32 sqrt(D)
    q = torch.ones((1, n, 2, D), dtype=dtype, device="cuda")
    seq = torch.tensor([S], dtype=torch.int32, device="cuda")
    assert torch.isfinite(nk.q4_attn(cache, q, seq, S)).all()
    sq = cache.k_sq if side == "k" else cache.v_sq
    sq[int(phys[10]), 0, int(row[10])] = float("nan")
    assert torch.isnan(nk.q4_attn(cache, q, seq, S)).all()
    assert torch.isfinite(nk.q4_attn(cache, q, seq, S, window=S - n - 11)).all()
