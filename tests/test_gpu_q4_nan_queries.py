"""4-bit attention of queries that are not finite and attend nothing: zeros, as every row that attends nothing."""

import numpy as np
import pytest
import torch

from test_gpu_q4_attn import BF, F32, make_cache, nk, say  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", (BF, F32))
@pytest.mark.parametrize("n,S", ((6, 3), (40, 30), (40, 1)))
@pytest.mark.parametrize("odd", (float("nan"), float("inf")))
def test_odd_queries_before_the_first_token(nk, odd, n, S, dtype):  # noqa: F811
    say(f"odd queries {odd} n={n} S={S} {dtype}")
    rng = np.random.default_rng(42)
    cache, _ = make_cache(nk, rng, [S, S], 2, 128, 16)
    q = torch.as_tensor(rng.standard_normal((2, n, 8, 128))).to(dtype).cuda()
    seq = torch.tensor([S, S], dtype=torch.int32, device="cuda")
    want = nk.q4_attn(cache, q, seq, S)
    q[0, :n - S, :, 7] = odd
    q[1, 0, 3, 9] = odd
    got = nk.q4_attn(cache, q, seq, S)
    assert torch.equal(got, want) and not got[:, :n - S].any()
