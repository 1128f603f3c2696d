"""4-bit attention of keys and queries near the ends of their types' ranges whose products are ordinary, and of zero
queries over large keys. Tolerances are those of test_gpu_q4_attn.py."""

import numpy as np
import pytest
import torch

from test_gpu_q4_attn import BF, F32, check, make_cache, nk, say  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", (2, 40))
@pytest.mark.parametrize("dtype", (BF, F32))
@pytest.mark.parametrize("q_size,key_size", ((1e-31, 1e31), (1e-33, 1e33), (1e31, 1e-31), (1e33, 1e-33)))
def test_ordinary_products(nk, q_size, key_size, dtype, n):  # noqa: F811
    check(nk, [150, 40], n, 8, 2, 64, dtype, block=16, q_size=q_size, key_size=key_size)


@pytest.mark.parametrize("n", (2, 40))
@pytest.mark.parametrize("dtype", (BF, F32))
def test_zero_queries(nk, dtype, n):  # noqa: F811
    """Logits of 0 whatever the keys are: the mean of what is attended."""
    say(f"zero queries n={n} {dtype}")
    rng = np.random.default_rng(71)
    cache, _ = make_cache(nk, rng, [100], 2, 128, 16, key_size=3e36)
    plain, _ = make_cache(nk, np.random.default_rng(71), [100], 2, 128, 16)
    q = torch.zeros((1, n, 8, 128), dtype=dtype, device="cuda")
    seq = torch.tensor([100], dtype=torch.int32, device="cuda")
    assert torch.equal(nk.q4_attn(cache, q, seq, 100), nk.q4_attn(plain, q, seq, 100))
