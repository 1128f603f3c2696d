"""4-bit attention of many bf16 queries beside tokens far above the others, in value or in key: hidden ones (in front
of the window, behind the first queries), and ones that are attended with a weight of nothing.

Tolerances are those of test_gpu_q4_attn.py, from what a row attends alone."""

import math

import numpy as np
import pytest
import torch

from oracle import q4
from test_gpu_q4_attn import BF, make_cache, nk, reference_and_bounds, say  # noqa: F401
from test_gpu_q4_weights import check_sampled

pytestmark = pytest.mark.gpu


def put(cache, host, side, b, tokens, scale, offset):
    sq, where = host[2 if side == "k" else 3], host[4]
    phys, row = (x[tokens] for x in where[b])
    sq[phys, :, row] = q4.to_bf16_bits(np.array([scale, offset]))
    (cache.k_sq if side == "k" else cache.v_sq).copy_(torch.as_tensor(sq.view(np.int16)).cuda().view(torch.bfloat16))


@pytest.mark.parametrize("side", ("k", "v"))
@pytest.mark.parametrize("D,block", ((64, 16), (128, 16), (128, 7)))
@pytest.mark.parametrize("size", (1e3, 1e4, 1e12, 1e30))
def test_hidden_tokens_far_above(nk, size, D, block, side):  # noqa: F811
    """Each call's last token, and one in front of every window, are `size` times the others: only the last query
    attends the first of them (its own position), none the other."""
    say(f"hidden {side} {size} D={D} block={block}")
    rng = np.random.default_rng(61)
    seqs, n, window = [200, 147], 40, 20
    cache, host = make_cache(nk, rng, seqs, 2, D, block)
    for b, S in enumerate(seqs):
        put(cache, host, side, b, np.array([S - n - window, S - 1]), size, -3 * size)
    q = torch.as_tensor(rng.standard_normal((2, n, 8, D))).to(BF).cuda()
    out = nk.q4_attn(cache, q, torch.tensor(seqs, dtype=torch.int32, device="cuda"), max(seqs), window=window)
    ref, tol = reference_and_bounds(host, q.double().cpu().numpy(), seqs, [n, n], window, None, 1 / math.sqrt(D), True)
    got = out.double().cpu().numpy()
    rest = slice(0, n - 1)
    assert np.isfinite(got[:, rest]).all()
    assert (np.abs(got - ref) <= tol)[:, rest].all(), f"{(np.abs(got - ref) - tol)[:, rest].max():.3e} over the bound"
    if side == "v":
        assert (np.abs(got - ref) <= tol).all()


@pytest.mark.parametrize("D", (64, 128))
@pytest.mark.parametrize("size", (2.0 ** 12, 2.0 ** 40, 2.0 ** 90))
def test_tokens_of_no_weight_far_above(nk, size, D):  # noqa: F811
    """Every fourth value is `size` times the others, and its weight e^-256 of theirs."""
    say(f"no weight {size} D={D}")
    rng = np.random.default_rng(62)
    S, n = 200, 40
    cache, host = make_cache(nk, rng, [S], 1, D, 16)
    (phys, row), = host[4]
    large = np.arange(S) % 4 == 3
    put(cache, host, "k", 0, np.flatnonzero(large), 0.0, -256.0 / math.sqrt(D))
    put(cache, host, "v", 0, np.flatnonzero(large), size, -3 * size)
    put(cache, host, "k", 0, np.flatnonzero(~large), 0.0, 0.0)
    q = torch.ones((1, n, 4, D), dtype=BF, device="cuda")   # logits: 0, and -256 of the large ones
    got = nk.q4_attn(cache, q, torch.tensor([S], dtype=torch.int32, device="cuda"), S).double().cpu().numpy()
    v = q4.unpack_codes(host[1][phys, 0, row]) * q4.from_bf16_bits(host[3][phys, 0, row, :1]) + q4.from_bf16_bits(host[3][phys, 0, row, 1:])
    V = np.abs(v[~large]).max()
    for i in range(n):
        ref = v[~large & (np.arange(S) <= S - n + i)].mean(0)
        # the output's rounding, a probability's and a value's to fp16, the sums'; of the large ones size e^-256 and less: nothing
        tol = np.abs(ref) * 2.0 ** -8 + V * (2.0 ** -11 + 2.0 ** -10 + 2.0 ** -18)
        assert (np.abs(got[0, i] - ref) <= tol).all(), i


@pytest.mark.parametrize("side,size", (("k", 1e3), ("k", 1e4), ("v", 1e4), ("v", 1e30)))
@pytest.mark.parametrize("D", (64, 128))
def test_hidden_tokens_of_large_tiles(nk, size, D, side):  # noqa: F811
    """The same in tiles of 256 rows: tokens that only the last queries attend."""
    say(f"hidden {side} {size} D={D}, tiles of 256 rows")
    rng = np.random.default_rng(63)
    seqs, n, window = [641, 650, 700] * 5, 300, 20
    cache, host = make_cache(nk, rng, seqs, 8, D, 16)
    for b, S in enumerate(seqs):
        put(cache, host, side, b, np.array([S - 3, S - 60]), size, -3 * size)
    q = torch.as_tensor(rng.standard_normal((len(seqs), n, 8, D))).to(BF).cuda()
    check_sampled(nk, cache, host, q, seqs, rng, window)


@pytest.mark.parametrize("D", (64, 128))
def test_hidden_keys_near_the_end_of_fp32(nk, D):  # noqa: F811
    """Hidden keys of 1e38 beside keys of 1e-5 under queries of 1e5, whose products are ordinary."""
    rng = np.random.default_rng(64)
    S, n, window = 200, 40, 20
    cache, host = make_cache(nk, rng, [S], 2, D, 16, key_size=1e-5)
    put(cache, host, "k", 0, np.array([S - 1]), 1e36, -1e38)   # only the last query attends it
    q = torch.as_tensor(1e5 * rng.standard_normal((1, n, 8, D))).to(BF).cuda()
    out = nk.q4_attn(cache, q, torch.tensor([S], dtype=torch.int32, device="cuda"), S, window=window).double().cpu().numpy()
    ref, tol = reference_and_bounds(host, q.double().cpu().numpy(), [S], [n], window, None, 1 / math.sqrt(D), True)
    off = (np.abs(out - ref) - tol)[:, :n - 1]
    assert (off <= 0).all(), f"{off.max():.3e} over the bound"


@pytest.mark.parametrize("seqs,n,Hq,H,D", (([700, 431], 40, 8, 2, 128), ([641, 650, 700] * 5, 300, 8, 8, 64), ([9000], 70, 8, 2, 64)))
def test_repeatable(nk, seqs, n, Hq, H, D):  # noqa: F811
    """Tiles of either size, whole and in splits, with and without tokens far above the others: the same every time."""
    rng = np.random.default_rng(65)
    cache, host = make_cache(nk, rng, seqs, H, D, 16)
    put(cache, host, "v", 0, np.arange(0, seqs[0], 150), 1e4, -3e4)
    q = torch.as_tensor(rng.standard_normal((len(seqs), n, Hq, D))).to(BF).cuda()
    seq = torch.tensor(seqs, dtype=torch.int32, device="cuda")
    want = nk.q4_attn(cache, q, seq, max(seqs))
    for _ in range(20):
        assert torch.equal(nk.q4_attn(cache, q, seq, max(seqs)), want)
