"""4-bit cache: values, keys and heads whose magnitudes lie far apart.

Tolerances of attention are those of test_gpu_q4_attn.py, from what a row attends
alone."""

import math

import numpy as np
import pytest
import torch

from oracle import q4
from test_gpu_q4_attn import BF, F32, make_cache, nk, reference_and_bounds, say  # noqa: F401

pytestmark = pytest.mark.gpu


def put_values(cache, host, b, tokens, scale, offset):
    """Scale and offset of the values of a sequence's tokens, in every KV head."""
    vsq, where = host[3], host[4]
    phys, row = (x[tokens] for x in where[b])
    vsq[phys, :, row] = q4.to_bf16_bits(np.array([scale, offset]))
    cache.v_sq.copy_(torch.as_tensor(vsq.view(np.int16)).cuda().view(torch.bfloat16))


def assert_within(nk, cache, host, q, seqs, window=0):
    n, D = q.shape[1], q.shape[3]
    out = nk.q4_attn(cache, q, torch.tensor(seqs, dtype=torch.int32, device="cuda"), max(seqs), window=window)
    ref, tol = reference_and_bounds(host, q.double().cpu().numpy(), seqs, [n] * len(seqs), window, None, 1 / math.sqrt(D),
                                    q.dtype == BF)
    got = out.double().cpu().numpy()
    assert np.isfinite(got).all()
    assert (np.abs(got - ref) <= tol).all(), f"{(np.abs(got - ref) - tol).max():.3e} over the bound"


@pytest.mark.parametrize("dtype", (BF, F32))
@pytest.mark.parametrize("n", (1, 5, 40))
@pytest.mark.parametrize("value", (0.0, -1000.0, 1e25, 1e-25))
def test_constant_values(nk, value, n, dtype):  # noqa: F811
    """Every value row is one constant (scale 0), while later logits grow."""
    say(f"constant values {value} n={n} {dtype}")
    rng = np.random.default_rng(11)
    seqs = [3000, 65]
    cache, host = make_cache(nk, rng, seqs, 2, 64, 16)
    for b, S in enumerate(seqs):
        put_values(cache, host, b, np.arange(S), 0.0, value)
    q = torch.as_tensor(3 * rng.standard_normal((2, n, 8, 64))).to(dtype).cuda()
    assert_within(nk, cache, host, q, seqs)


@pytest.mark.parametrize("dtype,n,Hq", ((BF, 1, 8), (BF, 4, 8), (BF, 16, 4), (F32, 4, 8), (F32, 40, 8)))
@pytest.mark.parametrize("size", (1e4, 1e12, 1e30))
def test_hidden_tokens_with_large_values(nk, size, dtype, n, Hq):  # noqa: F811
    """Tokens that some of a call's rows do not attend, with values far above the others'.
    (In front of the window, and behind the first queries.)"""
    say(f"hidden large values {size} n={n} heads={Hq} {dtype}")
    rng = np.random.default_rng(12)
    seqs = [100, 47]
    cache, host = make_cache(nk, rng, seqs, 2, 128, 16)
    for b, S in enumerate(seqs):
        put_values(cache, host, b, np.array([S - 20 - n, S - 1] if n > 1 else [S - 21]), size, -3 * size)
    q = torch.as_tensor(rng.standard_normal((2, n, Hq, 128))).to(dtype).cuda()
    assert_within(nk, cache, host, q, seqs, window=20)


@pytest.mark.parametrize("dtype", (BF, F32))
def test_large_values_of_little_weight(nk, dtype):  # noqa: F811
    """A token whose value is 2^40 times the others' and whose probability is nothing."""
    rng = np.random.default_rng(13)
    S, D = 64, 64
    cache, host = make_cache(nk, rng, [S], 1, D, 0)
    kc, vc, ksq, vsq, _ = host
    ksq[0, 0, :S] = q4.to_bf16_bits(np.array([0.0, 0.0]))
    ksq[0, 0, 40] = q4.to_bf16_bits(np.array([0.0, -8.0]))  # its logit: -8 sum(q) / 8, -256
    cache.k_sq.copy_(torch.as_tensor(ksq.view(np.int16)).cuda().view(torch.bfloat16))
    put_values(cache, host, 0, np.array([40]), 2.0 ** 40, -2.0 ** 42)
    q = torch.full((1, 1, 4, D), 4.0, dtype=dtype, device="cuda")
    out = nk.q4_attn(cache, q, torch.tensor([S], dtype=torch.int32, device="cuda"), S).double().cpu().numpy()
    keep = np.arange(S) != 40
    v = q4.unpack_codes(vc[0, 0, :S]) * q4.from_bf16_bits(vsq[0, 0, :S, :1]) + q4.from_bf16_bits(vsq[0, 0, :S, 1:])
    ref = v[keep].mean(0)
    # its weight is e^-256 / 63, of an output 2^42 e^-256: nothing; the others are alike, exactly 1 / 63.
    # Roundings: the output's; a probability's to fp16 (bf16 queries), the sum's 63 of fp32.
    tol = np.abs(ref) * 2.0 ** (-8 if dtype == BF else -24) + np.abs(v[keep]).max() * (2.0 ** -11 if dtype == BF else 0) + \
        np.abs(v[keep]).max() * 2.0 ** -18
    assert (np.abs(out[0, 0] - ref) <= tol).all()


@pytest.mark.parametrize("n", (40, 70))
@pytest.mark.parametrize("D", (64, 128))
def test_tokens_far_below_their_neighbours(nk, n, D):  # noqa: F811
    """Many bf16 queries over tokens of which every fourth is 2^8 times the others, with logits
    that hide it: keys and values are rounded to 2^-12 of theirs, or 2^-18 of the largest around."""
    say(f"far below n={n} D={D}")
    rng = np.random.default_rng(14)
    S, G = 200, 4
    cache, host = make_cache(nk, rng, [S], 1, D, 16)
    kc, vc, ksq, vsq, ((phys, row),) = host
    large = np.arange(S) % 4 == 3
    size = np.where(large, 2.0 ** 8, 1.0)
    ksq[phys, 0, row] = q4.to_bf16_bits(np.stack([np.where(large, 0.0, 0.01), np.where(large, -64.0, 0.25)], -1))
    vsq[phys, 0, row] = q4.to_bf16_bits(np.stack([0.25 * size, -1.5 * size], -1))
    dev = lambda x: torch.as_tensor(x.view(np.int16)).cuda().view(torch.bfloat16)  # noqa: E731
    cache.k_sq.copy_(dev(ksq))
    cache.v_sq.copy_(dev(vsq))
    q = torch.as_tensor(0.25 + 0.25 * rng.random((1, n, G, D))).to(BF).cuda()  # logits of large tokens: below -64 * 0.25 sqrt(D)
    got = nk.q4_attn(cache, q, torch.tensor([S], dtype=torch.int32, device="cuda"), S).double().cpu().numpy()
    qd = q.double().cpu().numpy()
    # every row attends a token that is not large, whose weight e^-128 leaves of the large ones below 2^8 e^-128
    k = q4.from_bf16_bits(ksq[phys, 0, row])
    v = q4.from_bf16_bits(vsq[phys, 0, row])
    kd = k[:, 1:] + k[:, :1] * q4.unpack_codes(kc[phys, 0, row])
    vd = v[:, 1:] + v[:, :1] * q4.unpack_codes(vc[phys, 0, row])
    small = ~large
    for i in range(n):
        at = np.flatnonzero(small & (np.arange(S) <= S - n + i))
        z = qd[0, i] @ kd[at].T / np.sqrt(D)
        p = np.exp(z - z.max(1, keepdims=True))
        p /= p.sum(1, keepdims=True)
        ref, V = p @ vd[at], np.abs(vd[at]).max()
        # a key's coordinate is off by 2^-18 * 64, a logit by that times sum(q) / sqrt(D), a probability by twice that;
        # a value by 2^-18 * 2.25 * 2^8; the output's rounding, a probability's, a sum's as elsewhere
        dz = 2.0 ** -12 * qd[0, i].sum(-1, keepdims=True) / np.sqrt(D)
        tol = np.abs(ref) * 2.0 ** -8 + 2 * dz * V + 2.25 * 2.0 ** -10 + V * (2.0 ** -11 + 2.0 ** -18)
        assert (np.abs(got[0, i] - ref) <= tol).all(), (i, (np.abs(got[0, i] - ref) - tol).max())


@pytest.mark.parametrize("dtype", (BF, F32))
@pytest.mark.parametrize("key_size,weight", ((1e-21, 1.0), (1e-23, 1e4), (2.0 ** 30, 2.0 ** -100), (3e19, 1.0)))
def test_norms_past_fp32(nk, key_size, weight, dtype):  # noqa: F811
    """Keys whose squares, or weights whose products, leave the normal fp32 numbers: the codes
    are those of fp64 all the same, of few tokens and of many."""
    say(f"norms past fp32: keys {key_size} weight {weight} {dtype}")
    rng = np.random.default_rng(15)
    H, D = 2, 128
    w = torch.full((D,), weight, device="cuda") * torch.as_tensor(rng.uniform(0.5, 1, D)).float().cuda()
    rot = nk.Rotary(H, H, D, k_norm=w, eps=0.0)
    for n in (3, 600):
        cache = nk.Q4Cache.zeros(nk.CacheLayout.contiguous(n), 1, H, D)
        k = torch.as_tensor(key_size * rng.standard_normal((1, n, H, D))).to(dtype).cuda()
        nk.q4_append(rot, cache, None, k, k, torch.zeros(1, dtype=torch.int32, device="cuda"))
        y = q4.norm_rotate(k.double().cpu().numpy(), w.double().cpu().numpy())
        codes, sq, gap = q4.quantize_rows(y[0].transpose(1, 0, 2))
        assert (cache.k_sq.view(torch.int16).cpu().numpy().view(np.uint16)[0] == sq).all()
        got = q4.unpack_codes(cache.k_codes.cpu().numpy()[0])
        assert ((got == codes) | (gap < 1e-9)).all()
