"""Calls whose outputs are too large for the caches, which store them as streamed, give what the same work gives in
parts that are not."""

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("with_axes", (False, True))
@pytest.mark.parametrize("D,dtype,interleaved", ((128, torch.bfloat16, False), (128, torch.bfloat16, True), (64, torch.bfloat16, False),
                                                 (64, torch.float32, False), (128, torch.float32, True)))
def test_norm_rotation_and_append(D, dtype, interleaved, with_axes):
    import paper_2608_04074_amd as nk
    H, HQ = 8 * 128 // D, 32 * 128 // D                # 12 KiB of bf16 a token
    B, n = 4, 22000 if dtype == torch.bfloat16 else 11000
    g = torch.Generator("cuda").manual_seed(D)
    x = torch.randn(B, n, (HQ + 2 * H) * D, device="cuda", generator=g).to(dtype)
    split = lambda t: [s.unflatten(-1, (-1, D)) for s in t.split((HQ * D, H * D, H * D), -1)]  # noqa: E731
    weight = torch.rand(D, device="cuda", generator=g) + 0.5
    rotary = nk.Rotary(HQ, H, D, nk.Rotary.table(n, D), interleaved=interleaved, q_norm=weight, k_norm=weight)
    axes = nk.RotaryAxes.cycle((D // 4, D // 4))
    positions = torch.randint(0, n, (2, B, n), device="cuda", generator=g, dtype=torch.int32)
    layout = nk.CacheLayout(n, 1)
    assert x.nbytes >= 1 << 30

    def rows(at, end):
        q, k, v = split(x[:, at:end])
        start = torch.full((B,), at, dtype=torch.int32, device="cuda")
        if with_axes:
            turned = nk.rotate_qkv_axes(rotary, axes, q, k, v, positions[:, :, at:end].contiguous())
        else:
            turned = nk.rotate_qkv(rotary, q, k, v, start)
        k_held, v_held = torch.empty(k.shape, dtype=dtype, device="cuda"), torch.empty(v.shape, dtype=dtype, device="cuda")
        if with_axes:
            q_out = nk.q4_append_axes(rotary, axes, cache, q, k, v, start, positions[:, :, at:end].contiguous(), k_held=k_held, v_held=v_held)
        else:
            q_out = nk.q4_append(rotary, cache, q, k, v, start, k_held=k_held, v_held=v_held)
        return [*turned, q_out, k_held, v_held]

    cache = nk.Q4Cache.zeros(layout, B, H, D)
    whole = rows(0, n)
    pools = [t.clone() for t in cache.tensors[1:]]
    for t in cache.tensors[1:]:
        t.zero_()
    for at in range(0, n, 6000):
        for t, part in zip(whole, rows(at, min(at + 6000, n))):
            assert torch.equal(t[:, at:at + 6000], part)
    assert all(torch.equal(t, u) for t, u in zip(pools, cache.tensors[1:]))


@pytest.mark.parametrize("D,dtype", ((128, torch.bfloat16), (64, torch.bfloat16), (64, torch.bfloat16), (64, torch.float32)))
def test_reading_the_4_bit_cache(D, dtype):
    import paper_2608_04074_amd as nk
    B, H, S = 10, 8 * 128 // D, 8192                 # 320 MiB in bf16
    g = torch.Generator("cuda").manual_seed(D)
    cache = nk.Q4Cache.zeros(nk.CacheLayout(16, S // 16, torch.randperm(B * S // 16, device="cuda", generator=g).int().view(B, -1)), B, H, D)
    for codes in (cache.k_codes, cache.v_codes):
        codes.copy_(torch.randint(0, 256, codes.shape, device="cuda", generator=g, dtype=torch.uint8))
    for sq in (cache.k_sq, cache.v_sq):
        sq.copy_(torch.randn(sq.shape, device="cuda", generator=g))
    start = torch.zeros(B, dtype=torch.int32, device="cuda")
    whole = nk.q4_read(cache, start, S, dtype=dtype)
    for at in range(0, S, 2048):
        part = nk.q4_read(cache, start + at, 2048, dtype=dtype)
        for x, y in zip(whole, part):
            assert torch.equal(x[:, at:at + 2048], y)
