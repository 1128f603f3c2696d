"""Calls whose outputs are too large for the caches, which store them as streamed, give what the same work gives in
parts that are not."""

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,dtype", ((128, torch.bfloat16), (64, torch.bfloat16), (64, torch.float32)))
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
