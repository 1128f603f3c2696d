"""Windows far longer than any sequence attend what no window attends, in nova_kv_chunk_attn and in
nova_kv_q4_attn: in the plan (on the CPU, where a call in splits is refused for its missing workspace) and in the
outputs, of calls with more queries than tokens among them."""

import numpy as np
import pytest
import torch

from chunk_cases import Cache
from test_chunk_host import attend
from test_q4_host import WORKSPACE

WIDE = (4096, 4097, 2 ** 30, 2 ** 31 - 300, 2 ** 31 - 2, 2 ** 31 - 1)


@pytest.mark.parametrize("window", WIDE)
@pytest.mark.parametrize("n,hq", ((1, 32), (3, 32), (20, 32), (100, 16)))
def test_a_wide_window_is_planned_like_none(n, hq, window):
    shape = dict(batch=1, n=n, hq=hq, ws=None)
    assert attend(window=0, **shape) == attend(window=window, **shape) == WORKSPACE


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", (torch.bfloat16, torch.float32))
@pytest.mark.parametrize("n", (2, 20, 70))
@pytest.mark.parametrize("fmt", ("plain", "deployed"))
def test_chunk_attention(n, fmt, dtype):
    import paper_2608_04074_amd as nk
    seqs = [900, 5, n, 0]
    c = Cache(nk, 3, seqs, 2, 64, 16, fmt)
    q = torch.as_tensor(np.random.default_rng(n).standard_normal((4, n, 8, 64))).to(dtype).cuda()
    run = lambda w: nk.chunk_attn(c.params, c.layout, q, c.k_codes, c.v_codes, c.seq_lens, c.top, window=w, **c.more)  # noqa: E731
    want = run(0)
    for b, S in enumerate(seqs):
        assert want[b, max(0, n - S):].ne(0).any(-1).all() and not want[b, :max(0, n - S)].any()
    for window in (900,) + WIDE:
        assert torch.equal(run(window), want), window


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", (torch.bfloat16, torch.float32))
@pytest.mark.parametrize("n", (2, 20, 70))
def test_attention_over_the_4_bit_cache(n, dtype):
    import paper_2608_04074_amd as nk
    seqs, D = [900, 5, n, 0], 64
    rng = np.random.default_rng(n)
    cache = nk.Q4Cache.zeros(nk.CacheLayout(16, 57), 4, 2, D)
    rotary = nk.Rotary(8, 2, D)
    rows = lambda heads, tokens: torch.as_tensor(rng.standard_normal((4, tokens, heads, D))).to(dtype).cuda()  # noqa: E731
    start = torch.zeros(4, dtype=torch.int32, device="cuda")
    nk.q4_append(rotary, cache, None, rows(2, 900), rows(2, 900), start)
    q, lens = rows(8, n), torch.tensor(seqs, dtype=torch.int32, device="cuda")
    run = lambda w: nk.q4_attn(cache, q, lens, 900, window=w)  # noqa: E731
    want = run(0)
    for b, S in enumerate(seqs):
        assert want[b, max(0, n - S):].ne(0).any(-1).all() and not want[b, :max(0, n - S)].any()
    for window in (900,) + WIDE:
        assert torch.equal(run(window), want), window
