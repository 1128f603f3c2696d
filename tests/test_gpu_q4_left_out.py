"""Outputs that rotate_qkv and q4_append make themselves: tokens that a call leaves out (positions outside the
table or the cache, blocks that hold nothing) are zeros in them, like padding."""

import pytest
import torch

pytestmark = pytest.mark.gpu


def used_memory(*shapes):
    """Leaves what the next tensors of these shapes may be made in full of sevens."""
    junk = [torch.full(s, 7.0, dtype=torch.bfloat16, device="cuda") for s in shapes for _ in range(4)]
    torch.cuda.synchronize()
    del junk


@pytest.mark.parametrize("append", (False, True))
def test_left_out_tokens_are_zeros(append):
    import paper_2608_04074_amd as nk
    B, n, Hq, H, D = 4, 6, 4, 2, 64
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    ones = lambda h: torch.ones((B, n, h, D), dtype=torch.bfloat16, device="cuda")  # noqa: E731
    q, k, v = ones(Hq), ones(H), ones(H)
    rot = nk.Rotary(Hq, H, D, cos_sin=nk.Rotary.table(40, D))
    start = i32([-3, 13, 0, 37])
    used_memory(q.shape, k.shape)
    if append:
        table = i32([[0, 1, 2], [3, -1, 4], [-1, -1, -1], [7, 8, 5]])   # sequence 2 is idle
        cache = nk.Q4Cache.zeros(nk.CacheLayout(16, 3, table), B, H, D, num_blocks=9)
        used_memory(q.shape, k.shape)
        outs = [nk.q4_append(rot, cache, q, k, v, start)]
        taken = [[i >= 3 for i in range(n)], [13 + i < 16 for i in range(n)], [False] * n, [37 + i < 40 for i in range(n)]]
    else:
        outs = nk.rotate_qkv(rot, q, k, v, start)
        taken = [[i >= 3 for i in range(n)], [True] * n, [True] * n, [37 + i < 40 for i in range(n)]]
    for out in outs:
        assert out.any(-1).any(-1).tolist() == taken
