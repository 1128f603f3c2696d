"""Debug mode of chunk attention and of the calls that read a cache back: the metadata is checked on the
host before a launch, and each rejected input launches nothing."""

import pytest
import torch

from chunk_cases import Cache

pytestmark = pytest.mark.gpu


def test_debug_mode_checks_metadata_before_launching():
    import paper_2608_04074_amd as nk
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    c = Cache(nk, 1, [40, 33], 2, 64, 16, "band")
    table, blocks = c.layout.block_table, c.k_codes.shape[0]
    q = torch.ones((2, 3, 4, 64), dtype=torch.bfloat16, device="cuda")
    attend = lambda lens, top=48: nk.chunk_attn(c.params, c.layout, q, c.k_codes, c.v_codes, i32(lens), top, **c.more)  # noqa: E731
    read = lambda start, n, lens=(40, 33): nk.read(c.params, c.layout, c.k_codes, c.v_codes, i32(start), n, seq_lens=i32(lens), **c.more)  # noqa: E731
    cache = nk.Q4Cache.zeros(nk.CacheLayout(16, 3, i32([[3, 0, 1], [4, 3, -1]])), 2, 2, 64, num_blocks=6)
    try:
        want, rows = attend([40, 33]), read([0, 0], 33)
        nk.set_debug(True, blocks)
        assert torch.equal(attend([40, 33]), want) and torch.equal(read([0, 0], 33)[0], rows[0])
        with pytest.raises(nk.NovaKVError, match="seq_lens\\[1\\] = 41 outside"):
            attend([8, 41], 40)
        with pytest.raises(nk.NovaKVError, match="sequence 1: positions \\[10, 34\\) are read of \\[0, 33\\)"):
            read([0, 10], 24)
        c = Cache(nk, 1, [40, 33], 2, 64, 16, "plain")
        table = c.layout.block_table
        read([0, 0], 33)
        table[1, 1] = blocks
        with pytest.raises(nk.NovaKVError, match="physical block"):
            attend([40, 33])
        with pytest.raises(nk.NovaKVError, match="sequence 1: block 1"):
            read([0, 10], 7)
        read([20, 0], 16)        # the block is not reached
        nk.q4_read(cache, i32([0, 0]), 48)      # a block that holds nothing passes, shared ones too
        cache.layout.block_table[0, 0] = 6
        with pytest.raises(nk.NovaKVError, match="physical block 6"):
            nk.q4_read(cache, i32([0, 0]), 4)
        with pytest.raises(nk.NovaKVError, match="positions \\[46, 50\\)"):
            nk.q4_read(cache, i32([16, 46]), 4)
    finally:
        nk.set_debug(False)
