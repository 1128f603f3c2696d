"""The workspace that chunk attention asks for is what its largest plan uses: partials of as many workgroups as the
CUs hold at most, no byte less than a call without a window needs, and nothing where no call is split."""

import pytest

from paper_2608_04074_amd import _native as nat
from test_chunk_host import attend, params
from test_q4_host import WORKSPACE, ref

COUNTERS = 4096


def size(batch, n, hq, max_seq, **kw):
    return nat.lib().nova_kv_chunk_attn_workspace_bytes(ref(params(**kw)), batch, n, hq, max_seq)


@pytest.mark.parametrize("D", (64, 128))
@pytest.mark.parametrize("batch,n,hq,max_seq", ((1, 4, 32, 2000), (1, 4, 32, 100000), (3, 5, 32, 4096), (1, 20, 16, 4096), (1, 256, 32, 8192), (2, 100, 8, 4096),
                                                (16, 1, 8, 4096), (15, 1, 64, 100000)))
def test_no_more_than_the_cus_hold(batch, n, hq, max_seq, D):
    rows = n * hq // 8
    tile = 16 if rows <= 16 else 32 if rows <= 32 else 128 if rows <= 128 else 256
    got = size(batch, n, hq, max_seq, head_dim=D)
    assert COUNTERS < got <= COUNTERS + 256 * tile * (D + 2) * 4 + 255
    if max_seq <= 4096:  # the layout's capacity
        for window in (0, max_seq):
            call = dict(batch=batch, n=n, hq=hq, max_seq=max_seq, window=window)
            assert attend(params(head_dim=D), ws_bytes=got - 1, **call) == WORKSPACE


@pytest.mark.parametrize("batch,n,hq,max_seq", ((31, 1, 64, 100000), (18, 1, 8, 100000), (18, 4, 32, 32768), (1, 1100, 32, 131072), (1, 1, 8, 511)))
def test_nothing_where_no_call_is_split(batch, n, hq, max_seq):
    assert size(batch, n, hq, max_seq) == 0
