"""The edges of nova_kv_chunk_attn in each of its kernels: up to 32 rows per KV head (8 here), up to 128 (80) and
more (200). Released blocks, rows and queries that are not finite, with one split and with several, pools past 32
bits, magnitudes: the bounds and the oracle of test_gpu_chunk_attn.py."""

import numpy as np
import pytest
import torch

from chunk_cases import Cache
from test_gpu_chunk_attn import BF, F32, call, check, nk, queries, say  # noqa: F401

pytestmark = pytest.mark.gpu

ROWS = (8, 80, 200)


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("D,dtype", ((64, F32), (128, BF)))
def test_released_blocks_are_not_looked_up(nk, rows, D, dtype):  # noqa: F811
    n = rows // 2
    c = Cache(nk, 6, [700, 400], 2, D, 16, "band")
    q = queries(np.random.default_rng(1), (2, n, 4, D), dtype)
    ref = [call(c, q, window=w) for w in (90, 0)]
    kept = c.layout.block_table.clone()
    for w, r in zip((90, 0), ref):
        c.layout.block_table.copy_(kept)
        for b, S in enumerate(c.seqs):
            low = max(0, S - n + 1 - w) if w else 5
            c.layout.block_table[b, :max(low, 5) // 16] = -5
            c.layout.block_table[b, -(-(S - 40) // 16):] = 2 ** 30
        assert torch.equal(call(c, q, window=w), r)


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("fmt,D,dtype", (("scaled", 128, BF), ("scaled", 64, F32), ("band", 128, BF), ("band", 64, F32)))
def test_rows_that_are_not_finite_reach_only_what_attends_them(nk, fmt, D, dtype, rows):  # noqa: F811
    n = 100
    c = Cache(nk, 7, [n, n], 1, D, 16, fmt)
    if fmt == "scaled":
        at = 60
        phys, row = (int(x[at]) for x in c.where[1])
        spots = [(c.v_sq, (phys, 0, row)), (c.k_scales, (phys, 0, row))]
    else:
        at = 80
        slot = c.band.n_sink + at % c.band.n_rec
        spots = [(c.band.k, (1, 0, slot, 3)), (c.band.v, (1, 0, slot, 3))]
    m = rows // 2
    q = queries(np.random.default_rng(2), (2, m, 2, D), dtype)
    pos = np.arange(n - m, n)
    for t, where in spots:
        for value in (float("nan"), float("inf")):
            old = t[where].clone()
            t[where] = value
            for window in (0, 20):
                say(f"{fmt} {D} rows={rows} {value} window={window}")
                out = call(c, q, window=window)
                bad = (~torch.isfinite(out)).any(-1).any(-1).cpu().numpy()
                sees = (pos >= at) & ((window == 0) | (pos < at + window))
                assert not bad[0].any() and not bad[1][~sees].any()
                if value != value:
                    assert bad[1][sees].all()
            t[where] = old


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("fmt,D,dtype", (("scaled", 128, BF), ("sq", 64, F32), ("band", 128, F32), ("band", 64, BF)))
def test_a_nan_row_in_one_of_several_splits(nk, fmt, D, dtype, rows):  # noqa: F811
    """A token that the first half of the queries attends, in the first split (of the band: the last ten, in the last)."""
    S, n, W = 6000, rows // 2, 3000
    c = Cache(nk, 16, [S], 1, D, 16, fmt)
    assert nk.chunk_attn_workspace_bytes(c.params, 1, n, 2, S)
    pos = np.arange(S - n, S)
    q = queries(c.rng, (1, n, 2, D), dtype)
    ref, tol = c.attend(q.double().cpu().numpy(), [n], W, bf16=dtype == BF)
    if fmt == "band":
        at = S - 10
        sees = pos >= at
        spots = [(x, (0, 0, c.band.n_sink + at % c.band.n_rec, 3)) for x in (c.band.k, c.band.v)]
    else:
        at = S - n + n // 2 - W
        sees = pos - W < at
        phys, row = (int(x[at]) for x in c.where[0])
        spots = [(x, (phys, 0, row)) for x in (c.v_sq, c.k_scales) if x is not None]
    for t, where in spots:
        old = t[where].clone()
        t[where] = float("nan")
        out = call(c, q, window=W).double().cpu().numpy()[0]
        t[where] = old
        assert sees.any() and np.isnan(out[sees]).any(-1).all() and np.isfinite(out[~sees]).all()
        assert (np.abs(out - ref[0]) <= tol[0])[~sees].all()
    assert (np.abs(call(c, q, window=W).double().cpu().numpy() - ref) <= tol).all()


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("fmt,S", (("plain", None), ("band", None), ("scaled", 5000)))
@pytest.mark.parametrize("dtype", (BF, F32))
def test_queries_that_are_not_finite(nk, rows, fmt, S, dtype):  # noqa: F811
    """S: cached tokens, of more than one split; None: as many as queries."""
    n = rows // 2
    c = Cache(nk, 8, [S or n, 2], 1, 128, 16, fmt)
    q = queries(c.rng, (2, n, 2, 128), dtype)
    ref, tol = c.attend(q.double().cpu().numpy(), [n, n], bf16=dtype == BF)
    i = (n - 1, n - 2)
    q[0, i[0], 1, 5], q[0, i[1], 0, 70] = float("nan"), float("inf")
    q[1, 0, 0, 0] = float("nan")           # attends nothing: position 2 - n
    out = call(c, q).double().cpu().numpy()
    bad = np.isnan(out).any(-1)
    assert bad[0, i[0]].tolist() == [False, True] and bad[0, i[1]].tolist() == [True, False] and bad.sum() == 2
    assert (np.abs(out - ref) <= tol)[~bad].all()


def test_long_cache_offsets(nk):  # noqa: F811
    """Pools whose byte offsets pass 32 bits: the blocks of one sequence lie at their two ends."""
    H, D, block = 8, 128, 16
    nblk = (1 << 32) // (H * block * D // 4) + 64
    small = Cache(nk, 9, [63], H, D, block, "scaled", extra_blocks=0)
    ends = torch.tensor([[nblk - 1, 0, nblk - 40, 7]], dtype=torch.int32, device="cuda")
    order = torch.as_tensor(small.order[0, :4]).long().cuda()
    big = []
    for t in (small.k_codes, small.v_codes, small.k_scales, small.v_sq):
        x = torch.zeros((nblk,) + tuple(t.shape[1:]), dtype=t.dtype, device="cuda")
        x[ends[0].long()] = t[order]
        big.append(x)
    for dtype in (BF, F32):
        for rows in ROWS:
            q = queries(small.rng, (1, rows // 4, 32, D), dtype)
            got = nk.chunk_attn(small.params, nk.CacheLayout(block, 4, ends), q, big[0], big[1], small.seq_lens, 63, k_scales=big[2], v_sq=big[3])
            assert torch.equal(got, call(small, q)), rows


@pytest.mark.parametrize("q_size,sizes,fmt,scale", ((1e-12, {}, "plain", 0.0), (1e4, {"k_size": 1e-4, "kbar_size": 1e-4}, "plain", 0.0),
                                                     (1e12, {"kbar_size": 0.0}, "plain", 1e-13), (2.0, {"v_size": 1e-15}, "sq", 0.0),
                                                     (2.0, {"v_size": 1e12}, "sq", 0.0), (0.5, {"kbar_size": 30.0}, "band", 0.0)))
@pytest.mark.parametrize("dtype", (BF, F32))
@pytest.mark.parametrize("D", (64, 128))
def test_magnitudes_of_many_rows(nk, q_size, sizes, fmt, scale, D, dtype):  # noqa: F811
    check(nk, [300, 40], 50, 8, 2, D, dtype, fmt=fmt, q_size=q_size, scale=scale, **sizes)


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("dtype", (BF, F32))
def test_sharp_logits(nk, rows, dtype):  # noqa: F811
    check(nk, [2000], rows // 8, 8, 1, 128, dtype, q_size=40.0, fmt="scaled")
    check(nk, [2000], rows // 8, 8, 1, 64, dtype, q_size=40.0)
