"""nova_kv_chunk_attn with more than 128 rows per KV head (tiles of 256 rows) in every format: the bounds and the
oracle of test_gpu_chunk_attn.py."""

import numpy as np
import pytest
import torch

from chunk_cases import FORMATS, Cache
from oracle.q4 import to_bf16_bits
from test_gpu_chunk_attn import BF, F32, call, check, nk  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("D,dtype", ((64, BF), (64, F32), (128, BF), (128, F32)))
def test_formats(nk, fmt, D, dtype):  # noqa: F811
    """Two tiles, the second of few rows; lengths that end inside a round; idle and short sequences."""
    check(nk, [333, 70, 0, 5], 66, 4, 1, D, dtype, block=16, fmt=fmt, q_lens=[66, 33, 0, 5])
    check(nk, [1100, 130], 130, 2, 1, D, dtype, fmt=fmt, q_lens=[130, 129])


@pytest.mark.parametrize("block", (1, 7, 24, 48))
@pytest.mark.parametrize("D,dtype,fmt", ((64, BF, "scaled"), (128, F32, "plain"), (128, BF, "deployed"), (64, F32, "sq")))
def test_pages(nk, block, D, dtype, fmt):  # noqa: F811
    check(nk, [515, 131], 67, 4, 2, D, dtype, block=block, fmt=fmt)


@pytest.mark.parametrize("window", (1, 33, 128, 400))
@pytest.mark.parametrize("D,dtype,fmt", ((64, BF, "plain"), (128, F32, "deployed"), (128, BF, "band")))
def test_windows_and_sinks(nk, window, D, dtype, fmt):  # noqa: F811
    """Windows shorter than a tile's positions: waves of one workgroup attend spans apart."""
    sinks = np.array([-np.inf, 3.0])
    check(nk, [700, 150], 150, 2, 2, D, dtype, block=16, fmt=fmt, window=window, sinks=sinks)


@pytest.mark.parametrize("seq,n,window", ((5000, 40, 0), (5000, 300, 700)))
@pytest.mark.parametrize("D,dtype,fmt", ((64, F32, "deployed"), (128, BF, "plain"), (128, F32, "scaled")))
def test_splits(nk, seq, n, window, D, dtype, fmt):  # noqa: F811
    check(nk, [seq, seq // 3], n, 8, 1, D, dtype, block=16, fmt=fmt, window=window)


@pytest.mark.parametrize("dtype", (BF, F32))
@pytest.mark.parametrize("n", (1, 40, 150))
def test_a_long_tail_of_small_weights(nk, n, dtype):  # noqa: F811
    """One key's weight is e^10.5 times that of each of 40000 others, which together weigh more than it: weights
    below fp16's normal numbers count, in sums as beside values."""
    S, D = 40000, 64
    c = Cache(nk, 11, [S], 1, D, 16, "key_scale", kbar_size=0.0)
    phys, row = c.where[0]
    c.ks[phys, :, row] = to_bf16_bits(np.full((S, 1), 2.0 ** -20))
    c.ks[phys[7], :, row[7]] = to_bf16_bits(np.ones(1))
    c.k_scales = torch.as_tensor(c.ks.view(np.int16)).cuda().view(BF)
    key = c.rows(0, 0)[0][7]
    q = torch.as_tensor(np.broadcast_to(key * (10.5 * np.sqrt(D) / (key @ key)), (1, n, 1, D)).copy()).to(dtype).cuda()
    got = call(c, q).double().cpu().numpy()
    ref, tol = c.attend(q.double().cpu().numpy(), [n], bf16=dtype == BF)
    assert (np.abs(got - ref) <= tol).all(), (np.abs(got - ref) - tol).max()
    # the bound tells a lost tail: without it the outputs are the one value
    assert (np.abs(c.rows(0, 0)[1][7] - ref) > 4 * tol).any()


@pytest.mark.parametrize("n", (30, 70))
def test_replays_with_other_lengths(nk, n):  # noqa: F811
    """A captured call in splits is replayed with lengths that shrink and grow on the device, eager calls between
    the replays in the same workspace: the same outputs every time."""
    c = Cache(nk, 14, [6000, 4000], 1, 128, 16)
    q = torch.as_tensor(2.0 * c.rng.standard_normal((2, n, 8, 128))).to(BF).cuda()
    need = nk.chunk_attn_workspace_bytes(c.params, 2, n, 8, c.top)
    assert need
    ws, out = torch.zeros(need, dtype=torch.uint8, device="cuda"), torch.empty_like(q)
    q_lens = torch.tensor([n, n], dtype=torch.int32, device="cuda")
    args = (c.params, c.layout, q, c.k_codes, c.v_codes, c.seq_lens, c.top, out, ws)
    eager = nk.prepare_chunk_attn(*args, q_lens=q_lens)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        nk.prepare_chunk_attn(*args, q_lens=q_lens)()
    for lens, seqs in (([n, n], [6000, 4000]), ([1, n], [33, 2]), ([0, 5], [6000, 0]), ([n, n - 1], [n, 3999]), ([n, n], [6000, 4000])):
        q_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        c.seq_lens.copy_(torch.tensor(seqs, dtype=torch.int32))
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        replayed = out.clone()
        for _ in range(3):
            out.fill_(7.0)
            eager()
            torch.cuda.synchronize()
            assert torch.equal(replayed, out)
        for b in range(2):
            assert (out[b, lens[b]:] == 7).all() and out[b, :lens[b]].isfinite().all()
    ref, tol = c.attend(q.double().cpu().numpy(), [n, n])
    assert (np.abs(out.double().cpu().numpy() - ref) <= tol).all()
