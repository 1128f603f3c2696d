"""nova_kv_q4_attn against the fp64 oracle, at the lengths, head counts, pages and
masks where it can go wrong.

Tolerance of an output value, from the roundings on its way (u = 2^-24):
  - its own rounding to bf16 or fp32: half a step, |ref| * 2^-8 or * 2^-24;
  - bf16 queries: probabilities times scales are rounded to fp16, half a step each,
    2^-11 * sum_j p_j s_j |c_j - 8|, below 2^-11 * sum_j p_j s_j max(c_j, 8), taken as 2^-11 (C + 8 V / 15) with
    C = sum_j p_j s_j c_j and V the largest magnitude of a value's parts; fp32 queries: nothing beside V's terms;
  - a query is rounded to a multiple of its row's largest magnitude / 16256 (fp32: / 2080768), each
    coordinate by at most half of it, so a logit by a sum of D independent errors of deviation
    unit / sqrt(12) * |k_i| * scale: six deviations are 1.74 * unit * |k| * scale, N below is max |q_i| * |k| * scale:
    1.74 / 16256 N <= 2^-13 N (fp32: 2^-20 N);
  - the rest of a logit is three fp32 roundings below its sum of magnitudes M: 2^-22 M;
    a probability then is off by a factor e^{2 dz} with its normalization, an output by 2 dz V;
  - fp32 sums over n tokens: below n u of the magnitudes summed, in practice
    sqrt(n) u; taken as 2^-18 V, which covers n = 64 in the worst case and n = 4096 as it is;
  - probabilities below 2^-31 of the largest leave fp16: n * 2^-30 V;
  - bf16 queries with more than 32 rows per KV head: keys and values are rounded to fp16 over a power of
    two at or above the largest magnitude of a coordinate's parts, K and V at most, so below twice them: a step of
    2^-11 below 1. A value: half a step for its offset and for itself, 2^-11 * 2 V. A key's
    coordinates: independent errors, six deviations of step / sqrt(12) * |q| * scale are
    1.74 * 2^-10 * K |q| * scale; its offset alike in all, 2^-11 K |sum q| * scale.
"""

import math

import numpy as np
import pytest
import torch

from oracle import q4

pytestmark = pytest.mark.gpu


def say(msg):
    print(f"[gpu-case] {msg}", flush=True)


@pytest.fixture(scope="module")
def nk():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2608_04074_amd as nk
    nk._native.lib()
    return nk


def make_cache(nk, rng, seqs, H, D, block, extra_blocks=3, key_size=1.0, v_size=1.0):
    """A cache whose rows are random for the tokens of `seqs` and hold NaN scales
    everywhere else; block 0: contiguous with odd capacity."""
    B, top = len(seqs), max(max(seqs), 1)
    if block:
        bps = -(-top // block) + 1
        nblk = B * bps + extra_blocks
        table = rng.permutation(nblk)[: B * bps].astype(np.int32).reshape(B, bps)
        rows = block
    else:
        bps, rows, nblk, table = 1, top + 5, B, None
    kc, vc = (rng.integers(0, 256, (nblk, H, rows, D // 2)).astype(np.uint8) for _ in range(2))
    ksq, vsq = (np.full((nblk, H, rows, 2), 0x7FC0, dtype=np.uint16) for _ in range(2))
    where = []
    for b, S in enumerate(seqs):
        t = np.arange(S)
        page = b * bps + t // rows
        phys = table.reshape(-1)[page] if table is not None else page
        where.append((phys, t % rows))
        for sq, size in ((ksq, key_size), (vsq, v_size)):
            scale = size * 0.35 * np.exp(0.3 * rng.standard_normal((S, H)))
            offset = -7.5 * scale + 0.3 * size * rng.standard_normal((S, H))
            sq[phys, :, t % rows] = q4.to_bf16_bits(np.stack([scale, offset], -1))
    dev = lambda x: torch.as_tensor(x).cuda()  # noqa: E731
    sqdev = lambda x: torch.as_tensor(x.view(np.int16)).cuda().view(torch.bfloat16)  # noqa: E731
    lay = nk.CacheLayout(rows, bps, None if table is None else dev(table))
    cache = nk.Q4Cache(lay, dev(kc), dev(vc), sqdev(ksq), sqdev(vsq))
    return cache, (kc, vc, ksq, vsq, where)


def bound(o, coded, mags, norms, key_mags, key_sums, vmax, n, bf16, tiled):
    """The tolerance above, of outputs [m][G][D]."""
    V, M, N, K, Q = vmax[:, None, None], *(x[..., None] for x in (mags, norms, key_mags, key_sums))
    dz = 2.0 ** (-13 if bf16 else -20) * N + 2.0 ** -22 * M
    if tiled:
        dz = dz + 1.74 * 2.0 ** -10 * K + 2.0 ** -11 * Q
    return (np.abs(o) * 2.0 ** (-8 if bf16 else -24) + ((coded + 8 * V / 15) * 2.0 ** -11 if bf16 else 0) +
            (2 * dz + 2.0 ** -18 + n * 2.0 ** -30 + (2.0 ** -10 if tiled else 0)) * V)


def reference_and_bounds(host, q, seqs, q_lens, window, sinks, scale, bf16):
    kc, vc, ksq, vsq, where = host
    B, n, Hq, D = q.shape
    H = kc.shape[1]
    G = Hq // H
    out, tol = np.zeros(q.shape), np.zeros(q.shape)
    for b in range(B):
        m, S = q_lens[b], seqs[b]
        if m == 0:
            continue
        phys, row = where[b]
        for h in range(H):
            hs = slice(h * G, (h + 1) * G)
            k, ks, v, vs = (x[phys, h, row] for x in (kc, ksq, vc, vsq))
            o, *parts = q4.attend(q[b, :m, hs], q4.unpack_codes(k), q4.from_bf16_bits(ks), q4.unpack_codes(v),
                                             q4.from_bf16_bits(vs), S - m + np.arange(m), window,
                                             None if sinks is None else sinks[hs], scale)
            out[b, :m, hs] = o
            tol[b, :m, hs] = bound(o, *parts, S, bf16, bf16 and n * G > 32)
    return out, tol


def check(nk, seqs, n, Hq, H, D, dtype, block=0, window=0, sinks=None, q_lens=None, scale=0.0, seed=0, q_size=1.0,
          key_size=1.0, v_size=1.0):
    say(f"seqs={seqs} n={n} heads={Hq}/{H} D={D} {dtype} block={block} window={window} sinks={sinks is not None} q_lens={q_lens}")
    rng = np.random.default_rng(seed)
    B = len(seqs)
    cache, host = make_cache(nk, rng, seqs, H, D, block, key_size=key_size, v_size=v_size)
    q = torch.as_tensor(q_size * rng.standard_normal((B, n, Hq, D))).to(dtype).cuda()
    out = torch.full((B, n, Hq, D), 7.0, dtype=dtype, device="cuda")
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    sk = None if sinks is None else torch.as_tensor(sinks, dtype=torch.float32).cuda()
    got = nk.q4_attn(cache, q, i32(seqs), max(max(seqs), 1), q_lens=None if q_lens is None else i32(q_lens), window=window,
                     sinks=sk, softmax_scale=scale, out=out)
    torch.cuda.synchronize()
    lens = [n] * B if q_lens is None else q_lens
    ref, tol = reference_and_bounds(host, q.double().cpu().numpy(), seqs, lens, window, sinks,
                                    scale or 1 / math.sqrt(D), dtype == torch.bfloat16)
    g = got.double().cpu().numpy()
    for b in range(B):
        assert (g[b, lens[b]:] == 7.0).all(), "padding rows were written"
        assert np.isfinite(g[b, :lens[b]]).all()
        off = np.abs(g[b, :lens[b]] - ref[b, :lens[b]]) - tol[b, :lens[b]]
        assert off.size == 0 or off.max() <= 0, f"sequence {b}: {off.max():.3e} over the bound"
    return cache, q, got


BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", (BF, F32))
@pytest.mark.parametrize("D", (64, 128))
@pytest.mark.parametrize("seqs", ([1], [2, 0, 31], [32, 33], [127, 128, 129, 1], [1000, 613]))
def test_single_tokens(nk, seqs, D, dtype):
    check(nk, seqs, 1, 8, 2, D, dtype)


@pytest.mark.parametrize("Hq,H", ((1, 1), (3, 1), (8, 8), (10, 5), (16, 2), (20, 1), (40, 1)))
@pytest.mark.parametrize("D,dtype", ((64, F32), (128, BF)))
def test_head_layouts(nk, Hq, H, D, dtype):
    check(nk, [77, 300], 1, Hq, H, D, dtype, block=16)


@pytest.mark.parametrize("block", (1, 7, 16, 24, 64, 256))
@pytest.mark.parametrize("D,dtype", ((64, BF), (128, F32), (128, BF)))
def test_pages(nk, block, D, dtype):
    check(nk, [1, 100, 515], 1, 8, 2, D, dtype, block=block)
    check(nk, [515, 260], 40, 8, 2, D, dtype, block=block)


@pytest.mark.parametrize("n,Hq,H", ((2, 8, 2), (5, 6, 2), (7, 8, 2), (33, 4, 4), (40, 8, 2), (130, 2, 1)))
@pytest.mark.parametrize("D,dtype", ((64, F32), (64, BF), (128, F32), (128, BF)))
def test_several_queries(nk, n, Hq, H, D, dtype):
    check(nk, [n, 200, 3, 0, 611], n, Hq, H, D, dtype, block=16, q_lens=[n, n, min(n, 3), 0, max(1, n - 1)])


@pytest.mark.parametrize("n", (1, 4, 40))
@pytest.mark.parametrize("window", (1, 5, 33, 128))
@pytest.mark.parametrize("D,dtype", ((64, BF), (128, F32), (128, BF)))
def test_windows_and_sinks(nk, n, window, D, dtype):
    rng = np.random.default_rng(window)
    sinks = 2 * rng.standard_normal(8)
    sinks[:3] = -np.inf, 60.0, -200.0
    check(nk, [n, 700, 129], n, 8, 2, D, dtype, block=16, window=window, sinks=sinks)
    check(nk, [700, n], n, 8, 2, D, dtype, window=window)


@pytest.mark.parametrize("dtype", (BF, F32))
def test_more_queries_than_tokens(nk, dtype):
    """Queries at negative positions attend nothing: zeros, with a sink too."""
    _, _, got = check(nk, [3, 0], 6, 8, 2, 128, dtype)
    assert not got[0, :3].any() and not got[1].any()
    _, _, got = check(nk, [3, 0], 6, 8, 2, 128, dtype, sinks=np.zeros(8))
    assert not got[0, :3].any() and not got[1].any()


@pytest.mark.parametrize("dtype", (BF, F32))
@pytest.mark.parametrize("seq,n,window", ((20000, 1, 0), (20000, 1, 3000), (9001, 33, 0)))
def test_long(nk, seq, n, window, dtype):
    check(nk, [seq, seq // 3], n, 4, 1, 128, dtype, block=16, window=window)


@pytest.mark.parametrize("q_size,key_size,v_size", ((1e-12, 1.0, 1e-9), (1e15, 1e-15, 1e9), (1e-3, 1e3, 1.0), (1.0, 1e-20, 1e-20)))
@pytest.mark.parametrize("dtype", (BF, F32))
def test_magnitudes(nk, q_size, key_size, v_size, dtype):
    check(nk, [300, 40], 2, 8, 2, 64, dtype, q_size=q_size, key_size=key_size, v_size=v_size)


def test_sharp_logits(nk):
    """Logits in the hundreds: the running reference moves many times, one token takes all."""
    check(nk, [2000], 1, 8, 2, 128, F32, q_size=40.0)
    check(nk, [2000], 9, 8, 2, 128, BF, q_size=40.0)


def test_scales_that_grow(nk):
    """Value scales that grow by orders of magnitude along the cache, and constant rows (scale 0)."""
    rng = np.random.default_rng(5)
    seqs = [700]
    cache, host = make_cache(nk, rng, seqs, 2, 128, 16)
    kc, vc, ksq, vsq, (where,) = host
    phys, row = where
    size = 10.0 ** np.linspace(-12, 4, 700)[:, None]
    zero = np.arange(700)[:, None] % 5 == 0
    vsq[phys, :, row] = q4.to_bf16_bits(np.stack([np.where(zero, 0, 0.3 * size) * np.ones((1, 2)), -2 * size * np.ones((1, 2))], -1))
    cache.v_sq.copy_(torch.as_tensor(vsq.view(np.int16)).cuda().view(torch.bfloat16))
    for dtype in (BF, F32):
        q = torch.as_tensor(rng.standard_normal((1, 1, 8, 128))).to(dtype).cuda()
        out = nk.q4_attn(cache, q, torch.tensor([700], dtype=torch.int32, device="cuda"), 700)
        ref, tol = reference_and_bounds(host, q.double().cpu().numpy(), seqs, [1], 0, None, 1 / math.sqrt(128), dtype == BF)
        assert (np.abs(out.double().cpu().numpy() - ref) <= tol).all()


def test_blocks_that_hold_nothing(nk):
    """Table entries outside the pool are not attended (and not read)."""
    rng = np.random.default_rng(6)
    seqs = [200, 90]
    for n in (1, 40):
        cache, host = make_cache(nk, rng, seqs, 2, 64, 16)
        kc, vc, ksq, vsq, where = host
        table = cache.layout.block_table.cpu().numpy().copy()
        table[0, 2], table[0, 5], table[1, 0] = -1, cache.num_blocks, 2 ** 31 - 1
        cache.layout.block_table.copy_(torch.as_tensor(table))
        q = torch.as_tensor(rng.standard_normal((2, n, 8, 64))).to(BF).cuda()
        got = nk.q4_attn(cache, q, torch.tensor(seqs, dtype=torch.int32, device="cuda"), 200).double().cpu().numpy()
        for b, gone in ((0, (2, 5)), (1, (0,))):
            keep = ~np.isin(np.arange(seqs[b]) // 16, gone)
            at = np.flatnonzero(keep)
            for h in range(2):
                k, ks, v, vs = (x[where[b][0], h, where[b][1]][keep] for x in (kc, ksq, vc, vsq))
                for i in range(n):
                    m = int((at <= seqs[b] - n + i).sum())
                    o, *parts = q4.attend(q[b, i:i + 1, 4 * h:4 * h + 4].double().cpu().numpy(), q4.unpack_codes(k),
                                                     q4.from_bf16_bits(ks), q4.unpack_codes(v), q4.from_bf16_bits(vs), np.array([m - 1]))
                    tol = bound(o, *parts, 200, True, n * 4 > 32)
                    assert (np.abs(got[b, i:i + 1, 4 * h:4 * h + 4] - o) <= tol).all(), (b, h, i)


def test_nan_rows_reach_only_what_attends_them(nk):
    rng = np.random.default_rng(7)
    cache, host = make_cache(nk, rng, [100, 100], 1, 128, 16)
    where = host[4][1]
    cache.v_sq[int(where[0][60]), 0, int(where[1][60])] = float("nan")
    q = torch.as_tensor(rng.standard_normal((2, 100, 2, 128))).to(BF).cuda()
    seq = torch.tensor([100, 100], dtype=torch.int32, device="cuda")
    for window in (0, 20):
        out = nk.q4_attn(cache, q, seq, 100, window=window)
        bad = torch.isnan(out).any(-1).any(-1).cpu().numpy()
        sees = (np.arange(100) >= 60) & ((window == 0) | (np.arange(100) < 60 + window))
        assert (bad[1] == sees).all() and not bad[0].any()
    q[0, 3, 1, 5] = float("nan")
    q[0, 4, 0, 5] = float("inf")
    out = nk.q4_attn(cache, q, seq, 100)
    bad = torch.isnan(out).any(-1).cpu().numpy()[0]
    assert bad[3].tolist() == [False, True] and bad[4].tolist() == [True, False] and bad.sum() == 2


def test_long_cache_offsets(nk):
    """A pool whose byte offsets pass 32 bits: the blocks of one sequence lie at its two ends."""
    H, D, block = 8, 128, 16
    nblk = (1 << 32) // (H * block * D // 2) + 64           # a little over 4 GiB of codes per side
    lay_table = torch.tensor([[nblk - 1, 0, nblk - 40, 7]], dtype=torch.int32, device="cuda")
    codes = lambda: torch.empty((nblk, H, block, D // 2), dtype=torch.uint8, device="cuda")  # noqa: E731
    sqs = lambda: torch.zeros((nblk, H, block, 2), dtype=torch.bfloat16, device="cuda")  # noqa: E731
    big = nk.Q4Cache(nk.CacheLayout(block, 4, lay_table), codes(), codes(), sqs(), sqs())
    rng = np.random.default_rng(8)
    small, _ = make_cache(nk, rng, [64], H, D, 16, extra_blocks=0)
    order = small.layout.block_table[0, :4].long()
    for x, y in zip(big.tensors[1:], small.tensors[1:]):
        x[lay_table[0].long()] = y[order]
    q = torch.as_tensor(rng.standard_normal((1, 2, 32, D))).to(BF).cuda()
    seq = torch.tensor([63], dtype=torch.int32, device="cuda")
    assert torch.equal(nk.q4_attn(big, q, seq, 64), nk.q4_attn(small, q, seq, 64))


@pytest.mark.parametrize("n", (1, 40))
def test_lengths_past_the_bound_are_cut(nk, n):
    """A length above max_seq_len is taken as max_seq_len, a negative one as 0."""
    rng = np.random.default_rng(9)
    cache, _ = make_cache(nk, rng, [200, 200], 2, 128, 16)
    q = torch.as_tensor(rng.standard_normal((2, n, 8, 128))).to(BF).cuda()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    got = nk.q4_attn(cache, q, i32([10 ** 9, -5]), 150)
    assert torch.equal(got[0], nk.q4_attn(cache, q, i32([150, 1]), 150)[0]) and not got[1].any()


@pytest.mark.parametrize("n,Hq,seqs", ((1, 8, [3000, 100]), (5, 8, [1500, 2000]), (40, 8, [700, 900])))
def test_workspace_reuse_streams_and_graphs(nk, n, Hq, seqs):
    """One workspace serves calls of several shapes, a side stream, and a captured call's replays."""
    rng = np.random.default_rng(10)
    cache, _ = make_cache(nk, rng, seqs, 2, 128, 16)
    B, top = len(seqs), max(seqs)
    seq = torch.tensor(seqs, dtype=torch.int32, device="cuda")
    q = torch.as_tensor(rng.standard_normal((B, n, Hq, 128))).to(BF).cuda()
    ref = nk.q4_attn(cache, q, seq, top)
    need = max(nk.q4_attn_workspace_bytes(cache, B, m, Hq, top) for m in (1, 2, 7, n))
    ws = torch.zeros(max(need, 256), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)
    for m in (1, 2, 7):
        qq = q[:, :1].expand(-1, m, -1, -1).contiguous()
        nk.q4_attn(cache, qq, seq, top, workspace=ws)
        assert torch.equal(nk.q4_attn(cache, q, seq, top, workspace=ws, out=out), ref)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = nk.q4_attn(cache, q, seq, top, stream=side)
    junk = torch.full((1 << 22,), 3.0, device="cuda")
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, ref) and junk[0] == 3
    call = nk.prepare_q4_attn(cache, q, seq, top, out, ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        nk.prepare_q4_attn(cache, q, seq, top, out, ws)()
    for r in range(3):
        q.copy_(torch.as_tensor(rng.standard_normal(q.shape)).to(BF))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        replayed = out.clone()
        call()
        torch.cuda.synchronize()
        assert torch.equal(replayed, out) and out.any(), f"replay {r}"


def test_repeatable(nk):
    """Partials are merged in the splits' order, whichever arrives last."""
    rng = np.random.default_rng(11)
    cache, _ = make_cache(nk, rng, [20000], 2, 128, 16)
    q = torch.as_tensor(rng.standard_normal((1, 1, 8, 128))).to(F32).cuda()
    seq = torch.tensor([20000], dtype=torch.int32, device="cuda")
    ref = nk.q4_attn(cache, q, seq, 20000)
    for _ in range(20):
        assert torch.equal(nk.q4_attn(cache, q, seq, 20000), ref)


def test_two_graphs_share_a_workspace(nk):
    """Graphs of calls of different shapes (whole rows, tiles of rows) on one workspace, replayed in turn with eager
    calls between them."""
    rng = np.random.default_rng(12)
    cache, _ = make_cache(nk, rng, [3000, 2500], 2, 64, 16)
    seq = torch.tensor([3000, 2500], dtype=torch.int32, device="cuda")
    qs = [torch.as_tensor(rng.standard_normal((2, n, 16, 64))).to(dt).cuda() for n, dt in ((1, BF), (3, F32), (20, BF), (9, F32))]
    ws = torch.zeros(max(nk.q4_attn_workspace_bytes(cache, 2, q.shape[1], 16, 3000) for q in qs), dtype=torch.uint8, device="cuda")
    outs = [torch.empty_like(q) for q in qs]
    graphs = []
    for q, out in zip(qs, outs):
        nk.q4_attn(cache, q, seq, 3000, out=out, workspace=ws)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            nk.q4_attn(cache, q, seq, 3000, out=out, workspace=ws)
        graphs.append(g)
    for r in range(3):
        for q in qs:
            q.copy_(torch.as_tensor(rng.standard_normal(tuple(q.shape))).to(q.dtype))
        for i in rng.permutation(4):
            outs[i].zero_()
            graphs[i].replay()
            torch.cuda.synchronize()
            assert torch.equal(outs[i], nk.q4_attn(cache, qs[i], seq, 3000)), f"round {r}, graph {i}"
            nk.q4_attn(cache, qs[0], seq, 3000, workspace=ws)


def test_refusals(nk):
    rng = np.random.default_rng(13)
    cache, _ = make_cache(nk, rng, [100], 2, 64, 16)
    q = torch.zeros((1, 3, 8, 64), dtype=BF, device="cuda")
    seq = torch.tensor([100], dtype=torch.int32, device="cuda")
    cases = [
        (ValueError, dict(q=q[0])), (ValueError, dict(q=q[..., :32])), (TypeError, dict(q=q.half())), (ValueError, dict(q=q.transpose(1, 2))),
        (TypeError, dict(seq_lens=seq.long())), (ValueError, dict(seq_lens=seq.cpu())), (ValueError, dict(seq_lens=seq.expand(2).contiguous())),
        (ValueError, dict(q=q.expand(2, -1, -1, -1).contiguous(), seq_lens=seq.expand(2).contiguous())),   # the table holds one sequence
        (TypeError, dict(out=q.float())), (ValueError, dict(out=q[:, :2].contiguous())), (ValueError, dict(sinks=torch.zeros(7, device="cuda"))),
        (ValueError, dict(q_lens=seq.expand(2).contiguous())), (nk.NovaKVError, dict(max_seq_len=10 ** 6)), (nk.NovaKVError, dict(window=-1)),
        (nk.NovaKVError, dict(softmax_scale=-1.0)), (TypeError, dict(workspace=torch.zeros(4, device="cuda"))),
        (nk.NovaKVError, dict(q=torch.zeros(q.numel() + 4, dtype=BF, device="cuda")[4:].view(q.shape))),   # 8-byte aligned
        (nk.NovaKVError, dict(q=torch.zeros((1, 3, 7, 64), dtype=BF, device="cuda"))),                     # 7 query heads, 2 KV heads
    ]
    for error, change in cases:
        args = dict(q=q, seq_lens=seq, max_seq_len=100)
        args.update(change)
        with pytest.raises(error):
            nk.q4_attn(cache, **args)
    assert nk.q4_attn(cache, q[:, :0], seq, 100).shape == (1, 0, 8, 64)
