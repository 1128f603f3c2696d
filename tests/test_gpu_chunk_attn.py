"""nova_kv_chunk_attn against the fp64 oracle, at the lengths, head counts, pages, formats and masks
where it can go wrong.

Tolerance of an output value, from the roundings on its way (u = 2^-24). U is the largest norm of an
attended value's coefficients (for the scalar arm, of its two parts): R_V's rows have norm 1, so what is
off by x U in the coefficients is off by at most x U in a coordinate.
  - its own rounding: half a step, |ref| 2^-8 (bf16) or 2^-24;
  - bf16 queries: probabilities (times scales) rounded to fp16, half a step each: 2^-11 U; the queries'
    coordinates q' = q R_K^-T rounded to fp16, a logit by 2^-11 M, M the largest sum of |q'_i| |r_i| times the
    scale; an output then by 2 dz U (a weight is off by e^{dz}, the sum of weights by as much);
  - fp32 queries: two parts each, 2^-22 of the same; with the fp32 sums of D products on the cores, the
    shift q . k_bar and the exponent's rounding, all below 2^-20 of the logit's sum of magnitudes,
    that of k_bar and of exact band rows among them;
  - fp32 sums over n tokens: below n u of the magnitudes summed, in practice sqrt(n) u, and R_V in two
    parts, 3 * 2^-22: taken as 2^-18 U together;
  - probabilities below 2^-30 of the largest leave fp16: n 2^-30 U.
"""

import numpy as np
import pytest
import torch

from chunk_cases import FORMATS, Cache

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def say(msg):
    print(f"[gpu-case] {msg}", flush=True)


@pytest.fixture(scope="module")
def nk():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2608_04074_amd as nk
    nk._native.lib()
    return nk


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def queries(rng, shape, dtype, size=1.0):
    return torch.as_tensor(size * rng.standard_normal(shape)).to(dtype).cuda()


def call(c, q, **kw):
    return c.nk.chunk_attn(c.params, c.layout, q, c.k_codes, c.v_codes, c.seq_lens, c.top, **c.more, **kw)


def check(nk, seqs, n, Hq, H, D, dtype, block=0, fmt="plain", window=0, sinks=None, q_lens=None, scale=0.0, seed=0, q_size=2.0, **sizes):
    say(f"seqs={seqs} n={n} heads={Hq}/{H} D={D} {dtype} block={block} {fmt} window={window} sinks={sinks is not None} q_lens={q_lens}")
    c = Cache(nk, seed, seqs, H, D, block, fmt, **sizes)
    B = len(seqs)
    q = queries(c.rng, (B, n, Hq, D), dtype, q_size)
    out = torch.full((B, n, Hq, D), 7.0, dtype=dtype, device="cuda")
    got = call(c, q, q_lens=None if q_lens is None else i32(q_lens), window=window, softmax_scale=scale, out=out,
               sinks=None if sinks is None else torch.as_tensor(sinks, dtype=torch.float32).cuda())
    torch.cuda.synchronize()
    lens = [n] * B if q_lens is None else q_lens
    ref, tol = c.attend(q.double().cpu().numpy(), lens, window, sinks, scale, dtype == BF)
    g = got.double().cpu().numpy()
    for b in range(B):
        assert (g[b, lens[b]:] == 7.0).all(), "padding rows were written"
        assert np.isfinite(g[b, :lens[b]]).all()
        off = np.abs(g[b, :lens[b]] - ref[b, :lens[b]]) - tol[b, :lens[b]]
        assert off.size == 0 or off.max() <= 0, f"sequence {b}: {off.max():.3e} over the bound"
    return c, q, got


@pytest.mark.parametrize("dtype", (BF, F32))
@pytest.mark.parametrize("D", (64, 128))
@pytest.mark.parametrize("seqs", ([1], [2, 0, 31], [32, 33], [127, 128, 129, 1], [1000, 613]))
def test_single_tokens(nk, seqs, D, dtype):
    check(nk, seqs, 1, 8, 2, D, dtype)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("D,dtype", ((64, BF), (64, F32), (128, BF), (128, F32)))
def test_formats(nk, fmt, D, dtype):
    check(nk, [300, 77, 5, 0, 41], 3, 8, 2, D, dtype, block=16, fmt=fmt, q_lens=[3, 2, 3, 0, 1])
    check(nk, [700, 250], 40, 8, 2, D, dtype, fmt=fmt, q_lens=[40, 33])
    check(nk, [130], 1, 4, 1, D, dtype, block=8, fmt=fmt)


@pytest.mark.parametrize("Hq,H", ((1, 1), (3, 1), (8, 8), (10, 5), (16, 2), (20, 1), (40, 1)))
@pytest.mark.parametrize("D,dtype", ((64, F32), (128, BF)))
def test_head_layouts(nk, Hq, H, D, dtype):
    check(nk, [77, 300], 1, Hq, H, D, dtype, block=16)


@pytest.mark.parametrize("block", (1, 7, 16, 24, 64, 256))
@pytest.mark.parametrize("D,dtype", ((64, BF), (128, F32), (128, BF)))
def test_pages(nk, block, D, dtype):
    check(nk, [1, 100, 515], 1, 8, 2, D, dtype, block=block)
    check(nk, [515, 260], 40, 8, 2, D, dtype, block=block, fmt="scaled")


@pytest.mark.parametrize("n,Hq,H", ((2, 8, 2), (5, 6, 2), (7, 8, 2), (33, 4, 4), (40, 8, 2), (130, 2, 1), (67, 8, 1)))
@pytest.mark.parametrize("D,dtype", ((64, F32), (64, BF), (128, F32), (128, BF)))
def test_several_queries(nk, n, Hq, H, D, dtype):
    check(nk, [n, 200, 3, 0, 611], n, Hq, H, D, dtype, block=16, q_lens=[n, n, min(n, 3), 0, max(1, n - 1)])


@pytest.mark.parametrize("n", (1, 4, 40))
@pytest.mark.parametrize("window", (1, 5, 33, 128))
@pytest.mark.parametrize("D,dtype,fmt", ((64, BF, "plain"), (128, F32, "deployed"), (128, BF, "band")))
def test_windows_and_sinks(nk, n, window, D, dtype, fmt):
    sinks = 2 * np.random.default_rng(window).standard_normal(8)
    sinks[:3] = -np.inf, 60.0, -200.0
    check(nk, [n, 700, 129], n, 8, 2, D, dtype, block=16, fmt=fmt, window=window, sinks=sinks)
    check(nk, [700, n], n, 8, 2, D, dtype, fmt=fmt, window=window)


@pytest.mark.parametrize("fmt", ("plain", "band"))
@pytest.mark.parametrize("dtype", (BF, F32))
def test_more_queries_than_tokens(nk, dtype, fmt):
    """Queries at negative positions attend nothing: zeros, with a sink too."""
    for n, sinks in ((6, None), (6, np.zeros(8)), (50, np.zeros(8))):
        _, _, got = check(nk, [3, 0], n, 8, 2, 128, dtype, fmt=fmt, sinks=sinks)
        assert not got[0, :n - 3].any() and not got[1].any()


@pytest.mark.parametrize("dtype", (BF, F32))
@pytest.mark.parametrize("seq,n,window,fmt", ((20000, 1, 0, "plain"), (20000, 1, 3000, "deployed"), (9001, 33, 0, "band"), (6000, 70, 0, "sq")))
def test_long(nk, seq, n, window, fmt, dtype):
    check(nk, [seq, seq // 3], n, 4, 1, 128, dtype, block=16, fmt=fmt, window=window)


@pytest.mark.parametrize("n", (2, 20))
@pytest.mark.parametrize("q_size,sizes,fmt", ((1e-12, {}, "plain"), (1e4, {"k_size": 1e-4, "kbar_size": 1e-4}, "plain"),
                                               (1e12, {"kbar_size": 0.0}, "tiny"), (2.0, {"v_size": 1e-15}, "sq"),
                                               (2.0, {"v_size": 1e12}, "sq"), (0.5, {"kbar_size": 30.0}, "band")))
@pytest.mark.parametrize("dtype", (BF, F32))
def test_magnitudes(nk, q_size, sizes, fmt, n, dtype):
    if fmt == "tiny":  # queries and scales of a softmax far apart whose products are ordinary
        check(nk, [300, 40], n, 8, 2, 64, dtype, q_size=q_size, scale=1e-13, **sizes)
    else:
        check(nk, [300, 40], n, 8, 2, 64, dtype, fmt=fmt, q_size=q_size, **sizes)


@pytest.mark.parametrize("dtype", (BF, F32))
def test_sharp_logits(nk, dtype):
    """Logits in the hundreds: the running reference moves many times, one token takes all."""
    check(nk, [2000], 1, 8, 2, 128, dtype, q_size=40.0, fmt="scaled")
    check(nk, [2000], 9, 8, 2, 128, dtype, q_size=40.0)


@pytest.mark.parametrize("dtype", (BF, F32))
@pytest.mark.parametrize("n", (1, 20))
def test_grids_that_grow(nk, n, dtype):
    """The scalar arm's scales growing by orders of magnitude along the cache, and constant rows (scale 0)."""
    c = Cache(nk, 5, [700], 2, 128, 16, "sq")
    from oracle.q4 import to_bf16_bits
    phys, row = c.where[0]
    size = 10.0 ** np.linspace(-12, 4, 700)[:, None]
    zero = np.arange(700)[:, None] % 5 == 0
    c.vs[phys, :, row] = to_bf16_bits(np.stack([np.where(zero, 0, 0.3 * size) * np.ones((1, 2)), -2 * size * np.ones((1, 2))], -1))
    c.v_sq.copy_(torch.as_tensor(c.vs.view(np.int16)).cuda().view(torch.bfloat16))
    q = queries(c.rng, (1, n, 8, 128), dtype)
    ref, tol = c.attend(q.double().cpu().numpy(), [n], bf16=dtype == BF)
    assert (np.abs(call(c, q).double().cpu().numpy() - ref) <= tol).all()


@pytest.mark.parametrize("n", (1, 40))
def test_released_blocks_are_not_looked_up(nk, n):
    """Table entries in front of a window, and of blocks whose positions are all the band's, may hold anything."""
    c = Cache(nk, 6, [700, 400], 2, 64, 16, "band")
    ref = [call(c, q, window=w) for q, w in ((queries(np.random.default_rng(1), (2, n, 8, 64), BF), w) for w in (90, 0))]
    table = c.layout.block_table
    kept = table.clone()
    for w, r in zip((90, 0), ref):
        table.copy_(kept)
        for b, S in enumerate(c.seqs):
            low = max(0, S - n + 1 - w) if w else 5
            table[b, :(max(low, 5) // 16)] = -5
            table[b, -(-(S - 40) // 16):] = 2 ** 30
        assert torch.equal(call(c, queries(np.random.default_rng(1), (2, n, 8, 64), BF), window=w), r)


def test_nan_rows_reach_only_what_attends_them(nk):
    n = 100
    for fmt, D in (("scaled", 128), ("scaled", 64), ("band", 128)):
        say(f"nan rows {fmt} {D}")
        c = Cache(nk, 7, [n, n], 1, D, 16, fmt)
        at = 60
        spots = []
        if fmt == "scaled":
            phys, row = (int(x[at]) for x in c.where[1])
            spots = [(c.v_sq, (phys, 0, row)), (c.k_scales, (phys, 0, row))]
        else:
            at = 80
            slot = c.band.n_sink + at % c.band.n_rec
            spots = [(c.band.k, (1, 0, slot, 3)), (c.band.v, (1, 0, slot, 3))]
        for m in (n, 7):
            q = queries(np.random.default_rng(2), (2, m, 2, D), BF)
            for t, where in spots:
                for bad_value in (float("nan"), float("inf")):
                    old = t[where].clone()
                    t[where] = bad_value
                    for window in (0, 20):
                        out = call(c, q, window=window)
                        bad = torch.isnan(out).any(-1).any(-1) | torch.isinf(out).any(-1).any(-1)
                        pos = np.arange(n - m, n)
                        sees = (pos >= at) & ((window == 0) | (pos < at + window))
                        got = bad.cpu().numpy()
                        assert not got[0].any() and not got[1][~sees].any(), (fmt, m, window)
                        if bad_value != bad_value:
                            assert got[1][sees].all(), (fmt, m, window)
                    t[where] = old


def test_nan_queries(nk):
    for fmt in ("plain", "band"):
        for n in (5, 40):
            c = Cache(nk, 8, [n, 2], 1, 128, 16, fmt)
            q = queries(c.rng, (2, n, 2, 128), BF)
            clean = call(c, q)
            q[0, 3, 1, 5], q[0, 4, 0, 70] = float("nan"), float("inf")
            q[1, 0, 0, 0] = float("nan")           # attends nothing: position 2 - n
            out = call(c, q)
            bad = torch.isnan(out).any(-1).cpu().numpy()
            assert bad[0, 3].tolist() == [False, True] and bad[0, 4].tolist() == [True, False] and bad.sum() == 2
            assert torch.equal(out[torch.as_tensor(~bad)], clean[torch.as_tensor(~bad)])


@pytest.mark.parametrize("n", (2, 20))
def test_long_cache_offsets(nk, n):
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
    q = queries(small.rng, (1, n, 32, D), BF)
    got = nk.chunk_attn(small.params, nk.CacheLayout(block, 4, ends), q, big[0], big[1], small.seq_lens, 63, k_scales=big[2], v_sq=big[3])
    assert torch.equal(got, call(small, q))


@pytest.mark.parametrize("n", (1, 40))
def test_lengths_past_the_bound_are_cut(nk, n):
    """A length above max_seq_len is taken as max_seq_len, a negative one as 0."""
    c = Cache(nk, 10, [200, 200], 2, 128, 16)
    q = queries(c.rng, (2, n, 8, 128), BF)
    run = lambda lens: nk.chunk_attn(c.params, c.layout, q, c.k_codes, c.v_codes, i32(lens), 150)  # noqa: E731
    got = run([10 ** 9, -5])
    assert torch.equal(got[0], run([150, 1])[0]) and not got[1].any()


@pytest.mark.parametrize("fmt", ("plain", "deployed"))
def test_agrees_with_the_single_token_call(nk, fmt):
    c = Cache(nk, 11, [900, 333, 0], 2, 128, 16, fmt)
    q = queries(c.rng, (3, 1, 8, 128), F32)
    one = nk.decode_attn(c.params, c.layout, q[:, 0], c.k_codes, c.v_codes, c.seq_lens, c.top, **c.more)
    ref, tol = c.attend(q.double().cpu().numpy(), [1, 1, 1], bf16=False)
    got = call(c, q)
    # the single token's tables and probabilities are fp16: 2e-3 of the row's norm
    near = 2e-3 * one.norm(dim=-1, keepdim=True) + torch.as_tensor(tol[:, 0]).cuda()
    assert ((got[:, 0] - one).abs() <= near).all()


@pytest.mark.parametrize("n,seqs,fmt", ((1, [3000, 100], "plain"), (5, [1500, 2000], "deployed"), (40, [700, 900], "band")))
def test_workspace_reuse_streams_and_graphs(nk, n, seqs, fmt):
    """One workspace serves calls of several shapes, a side stream, and a captured call's replays."""
    c = Cache(nk, 12, seqs, 2, 128, 16, fmt)
    rng, B, top = c.rng, len(seqs), max(seqs)
    q = queries(rng, (B, n, 8, 128), BF)
    ref = call(c, q)
    need = max(nk.chunk_attn_workspace_bytes(c.params, B, m, 8, top) for m in (1, 2, 7, n))
    ws = torch.zeros(max(need, 256), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)
    for m in (1, 2, 7):
        call(c, q[:, :1].expand(-1, m, -1, -1).contiguous(), workspace=ws)
        assert torch.equal(call(c, q, workspace=ws, out=out), ref)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = call(c, q, stream=side)
    junk = torch.full((1 << 22,), 3.0, device="cuda")
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, ref) and junk[0] == 3
    again = lambda: nk.prepare_chunk_attn(c.params, c.layout, q, c.k_codes, c.v_codes, c.seq_lens, top, out, ws, **c.more)  # noqa: E731
    eager = again()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        again()()
    for r in range(3):
        q.copy_(queries(rng, tuple(q.shape), BF))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        replayed = out.clone()
        eager()
        torch.cuda.synchronize()
        assert torch.equal(replayed, out) and out.any(), f"replay {r}"


def test_repeatable(nk):
    """Partials are merged in the splits' order, whichever arrives last."""
    for n in (1, 30):
        c = Cache(nk, 13, [9000], 2, 128, 16)
        q = queries(c.rng, (1, n, 8, 128), F32)
        ref = call(c, q)
        for _ in range(10):
            assert torch.equal(call(c, q), ref)


def test_two_graphs_share_a_workspace(nk):
    """Graphs of calls of different shapes on one workspace, replayed in turn with eager calls between them."""
    c = Cache(nk, 14, [3000, 2500], 2, 64, 16, "key_scale")
    qs = [queries(c.rng, (2, n, 16, 64), dt) for n, dt in ((1, BF), (3, F32), (20, BF), (9, F32))]
    ws = torch.zeros(max(nk.chunk_attn_workspace_bytes(c.params, 2, q.shape[1], 16, 3000) for q in qs), dtype=torch.uint8, device="cuda")
    outs = [torch.empty_like(q) for q in qs]
    graphs = []
    for q, out in zip(qs, outs):
        call(c, q, out=out, workspace=ws)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(c, q, out=out, workspace=ws)
        graphs.append(g)
    for r in range(3):
        for q in qs:
            q.copy_(queries(c.rng, tuple(q.shape), q.dtype))
        for i in c.rng.permutation(4):
            outs[i].zero_()
            graphs[i].replay()
            torch.cuda.synchronize()
            assert torch.equal(outs[i], call(c, qs[i])), f"round {r}, graph {i}"
            call(c, qs[0], workspace=ws)


def test_refusals(nk):
    c = Cache(nk, 15, [100], 2, 64, 16, "scaled")
    q = torch.zeros((1, 3, 8, 64), dtype=BF, device="cuda")
    seq, codes = c.seq_lens, c.k_codes
    cases = [
        (ValueError, dict(q=q[0])), (ValueError, dict(q=q[..., :32])), (TypeError, dict(q=q.half())), (ValueError, dict(q=q.transpose(1, 2))),
        (TypeError, dict(seq_lens=seq.long())), (ValueError, dict(seq_lens=seq.cpu())), (ValueError, dict(seq_lens=seq.expand(2).contiguous())),
        (ValueError, dict(q=q.expand(2, -1, -1, -1).contiguous(), seq_lens=seq.expand(2).contiguous())),   # the table holds one sequence
        (TypeError, dict(out=q.float())), (ValueError, dict(out=q[:, :2].contiguous())), (ValueError, dict(sinks=torch.zeros(7, device="cuda"))),
        (ValueError, dict(q_lens=seq.expand(2).contiguous())), (nk.NovaKVError, dict(max_seq_len=10 ** 6)), (nk.NovaKVError, dict(window=-1)),
        (nk.NovaKVError, dict(softmax_scale=-1.0)), (TypeError, dict(workspace=torch.zeros(4, device="cuda"))),
        (nk.NovaKVError, dict(q=torch.zeros(q.numel() + 4, dtype=BF, device="cuda")[4:].view(q.shape))),   # 8-byte aligned
        (nk.NovaKVError, dict(q=torch.zeros((1, 3, 7, 64), dtype=BF, device="cuda"))),                     # 7 query heads, 2 KV heads
        (ValueError, dict(k_codes=codes[:, :1].contiguous())), (ValueError, dict(v_codes=codes[..., :8].contiguous())),
        (ValueError, dict(k_scales=None)), (ValueError, dict(v_sq=None)), (TypeError, dict(k_codes=codes.int())),
    ]
    for error, change in cases:
        args = dict(q=q, k_codes=codes, v_codes=c.v_codes, seq_lens=seq, max_seq_len=100, k_scales=c.k_scales, v_sq=c.v_sq)
        args.update(change)
        with pytest.raises(error):
            nk.chunk_attn(c.params, c.layout, **args)
    assert nk.chunk_attn(c.params, c.layout, q[:, :0], codes, c.v_codes, seq, 100, k_scales=c.k_scales, v_sq=c.v_sq).shape == (1, 0, 8, 64)
