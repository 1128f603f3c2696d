"""nova_kv_rotate_qkv and nova_kv_q4_append against the fp64 oracle.

Tolerance of a rotated value y_a' = y_a c - y_b s, u = 2^-24 and m the largest
|y| of its row: the norm is a sum of D squares (in lanes of 8, then a tree: at most 12
roundings), a division, a root and two products, below 16 u; the rotation three
roundings of terms of at most m each: below 40 u m, taken as 2^-18 m.  Then half a
step of the output's type, 2^-8 or 2^-24 of the value.  Codes, scales and offsets
must be the oracle's, except that a quotient within 1e-9 of a border may fall
on either side (both are fp64, in another order of sums)."""

import numpy as np
import pytest
import torch

from oracle import q4

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


def heads_of(rng, B, n, Hq, H, D, dtype, fused, offset=0):
    """q, k, v: slices of one projection (starting `offset` elements into it), or tensors of their own."""
    w = (Hq + 2 * H) * D
    x = rng.standard_normal((B, n, w)) * np.exp(0.5 * rng.standard_normal(w)) + 0.3 * rng.standard_normal(w)
    if fused:
        buf = torch.zeros((B, n, w + offset + (3 if offset % 8 else 0)), dtype=dtype, device="cuda")
        buf[..., offset:offset + w] = torch.as_tensor(x).to(dtype)
        x = buf[..., offset:offset + w].unflatten(-1, (Hq + 2 * H, D))
        return x[:, :, :Hq], x[:, :, Hq:Hq + H], x[:, :, Hq + H:]
    x = torch.as_tensor(x).to(dtype).cuda().unflatten(-1, (Hq + 2 * H, D))
    return tuple(t.contiguous() for t in (x[:, :, :Hq], x[:, :, Hq:Hq + H], x[:, :, Hq + H:]))


def rotary_of(nk, rng, Hq, H, D, rotary, interleaved, norm, P=700):
    table = nk.Rotary.table(P, rotary, 1e4) if rotary else None
    w = lambda h: None if norm is None else torch.as_tensor(1 + 0.3 * rng.standard_normal((D,) if norm == "shared" else (h, D))).float().cuda()  # noqa: E731
    return nk.Rotary(Hq, H, D, cos_sin=table, interleaved=interleaved, q_norm=w(Hq), k_norm=w(H), eps=1e-5)


def oracle_heads(rot, x, weight, start):
    pos = np.asarray(start)[:, None] + np.arange(x.shape[1])
    table = None if rot.cos_sin is None else rot.cos_sin.cpu().numpy()
    return q4.norm_rotate(x.double().cpu().numpy(), None if weight is None else weight.double().cpu().numpy(), rot.eps, table,
                          rot.interleaved, np.clip(pos, 0, None if table is None else len(table) - 1))


def assert_close(got, ref, dtype, rows):
    m = np.abs(ref).max(-1, keepdims=True)
    off = np.abs(got.double().cpu().numpy() - ref) - np.abs(ref) * 2.0 ** (-8 if dtype == BF else -24) - m * 2.0 ** -18
    assert off[rows].size == 0 or off[rows].max() <= 0, f"{off[rows].max():.3e} over the bound"


SHAPES = [  # B, n, Hq, H, D, rotary, interleaved, norm, fused, offset of the projection's rows
    (1, 1, 32, 8, 128, 128, False, "shared", True, 0),
    (3, 5, 4, 2, 64, 64, False, "shared", True, 8),
    (2, 7, 3, 1, 128, 64, True, "heads", True, 1),
    (2, 33, 8, 8, 64, 16, True, None, False, 0),
    (5, 2, 6, 3, 64, 8, False, "heads", True, 3),
    (1, 300, 5, 5, 128, 96, False, "shared", False, 0),
    (2, 3, 17, 1, 128, 0, False, "shared", True, 0),
    (1, 2, 1, 1, 64, 0, False, None, True, 5),
    (4, 1, 64, 8, 64, 32, False, None, True, 0),
]


@pytest.mark.parametrize("dtype", (BF, F32))
@pytest.mark.parametrize("shape", SHAPES)
def test_rotate(nk, shape, dtype):
    B, n, Hq, H, D, rotary, il, norm, fused, offset = shape
    say(f"rotate {shape} {dtype}")
    rng = np.random.default_rng(1)
    rot = rotary_of(nk, rng, Hq, H, D, rotary, il, norm)
    q, k, v = heads_of(rng, B, n, Hq, H, D, dtype, fused, offset)
    start = [int(rng.integers(0, 700 - n + 1)) for _ in range(B)]
    start[-1] = 700 - n
    lens = [max(0, n - i) for i in range(B)]
    for new_lens in (None, lens):
        outs = [torch.full((B, n, h, D), 7.0, dtype=dtype, device="cuda") for h in (Hq, H, H)]
        got = nk.rotate_qkv(rot, q, k, v, i32(start), new_lens=None if new_lens is None else i32(new_lens), q_out=outs[0],
                            k_out=outs[1], v_out=outs[2])
        torch.cuda.synchronize()
        mine = np.arange(n) < np.array([n] * B if new_lens is None else new_lens)[:, None]
        for g, x, w in ((got[0], q, rot.q_norm), (got[1], k, rot.k_norm)):
            assert_close(g, oracle_heads(rot, x, w, start), dtype, mine)
            assert (g[torch.as_tensor(~mine).cuda()] == 7).all()
        rows = torch.as_tensor(mine).cuda()
        assert torch.equal(got[2][rows], v[rows]) and (got[2][~rows] == 7).all()


def test_rotate_outputs_and_sides(nk):
    """Sides left out; outputs in place; outputs that the call makes; positions outside the table."""
    rng = np.random.default_rng(2)
    rot = rotary_of(nk, rng, 8, 2, 128, 128, False, "shared", P=100)
    q, k, v = heads_of(rng, 3, 4, 8, 2, 128, BF, False)
    start = i32([0, 98, -2])
    full = nk.rotate_qkv(rot, q, k, v, start, q_out=torch.zeros_like(q), k_out=torch.zeros_like(k), v_out=torch.zeros_like(v))
    assert full[0][0].any() and not full[0][1, 2:].any() and full[2][1, :2].any() and not full[2][1, 2:].any()
    assert not full[1][2, :2].any() and full[1][2, 2:].any()
    only_k = nk.rotate_qkv(rot, None, k, None, start, k_out=torch.zeros_like(k))
    assert only_k[0] is None and only_k[2] is None and torch.equal(only_k[1], full[1])
    made = nk.rotate_qkv(rot, q, k, v, start, new_lens=i32([4, 2, 0]))
    assert torch.equal(made[0][:2], full[0][:2]) and not made[0][2].any()
    q2, k2 = q.clone(), k.clone()
    nk.rotate_qkv(rot, q2, k2, None, i32([3, 0, 40]), q_out=q2, k_out=k2)
    apart = nk.rotate_qkv(rot, q, k, None, i32([3, 0, 40]))
    assert torch.equal(q2, apart[0]) and torch.equal(k2, apart[1])
    none = nk.rotate_qkv(rot, q[:, :0], k[:, :0], v[:, :0], start)
    assert none[0].shape == (3, 0, 8, 128)
    plain = nk.Rotary(8, 2, 128)
    same = nk.rotate_qkv(plain, q, k, v, None)
    assert all(torch.equal(a, b) for a, b in zip(same, (q, k, v)))


def test_rotate_feeds_the_two_bit_cache(nk):
    """The dense tensors go to encode and to the step as they are."""
    import synth
    from oracle_cache import calibrated_params
    wl = synth.get_workload("qwen3_8b")
    P = nk.NovaKVParams.from_arrays(calibrated_params(wl, 0))
    H, Hq, D, L = wl.num_kv_heads, wl.num_q_heads, wl.head_dim, wl.groups
    rng = np.random.default_rng(3)
    rot = rotary_of(nk, rng, Hq, H, D, D, False, "shared")
    lay = nk.CacheLayout(16, 8, torch.as_tensor(rng.permutation(16).astype(np.int32).reshape(2, 8)).cuda())
    pools = [torch.zeros(nk.code_pool_shape(P, lay, 2), dtype=torch.uint8, device="cuda") for _ in range(4)]
    q, k, v = heads_of(rng, 2, 40, Hq, H, D, BF, True)
    start = i32([0, 17])
    _, kd, vd = nk.rotate_qkv(rot, q, k, v, start)
    nk.encode(P, lay, kd, vd, start, pools[0], pools[1])
    nk.encode(P, lay, torch.as_tensor(oracle_heads(rot, k, rot.k_norm, [0, 17])).float().to(BF).cuda(), v.contiguous(), start, pools[2], pools[3])
    same = float((pools[0] == pools[2]).float().mean())
    assert torch.equal(pools[1], pools[3]) and same > 0.999      # a key coordinate may round to the next bf16 value
    qs, ks, vs = heads_of(rng, 2, 1, Hq, H, D, BF, True)
    lens = i32([41, 58])
    qd, kd, vd = nk.rotate_qkv(rot, qs, ks, vs, lens - 1)
    out = nk.append_decode_attn(P, lay, kd[:, 0], vd[:, 0], qd[:, 0], pools[0], pools[1], lens, 128)
    assert torch.isfinite(out).all() and out.any()


@pytest.mark.parametrize("dtype", (BF, F32))
@pytest.mark.parametrize("block", (0, 7, 16, 64))
@pytest.mark.parametrize("shape", SHAPES)
def test_append(nk, shape, block, dtype):
    B, n, Hq, H, D, rotary, il, norm, fused, offset = shape
    say(f"append {shape} block={block} {dtype}")
    rng = np.random.default_rng(4)
    rot = rotary_of(nk, rng, Hq, H, D, rotary, il, norm)
    q, k, v = heads_of(rng, B, n, Hq, H, D, dtype, fused, offset)
    cap = n + 60
    rows = block or cap
    bps = -(-cap // rows)
    nblk = B * bps + 2
    table = None if not block else rng.permutation(nblk)[: B * bps].astype(np.int32).reshape(B, bps)
    lay = nk.CacheLayout(rows, bps, None if table is None else torch.as_tensor(table).cuda())
    start = [int(rng.integers(0, 60)) for _ in range(B)]
    lens = [max(0, n - i) for i in range(B)]
    for new_lens in (None, lens):
        cache = nk.Q4Cache.zeros(lay, B, H, D, num_blocks=nblk)
        for t, fill in zip(cache.tensors[1:], (0xA5, 0x5A, 2.0, 3.0)):
            t.fill_(fill)
        held = [torch.full((B, n, H, D), 7.0, dtype=dtype, device="cuda") for _ in range(2)]
        q_out = nk.q4_append(rot, cache, q, k, v, i32(start), new_lens=None if new_lens is None else i32(new_lens),
                             k_held=held[0], v_held=held[1])
        torch.cuda.synchronize()
        mine = np.arange(n) < np.array([n] * B if new_lens is None else new_lens)[:, None]
        assert_close(q_out, oracle_heads(rot, q, rot.q_norm, start), dtype, mine)
        pos = np.asarray(start)[:, None] + np.arange(n)
        page = np.arange(B)[:, None] * bps + pos // rows
        page = page if table is None else table.reshape(-1)[page]
        at = (page[mine], slice(None), (pos % rows)[mine])
        ties = 0
        for side, x, w, codes, sq, h in ((0, k, rot.k_norm, cache.k_codes, cache.k_sq, held[0]), (1, v, None, cache.v_codes, cache.v_sq, held[1])):
            y = oracle_heads(rot, x, w, start) if side == 0 else x.double().cpu().numpy()
            rc, rsq, gap = q4.quantize_rows(y[mine])
            got_c = codes.cpu().numpy()
            got_sq = sq.view(torch.int16).cpu().numpy().view(np.uint16)
            assert (got_sq[at] == rsq).all()
            bad = q4.unpack_codes(got_c[at]) != rc
            assert not (bad & (gap > 1e-9)).any(), f"side {side}: {int((bad & (gap > 1e-9)).sum())} codes differ"
            ties += int((gap == 0).sum())
            value = (q4.from_bf16_bits(rsq[..., :1]).astype(np.float32) * rc.astype(np.float32) + q4.from_bf16_bits(rsq[..., 1:]).astype(np.float32))
            want = torch.as_tensor(value).to(dtype)
            hold = h.cpu()[torch.as_tensor(mine)]
            assert torch.equal(hold[torch.as_tensor(~bad)], want[torch.as_tensor(~bad)])
            assert (h[torch.as_tensor(~mine).cuda()] == 7).all()
            got_c[at] = (0xA5, 0x5A)[side]                      # all else is as it was
            got_sq[at] = q4.to_bf16_bits((2.0, 3.0)[side])
            assert (got_c == (0xA5, 0x5A)[side]).all() and (got_sq == q4.to_bf16_bits((2.0, 3.0)[side])).all()


@pytest.mark.parametrize("dtype", (BF, F32))
@pytest.mark.parametrize("shape", [(2, 300, 4, 2, 128, 128, False, "shared"), (1, 8200, 2, 1, 64, 64, True, "heads"),
                                   (3, 2800, 3, 1, 128, 48, False, None), (600, 1, 2, 2, 64, 24, False, "shared")])
def test_many_tokens(nk, shape, dtype):
    """Launches of many tokens quantize in fp32, and again in fp64 where that may not decide:
    the codes are those of fp64 all the same."""
    B, n, Hq, H, D, rotary, il, norm = shape
    say(f"many tokens {shape} {dtype}")
    rng = np.random.default_rng(7)
    rot = rotary_of(nk, rng, Hq, H, D, rotary, il, norm, P=n + 5)
    q, k, v = heads_of(rng, B, n, Hq, H, D, dtype, True)
    start = [int(rng.integers(0, 5)) for _ in range(B)]
    lay = nk.CacheLayout(16, -(-(n + 5) // 16), None)
    cache = nk.Q4Cache.zeros(lay, B, H, D)
    q_out = nk.q4_append(rot, cache, q, k, v, i32(start))
    rotated = nk.rotate_qkv(rot, q, k, v, i32(start))
    assert torch.equal(q_out, rotated[0]) and torch.equal(rotated[2], v)
    every = np.ones((B, n), dtype=bool)
    ref_k = oracle_heads(rot, k, rot.k_norm, start)
    assert_close(q_out, oracle_heads(rot, q, rot.q_norm, start), dtype, every)
    assert_close(rotated[1], ref_k, dtype, every)
    pos = np.asarray(start)[:, None] + np.arange(n)
    page = np.arange(B)[:, None] * lay.blocks_per_seq + pos // 16
    for y, codes, sq in ((ref_k, cache.k_codes, cache.k_sq), (v.double().cpu().numpy(), cache.v_codes, cache.v_sq)):
        rc, rsq, gap = q4.quantize_rows(y)
        assert (sq.view(torch.int16).cpu().numpy().view(np.uint16)[page, :, pos % 16] == rsq).all()
        bad = q4.unpack_codes(codes.cpu().numpy()[page, :, pos % 16]) != rc
        assert not (bad & (gap > 1e-9)).any()


@pytest.mark.parametrize("copies", (1, 40, 600))
def test_append_borders(nk, copies):
    """Rows of quotients that are ties, constant rows, tiny and huge ones, NaN and infinities."""
    D = 64
    rows = [np.arange(D) % 31 / 2 - 3.0,                                   # every half: ties to even
            np.full(D, 0.3), np.zeros(D), -np.zeros(D),
            np.where(np.arange(D) == 5, 1e-40, 0.0), np.linspace(-1e-39, 1e-39, D),
            np.linspace(-3e38, 3e38, D), np.linspace(-1, 1, D) * 2.0 ** -120,
            np.where(np.arange(D) == 63, 1e30, 1.0), np.linspace(100, 100.01, D),
            np.where(np.arange(D) == 9, np.nan, 1.0), np.where(np.arange(D) == 63, np.inf, 1.0),
            np.where(np.arange(D) == 0, -np.inf, 1.0), np.where(np.arange(D) == 31, -3.4e38, 1.0)]
    rows = rows * copies
    x = np.array(rows, dtype=np.float32)[None, :, None]
    for dtype in (F32, BF):
        t = torch.as_tensor(x).to(dtype).cuda()
        lay = nk.CacheLayout.contiguous(len(rows))
        cache = nk.Q4Cache.zeros(lay, 1, 1, D)
        held = torch.zeros_like(t), torch.zeros_like(t)
        nk.q4_append(nk.Rotary(1, 1, D), cache, None, t, t, i32([0]), k_held=held[0], v_held=held[1])
        rc, rsq, _ = q4.quantize_rows(t.double().cpu().numpy()[0, :, 0])
        for codes, sq, h in ((cache.k_codes, cache.k_sq, held[0]), (cache.v_codes, cache.v_sq, held[1])):
            got_sq = sq.view(torch.int16).cpu().numpy().view(np.uint16)[0, 0]
            assert (got_sq == rsq).all(), (got_sq, rsq)
            assert (q4.unpack_codes(codes.cpu().numpy()[0, 0]) == rc).all()
            assert (torch.isnan(h[0, :, 0]).all(-1).cpu().numpy() == (rsq[:, 0] == 0x7FC0)).all()


def test_append_outside(nk):
    """Positions outside the cache or the table, and blocks that hold nothing, are left out."""
    rng = np.random.default_rng(5)
    q, k, v = heads_of(rng, 4, 6, 4, 2, 64, BF, True)
    rot = rotary_of(nk, rng, 4, 2, 64, 64, False, None, P=40)
    table = np.array([[0, 1, 2], [3, -1, 4], [9, 5, 6], [7, 8, 10]], dtype=np.int32)   # the pool has 9 blocks
    lay = nk.CacheLayout(16, 3, torch.as_tensor(table).cuda())
    cache = nk.Q4Cache.zeros(lay, 4, 2, 64, num_blocks=9)
    held = torch.zeros_like(k.contiguous()), torch.zeros_like(k.contiguous())
    q_out = torch.zeros_like(q.contiguous())
    nk.q4_append(rot, cache, q, k, v, i32([-3, 13, 12, 37]), q_out=q_out, k_held=held[0], v_held=held[1])
    wrote = q_out.any(-1).any(-1).cpu().numpy()
    want = np.array([[p >= 0 and p < 40 for p in range(s, s + 6)] for s in (-3, 13, 12, 37)])
    want[1, 3:] = False          # positions 16.. of sequence 1: no block
    want[2, :4] = False          # positions 12..15 of sequence 2: block 9 of 9
    want[3, :] = False           # positions 37..: past block 10, and the table
    assert (wrote == want).all()
    assert (held[0].any(-1).any(-1).cpu().numpy() == want).all() and (held[1].any(-1).any(-1).cpu().numpy() == want).all()
    stored = cache.k_sq.any(-1).any(1).cpu().numpy()             # [blocks][rows]
    assert stored.sum() == want.sum() and stored[0, :3].all() and stored[3, 13:].all() and stored[5, :2].all()


def test_append_then_attend(nk):
    """A layer in use: a ragged prompt, a drafted chunk, then steps, captured in a graph and replayed;
    the held values under a plain attention give the same outputs."""
    rng = np.random.default_rng(6)
    B, Hq, H, D, block, cap = 3, 8, 2, 128, 16, 128
    rot = rotary_of(nk, rng, Hq, H, D, D, False, "shared")
    table = torch.as_tensor(rng.permutation(B * 8).astype(np.int32).reshape(B, 8)).cuda()
    cache = nk.Q4Cache.zeros(nk.CacheLayout(block, 8, table), B, H, D)
    k_all, v_all = (np.zeros((B, H, cap, D)) for _ in range(2))
    lens = np.zeros(B, dtype=np.int64)
    ws = torch.zeros(max(256, *(nk.q4_attn_workspace_bytes(cache, B, m, Hq, cap) for m in (1, 4, 50))), dtype=torch.uint8, device="cuda")

    def keep(held, counts):
        for x, h in ((k_all, held[0]), (v_all, held[1])):
            h = h.double().cpu().numpy()
            for b in range(B):
                x[b, :, lens[b]:lens[b] + counts[b]] = h[b, :counts[b]].transpose(1, 0, 2)
        lens[:] += counts

    def expect(q, counts, out):
        q, out = q.double().cpu().numpy(), out.double().cpu().numpy()
        for b in range(B):
            for i in range(counts[b]):
                S = lens[b] - counts[b] + i + 1
                for h in range(Hq):
                    z = k_all[b, h // 4, :S] @ q[b, i, h] / np.sqrt(D)
                    p = np.exp(z - z.max())
                    ref = (p / p.sum()) @ v_all[b, h // 4, :S]
                    # the output's bf16 step, fp16 probabilities (of 15 s <= 2 V), bf16 steps of the held values and keys
                    V, dz = np.abs(v_all[b]).max(), 2.0 ** -8 * (np.abs(k_all[b, h // 4, :S]) @ np.abs(q[b, i, h])).max() / np.sqrt(D)
                    tol = 2.0 ** -8 * np.abs(ref) + (2.0 ** -10 + 2.0 ** -8 + 2 * dz) * V
                    assert (np.abs(out[b, i, h] - ref) <= tol).all()

    for n, counts in ((50, [50, 31, 1]), (4, [4, 2, 3])):
        q, k, v = heads_of(rng, B, n, Hq, H, D, BF, True)
        held = [torch.zeros((B, n, H, D), dtype=BF, device="cuda") for _ in range(2)]
        qr = nk.q4_append(rot, cache, q, k, v, i32(lens.tolist()), new_lens=i32(counts), k_held=held[0], v_held=held[1])
        keep(held, np.array(counts))
        out = nk.q4_attn(cache, qr, i32(lens.tolist()), cap, q_lens=i32(counts), workspace=ws)
        expect(qr, counts, out)

    x = torch.zeros((B, 1, Hq + 2 * H, D), dtype=BF, device="cuda")
    qr, out = (torch.zeros((B, 1, Hq, D), dtype=BF, device="cuda") for _ in range(2))
    held = [torch.zeros((B, 1, H, D), dtype=BF, device="cuda") for _ in range(2)]
    seq, start = i32((lens + 1).tolist()), i32(lens.tolist())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        nk.q4_append(rot, cache, x[:, :, :Hq], x[:, :, Hq:Hq + H], x[:, :, Hq + H:], start, q_out=qr, k_held=held[0], v_held=held[1])
        nk.q4_attn(cache, qr, seq, cap, out=out, workspace=ws)
        seq.add_(1)
        start.add_(1)
    for _ in range(4):
        x.copy_(torch.as_tensor(rng.standard_normal(tuple(x.shape))).to(BF))
        graph.replay()
        torch.cuda.synchronize()
        keep(held, np.ones(B, dtype=np.int64))
        expect(qr, [1] * B, out)
    assert start.tolist() == lens.tolist()


def test_refusals(nk):
    rng = np.random.default_rng(8)
    q, k, v = heads_of(rng, 2, 3, 8, 2, 64, BF, True)
    rot = rotary_of(nk, rng, 8, 2, 64, 64, False, "shared")
    cache = nk.Q4Cache.zeros(nk.CacheLayout.contiguous(16), 2, 2, 64)
    start = i32([0, 1])
    dense = q.contiguous()
    cases = [
        (TypeError, dict(k=k.float())), (TypeError, dict(q=q.half())), (ValueError, dict(k=k[:, :, :1])), (ValueError, dict(v=v.transpose(1, 2))),
        (ValueError, dict(q=q[..., :32])), (ValueError, dict(q=dense.transpose(2, 3).contiguous().transpose(2, 3))),
        (TypeError, dict(start_pos=start.long())), (ValueError, dict(start_pos=i32([0]))), (ValueError, dict(new_lens=i32([0]))),
        (ValueError, dict(q_out=q)), (TypeError, dict(q_out=dense.float())), (ValueError, dict(q_out=dense[:, :1].contiguous())),
        (ValueError, dict(start_pos=start.cpu())), (nk.NovaKVError, dict(q=dense[:, :, :].clone(), start_pos=None)),
    ]
    for error, change in cases:
        for append in (False, True):
            args = dict(q=q, k=k, v=v, start_pos=start)
            args.update(change)
            with pytest.raises(error):
                nk.q4_append(rot, cache, **args) if append else nk.rotate_qkv(rot, **args)
    with pytest.raises(nk.NovaKVError):
        nk.rotate_qkv(rot, dense, None, None, start, q_out=torch.zeros(dense.numel() + 1, dtype=BF, device="cuda")[1:].view(dense.shape))
    buf = torch.zeros(2 * dense.numel(), dtype=BF, device="cuda")
    with pytest.raises(nk.NovaKVError, match="overlaps"):
        nk.rotate_qkv(rot, buf[:dense.numel()].view(dense.shape), None, None, start, q_out=buf[64:64 + dense.numel()].view(dense.shape))
    with pytest.raises(nk.NovaKVError):       # another head_dim than the cache's
        nk.q4_append(nk.Rotary(8, 2, 128), cache, None, torch.zeros((2, 1, 2, 128), device="cuda"), torch.zeros((2, 1, 2, 128), device="cuda"), start)
    with pytest.raises(ValueError):
        nk.rotate_qkv(rot, None, None, None, start)
