"""nova_kv_rotate_qkv_axes and nova_kv_q4_append_axes against the fp64 oracle, and a run of the calls as
a prompt with images takes them.

Tolerances of rotated values as in test_gpu_rotate_append.py: below 40 u of the row's largest magnitude
m, taken as 2^-18 m, and half a step of the output's type. Codes, scales and offsets must be the oracle's,
except that a quotient within 1e-9 of a border may fall on either side."""

import numpy as np
import pytest
import torch

from chunk_cases import Cache
from oracle import chunk, q4
from test_gpu_rotate_append import assert_close, heads_of, i32, rotary_of

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


def oracle_heads(rot, axes, x, weight, positions):
    """The oracle's heads: every token with a table row of its own."""
    B, n = x.shape[:2]
    table = rot.cos_sin.cpu().numpy()
    rows = chunk.axis_angles(table, axes.pair_axis, np.clip(positions, 0, len(table) - 1)).reshape(B * n, -1)
    return q4.norm_rotate(x.double().cpu().numpy(), None if weight is None else weight.double().cpu().numpy(), rot.eps, rows,
                          rot.interleaved, np.arange(B * n).reshape(B, n))


SHAPES = [  # B, n, Hq, H, D, rotary, interleaved, norm, fused, offset of the projection's rows, axes
    (1, 1, 32, 8, 128, 128, False, "shared", True, 0, ("blocks", (16, 24, 24))),
    (3, 5, 4, 2, 64, 64, False, "shared", True, 8, ("cycle", (12, 10, 10))),
    (2, 7, 3, 1, 128, 64, True, "heads", True, 1, ("blocks", (16, 16))),
    (2, 33, 8, 8, 64, 16, True, None, False, 0, ("cycle", (2, 2, 2, 2))),
    (5, 2, 6, 3, 64, 8, False, "heads", True, 3, ("blocks", (1, 3))),
    (1, 300, 5, 5, 128, 96, False, "shared", False, 0, ("blocks", (7, 30, 11))),
    (4, 1, 64, 8, 64, 32, False, None, True, 0, ("blocks", (16,))),
    (2, 4500, 2, 1, 128, 128, False, "shared", True, 0, ("cycle", (24, 20, 20))),
]


def case(nk, shape, seed, P=700):
    B, n, Hq, H, D, rotary, il, norm, fused, offset, (order, lengths) = shape
    rng = np.random.default_rng(seed)
    rot = rotary_of(nk, rng, Hq, H, D, rotary, il, norm, P=P)
    axes = getattr(nk.RotaryAxes, order)(lengths)
    positions = rng.integers(0, P, (len(lengths), B, n)).astype(np.int32)
    positions[:, -1, -1] = P - 1
    return rng, rot, axes, positions


@pytest.mark.parametrize("dtype", (BF, F32))
@pytest.mark.parametrize("shape", SHAPES)
def test_rotate(nk, shape, dtype):
    B, n, Hq, H, D = shape[:5]
    say(f"rotate axes {shape} {dtype}")
    rng, rot, axes, positions = case(nk, shape, 1)
    q, k, v = heads_of(rng, B, n, Hq, H, D, dtype, *shape[8:10])
    bad = positions.copy()
    if n > 2:
        bad[0, 0, 1], bad[-1, -1, 0] = -1, 700      # one axis outside the table: the token is left out
    for new_lens, pos in ((None, positions), ([max(0, n - i) for i in range(B)], bad)):
        outs = [torch.full((B, n, h, D), 7.0, dtype=dtype, device="cuda") for h in (Hq, H, H)]
        got = nk.rotate_qkv_axes(rot, axes, q, k, v, torch.as_tensor(pos).cuda(), new_lens=None if new_lens is None else i32(new_lens),
                                 q_out=outs[0], k_out=outs[1], v_out=outs[2])
        torch.cuda.synchronize()
        mine = np.arange(n) < np.array([n] * B if new_lens is None else new_lens)[:, None]
        mine &= ((pos >= 0) & (pos < 700)).all(0)
        rows = torch.as_tensor(mine).cuda()
        for g, x, w in ((got[0], q, rot.q_norm), (got[1], k, rot.k_norm)):
            assert_close(g, oracle_heads(rot, axes, x, w, pos), dtype, mine)
            assert (g[~rows] == 7).all()
        assert torch.equal(got[2][rows], v[rows]) and (got[2][~rows] == 7).all()


@pytest.mark.parametrize("dtype", (BF, F32))
@pytest.mark.parametrize("shape", SHAPES)
def test_append(nk, shape, dtype):
    B, n, Hq, H, D = shape[:5]
    say(f"append axes {shape} {dtype}")
    rng, rot, axes, positions = case(nk, shape, 2)
    q, k, v = heads_of(rng, B, n, Hq, H, D, dtype, *shape[8:10])
    start = [3 + 2 * b for b in range(B)]
    cap = max(start) + n + 1
    bps = -(-cap // 16)
    table = rng.permutation(B * bps).astype(np.int32).reshape(B, bps)
    cache = nk.Q4Cache.zeros(nk.CacheLayout(16, bps, torch.as_tensor(table).cuda()), B, H, D)
    held = [torch.zeros((B, n, H, D), dtype=dtype, device="cuda") for _ in range(2)]
    q_out = nk.q4_append_axes(rot, axes, cache, q, k, v, i32(start), torch.as_tensor(positions).cuda(), k_held=held[0], v_held=held[1])
    torch.cuda.synchronize()
    every = np.ones((B, n), dtype=bool)
    assert_close(q_out, oracle_heads(rot, axes, q, rot.q_norm, positions), dtype, every)
    at = np.array(start)[:, None] + np.arange(n)
    phys = table[np.arange(B)[:, None], at // 16]
    for x, codes, sq in ((oracle_heads(rot, axes, k, rot.k_norm, positions), cache.k_codes, cache.k_sq),
                         (v.double().cpu().numpy(), cache.v_codes, cache.v_sq)):
        want, bits, gap = q4.quantize_rows(x)
        got = q4.unpack_codes(codes.cpu().numpy()[phys, :, at % 16])
        assert ((got == want) | (gap < 1e-9)).all()
        assert (sq.view(torch.int16).cpu().numpy().view(np.uint16)[phys, :, at % 16] == bits).all()
    back = nk.q4_read(cache, i32(start), n, dtype=dtype)
    assert torch.equal(back[0], held[0]) and torch.equal(back[1], held[1])


def test_one_axis_is_the_plain_rotation(nk):
    """All pairs on one axis at start + i: bit for bit the call without axes."""
    rng = np.random.default_rng(3)
    rot = rotary_of(nk, rng, 8, 2, 128, 128, False, "shared")
    q, k, v = heads_of(rng, 2, 50, 8, 2, 128, BF, True)
    axes = nk.RotaryAxes([1] * 64, num_axes=2)
    pos = torch.zeros((2, 2, 50), dtype=torch.int32, device="cuda")
    pos[1] = i32([5, 100])[:, None] + torch.arange(50, device="cuda")
    for got, ref in zip(nk.rotate_qkv_axes(rot, axes, q, k, v, pos), nk.rotate_qkv(rot, q, k, v, i32([5, 100]))):
        assert torch.equal(got, ref)


def test_streams_graphs_and_in_place(nk):
    rng, rot, axes, positions = case(nk, SHAPES[0], 4)
    q, k, v = heads_of(rng, 1, 1, 32, 8, 128, BF, False)
    pos = torch.as_tensor(positions).cuda()
    want = nk.rotate_qkv_axes(rot, axes, q, k, v, pos)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = nk.rotate_qkv_axes(rot, axes, q, k, v, pos, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    x = [t.clone() for t in (q, k, v)]
    outs = [torch.zeros_like(t) for t in want]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        nk.prepare_rotate_qkv_axes(rot, axes, *x, pos, *outs)()
    for r in range(3):
        for t in x:
            t.add_(0.5)
        pos.fill_(100 + r)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, nk.rotate_qkv_axes(rot, axes, *x, pos)))
    pos.copy_(torch.as_tensor(positions))
    x = [t.clone() for t in (q, k, v)]
    nk.rotate_qkv_axes(rot, axes, *x, pos, q_out=x[0], k_out=x[1], v_out=x[2])
    assert all(torch.equal(a, b) for a, b in zip(x, want))


def test_refusals(nk):
    rng, rot, axes, positions = case(nk, SHAPES[1], 5)
    q, k, v = heads_of(rng, 3, 5, 4, 2, 64, BF, False)
    pos = torch.as_tensor(positions).cuda()
    for error, a, p in ((TypeError, axes, pos.long()), (ValueError, axes, pos[:2].contiguous()), (ValueError, axes, pos.cpu()),
                        (ValueError, axes, pos[:, :2].contiguous()), (ValueError, nk.RotaryAxes.blocks((8, 8, 8)), pos),
                        (ValueError, axes, pos.transpose(1, 2)), (TypeError, axes, None)):
        with pytest.raises(error):
            nk.rotate_qkv_axes(rot, a, q, k, v, p)
    for make in (lambda: nk.RotaryAxes([]), lambda: nk.RotaryAxes([0] * 65), lambda: nk.RotaryAxes([0, 4]), lambda: nk.RotaryAxes([0, -1]),
                 lambda: nk.RotaryAxes([0, 1], num_axes=1), lambda: nk.RotaryAxes([0], num_axes=5)):
        with pytest.raises(ValueError):
            make()
    assert nk.RotaryAxes.cycle((3, 1, 2)).pair_axis == (0, 1, 2, 0, 2, 0) and nk.RotaryAxes.blocks((1, 2)).pair_axis == (0, 1, 1)


@pytest.mark.parametrize("D,fmt,dtype", ((128, "plain", BF), (64, "deployed", F32)))
def test_a_prompt_in_chunks(nk, D, fmt, dtype):
    """Rotated on three axes, appended to the 2-bit cache, attended chunk by chunk and read back; the attention over the
    rows that are read back is the attention over the cache."""
    say(f"prompt in chunks D={D} {fmt} {dtype}")
    H, Hq, B, total = 2, 8, 2, 150
    c = Cache(nk, 6, [total] * B, H, D, 16, fmt)
    if c.band is not None:
        c.band.k.zero_()
        c.band.v.zero_()
    rng = c.rng
    rot = rotary_of(nk, rng, Hq, H, D, D, False, "shared")
    axes = nk.RotaryAxes.cycle((D // 2 - 2 * (D // 8), D // 8, D // 8))
    for first, n in ((0, 90), (90, 50), (140, 10)):
        q, k, v = heads_of(rng, B, n, Hq, H, D, dtype, True)
        pos = torch.as_tensor(rng.integers(0, 700, (3, B, n)).astype(np.int32)).cuda()
        qr, kr, vr = nk.rotate_qkv_axes(rot, axes, q, k, v, pos)
        nk.encode(c.params, c.layout, kr, vr, i32([first] * B), c.k_codes, c.v_codes, **c.more)
        lens = i32([first + n] * B)
        got = nk.chunk_attn(c.params, c.layout, qr, c.k_codes, c.v_codes, lens, first + n, **c.more)
        bk, bv = nk.read(c.params, c.layout, c.k_codes, c.v_codes, i32([0] * B), first + n, seq_lens=lens, dtype=F32, **c.more)
        if c.band is not None:
            assert torch.equal(bk[:, -min(n, 70):], kr[:, -min(n, 70):].to(BF).float())
        for b in range(B):
            for h in range(H):
                hs = slice(4 * h, 4 * h + 4)
                kd, vd = bk[b, :, h].double().cpu().numpy(), bv[b, :, h].double().cpu().numpy()
                x = qr[b, :, hs].double().cpu().numpy()
                ref = chunk.attend(x, kd, vd, first + np.arange(n))
                logit = (np.abs(x) @ np.abs(kd).T).max() / np.sqrt(D)      # of the rows as they are, a bound of the roundings' size
                eps = 2.0 ** -10 if dtype == BF else 2.0 ** -18
                tol = np.abs(ref) * 2.0 ** (-8 if dtype == BF else -24) + 4 * eps * (1 + logit) * np.linalg.norm(vd, axis=1).max()
                assert (np.abs(got[b, :, hs].double().cpu().numpy() - ref) <= tol).all()


def test_a_prompt_in_chunks_4_bits(nk):
    """The same into a 4-bit cache: append, attend, read back."""
    rng = np.random.default_rng(7)
    rot = rotary_of(nk, rng, 8, 2, 128, 128, False, "shared")
    axes = nk.RotaryAxes.blocks((16, 24, 24))
    cache = nk.Q4Cache.zeros(nk.CacheLayout(16, 8, i32([[3, 1, 0, 2, 4, 7, 6, 5]])), 1, 2, 128)
    for first, n in ((0, 60), (60, 40)):
        q, k, v = heads_of(rng, 1, n, 8, 2, 128, F32, True)
        pos = torch.as_tensor(rng.integers(0, 700, (3, 1, n)).astype(np.int32)).cuda()
        qr = nk.q4_append_axes(rot, axes, cache, q, k, v, i32([first]), pos)
        got = nk.q4_attn(cache, qr, i32([first + n]), 128)
        bk, bv = nk.q4_read(cache, i32([0]), first + n, dtype=F32)
        for h in range(2):
            ref = chunk.attend(qr[0, :, 4 * h:4 * h + 4].double().cpu().numpy(), bk[0, :, h].double().cpu().numpy(),
                               bv[0, :, h].double().cpu().numpy(), first + np.arange(n))
            size = bv[0, :, h].abs().max().item()
            assert np.abs(got[0, :, 4 * h:4 * h + 4].double().cpu().numpy() - ref).max() <= 2.0 ** -14 * size
