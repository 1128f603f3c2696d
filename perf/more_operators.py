"""Operators of prompts over the caches, as cases that can be timed and checked.

A prompt that comes in chunks, with images in it, is rotated at positions of
several axes (time, height, width), appended to its layer's cache and attended
over that cache; drafted tokens are attended the same way; and a prefix that is
cached already is read back as dense rows, for another engine or for attention
by other means.  ``axes`` is the norm and rotation at positions of several axes
in front of the 2-bit cache's calls, ``append`` the same with the append to a
cache held in 4 bits, ``chunk`` the causal attention of one or more query tokens
per sequence over the 2-bit cache, ``read`` and ``read4`` the way back out of the
2-bit and of the 4-bit cache.

A case is a dict: ``op``, ``batch``, ``n`` (tokens per sequence: new ones, queries,
or tokens read), ``q_heads``, ``kv_heads``, ``head_dim``, ``dtype`` ("bf16" or
"f32": of the rows that go in and come out), ``ragged`` (lengths and positions
differ per sequence, rows behind a sequence's own are padding); for axes and
append ``axes`` (how many), ``order`` (which axis a rotated pair follows: "blocks"
of neighbours, a "cycle" through the axes, or a "grid" of blocks whose
frequencies start again), ``norm``, ``rotary``, ``interleaved`` (pairs of
neighbours, not of halves), ``fused`` (q, k and v are slices of one projection),
``start`` (the first new token's place); for the others ``seq`` (cached tokens of
the longest sequence); for all but axes ``block`` (tokens per cache block, 0 =
contiguous with ``capacity`` rows per sequence); for chunk ``window`` and
``sinks``; for chunk and read the 2-bit cache's formats ``key_scale``, ``sq``,
``fp8``, ``bf16_transforms``, ``band`` (64 sink and 256 recent positions).
"""
import math

import torch

own = False

EPS = 1e-6         # of the norms
THETA = 1e6        # base of the rotation's angles
BAND = (64, 256)   # sink and recent positions of the band
G, K = 4, 256      # coordinates of a group, codewords of a codebook
DEPLOYED = {"key_scale": True, "sq": True, "fp8": True, "bf16_transforms": True, "band": True}


def _case(name, op, batch, n, q_heads, kv_heads, head_dim, **more):
    c = {"name": name, "op": op, "batch": batch, "n": n, "q_heads": q_heads, "kv_heads": kv_heads, "head_dim": head_dim,
         "dtype": "bf16", "ragged": False}
    if op in ("axes", "append"):
        c.update(axes=3, order="blocks", norm=True, rotary=head_dim, interleaved=False, fused=True, start=0)
    else:
        c.update(seq=0)
    if op == "chunk":
        c.update(window=0, sinks=False)
    if op in ("chunk", "read"):
        c.update(key_scale=False, sq=False, fp8=False, bf16_transforms=False, band=False)
    if op != "axes":
        c.update(block=0, capacity=0)
    c.update(more)
    return c


def listed():
    return [
        # one user's decode step behind a prompt with images, in front of the 2-bit cache's step: the smallest call
        _case("axes_one_token", "axes", 1, 1, 32, 8, 128, start=1999),
        # prompts with images of 32 sequences of 4096 tokens, in front of the encoder
        _case("axes_prompt", "axes", 32, 4096, 32, 8, 128),
        # the same prompts on their way to 16-token pages of a layer that is kept at 4 bits
        _case("append_prompt", "append", 32, 4096, 32, 8, 128, order="cycle", block=16, capacity=4096),
        # a ragged fp32 chunk of an image's patches at (row, column), heads of 64 without norms, an odd capacity
        _case("append_patches_f32", "append", 8, 24, 64, 8, 64, dtype="f32", ragged=True, axes=2, order="grid", norm=False,
              start=577, capacity=613),
        # one user's four drafted tokens at 2000 tokens: launch and set-up time
        _case("chunk_drafted_2k", "chunk", 1, 4, 32, 8, 128, seq=2000, capacity=2048),
        # a busy server's drafted tokens: 64 sequences of up to 16K tokens on 16-token pages
        _case("chunk_drafted_64x16k", "chunk", 64, 4, 32, 8, 128, seq=16384, ragged=True, block=16, capacity=16384),
        # a chunk of two prompts over what is cached already
        _case("chunk_prompt_2k", "chunk", 2, 2048, 32, 8, 128, seq=8192, block=16, capacity=8192),
        # ragged chunks in fp32 over the deployed format, heads of 64 with learned sinks, an odd capacity
        _case("chunk_deployed_f32", "chunk", 5, 77, 64, 8, 64, dtype="f32", seq=5003, ragged=True, capacity=5003, sinks=True,
              **DEPLOYED),
        # the cached prefixes of 16 sequences read back, in the benchmark's format
        _case("read_prefix_16x8k", "read", 16, 8192, 32, 8, 128, seq=8192, block=16, capacity=8192),
        # parts of ragged sequences in the deployed format, fp32, heads of 64
        _case("read_deployed_f32", "read", 6, 1201, 64, 8, 64, dtype="f32", seq=1500, ragged=True, capacity=1511, **DEPLOYED),
        # the same prefixes out of a 4-bit cache
        _case("read4_prefix_16x8k", "read4", 16, 8192, 32, 8, 128, seq=8192, block=16, capacity=8192),
        # a few tokens of ragged sequences, fp32, heads of 64, odd sizes
        _case("read4_few_f32", "read4", 3, 61, 64, 8, 64, dtype="f32", seq=613, ragged=True, capacity=613),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("axes", "append", "chunk", "chunk", "chunk", "read", "read4"))
    d = rng.choice((128, 128, 64))
    kv = rng.choice((8, 8, 8, 4, 2, 1, 5))
    hq = kv * rng.choice((1, 2, 3, 4, 4, 4, 5, 6, 7, 8, 8))
    block = rng.choice((0, 0, 16, 16, 32, 64, 24))
    batch = _log(rng, 1, 64)
    more = dict(dtype=rng.choice(("bf16", "bf16", "f32")), ragged=rng.random() < 0.6)
    formats = rng.choice(({}, {}, {"fp8": True}, {"key_scale": True}, {"sq": True}, {"band": True}, DEPLOYED,
                          {"key_scale": True, "sq": True, "bf16_transforms": True}))
    if op in ("axes", "append"):
        # at most the listed prompts' projected heads
        n = rng.choice((1, _log(rng, 2, 64), _log(rng, 64, 8192)))
        n = max(1, min(n, (1 << 22) // (batch * (hq + 2 * kv))))
        more.update(axes=rng.choice((1, 2, 3, 3, 4)), order=rng.choice(("blocks", "cycle", "grid")), norm=rng.random() < 0.6,
                    rotary=rng.choice((d, d, d, d // 2, d // 4)), interleaved=rng.random() < 0.3, fused=rng.random() < 0.7,
                    start=_log(rng, 1, 100000) - 1)
        if op == "append":
            # places in front of the new tokens are cache too: a pool of at most 2^18 rows
            more["start"] %= max(1, (1 << 18) // batch - n)
            more.update(block=block, capacity=more["start"] + n + rng.randint(0, 200))
        c = _case("", op, batch, n, hq, kv, d, **more)
    elif op == "chunk":
        # at most the listed server's cached token-heads, and the listed chunk's logits
        s = _log(rng, 1, max(1, min(131072, (1 << 23) // (batch * kv))))
        n = rng.choice((1, _log(rng, 2, 16), _log(rng, 2, 16), _log(rng, 16, 2048)))
        n = max(1, min(n, s, (1 << 30) // (batch * hq * s)))
        c = _case("", op, batch, n, hq, kv, d, seq=s, window=rng.choice((0, 0, 0, 128, _log(rng, 1, 4096))),
                  sinks=rng.random() < 0.3, block=block, capacity=s + rng.randint(0, 200), **formats, **more)
    else:
        # at most the listed prefixes' rows
        s = _log(rng, 1, max(1, min(131072, (1 << 20) // (batch * kv))))
        c = _case("", op, batch, rng.choice((s, _log(rng, 1, s))), hq, kv, d, seq=s, block=block,
                  capacity=s + rng.randint(0, 200), **(formats if op == "read" else {}), **more)
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs

def _lens(c):
    """Each sequence's own tokens (new ones, queries, or those read), and its cached tokens (or the first new one's place)."""
    b, n = c["batch"], c["n"]
    if c["op"] in ("axes", "append"):
        if not c["ragged"]:
            return [n] * b, [c["start"]] * b
        return [max(1, n - i * (n // 2) // b) for i in range(b)], [max(0, c["start"] - 37 * i) for i in range(b)]
    seq = [c["seq"]] * b
    if c["ragged"]:  # from all to half of the longest, the last of several sequences an idle one
        seq = [c["seq"] - (c["seq"] // 2) * i // b for i in range(b)]
        if b > 3:
            seq[-1] = 0
    return [min(max(1, n - i % n), s) if c["ragged"] else min(n, s) for i, s in enumerate(seq)], seq


def _place(m, size):
    """The first of the m tokens that a case reads of a sequence of `size`: three of four of the others lie in front of it."""
    return 3 * (size - m) // 4


def _pages(c, gen):
    """(rows of a block, blocks per sequence, block table or None, blocks of the pool)"""
    b = c["batch"]
    if not c["block"]:
        return c["capacity"], 1, None, b
    bps = -(-c["capacity"] // c["block"])
    table = torch.randperm(b * bps, generator=gen, device="cuda").to(torch.int32).reshape(b, bps)
    return c["block"], bps, table, b * bps


def _axis_of(c):
    """Which axis each rotated pair follows."""
    pairs, axes = c["rotary"] // 2, c["axes"]
    if c["order"] == "cycle":
        return [j % axes for j in range(pairs)]
    first = pairs // axes if c["order"] == "grid" else max(1, pairs // (axes + 1))  # blocks: a shorter one of time in front
    return [0 if j < first or axes == 1 else min(axes - 1, 1 + (j - first) * (axes - 1) // (pairs - first)) for j in range(pairs)]


def _frequencies(c):
    """Of each pair: theta^(-2j / rotary), for a grid with j counted from its block's first."""
    axis, r = _axis_of(c), c["rotary"]
    j = [i - axis.index(a) if c["order"] == "grid" else i for i, a in enumerate(axis)]
    span = max(j) + 1 if c["order"] == "grid" else r // 2
    return THETA ** (-torch.tensor(j, dtype=torch.float64, device="cuda") / span)


def _positions(c, first):
    """[axes][B][n]: text, at the same position on all axes, with an image of 16 columns in every 300 tokens: there the
    first axis stands still, the second counts rows, the third columns (a fourth rows again)."""
    i = torch.arange(c["n"], device="cuda")
    at = torch.tensor(first, device="cuda")[:, None] + i
    inside = (at % 300) - 40
    image = (inside >= 0) & (inside < 256)
    base = at - inside
    grid = [base, base + inside // 16, base + inside % 16, base + inside // 16]
    if c["axes"] < 3:
        grid = grid[1:]
    return torch.stack([torch.where(image, g, at) for g in grid[:c["axes"]]]).to(torch.int32)


def _spectrum(h, d, gen):
    """Standard deviations of a layer's channels: most alike, a few of them several times as large."""
    s = torch.randn((h, d), generator=gen, device="cuda").mul_(0.3).exp_()
    return s * (1 + 3 * (torch.rand((h, d), generator=gen, device="cuda") < 0.04))


def _new_rows(c, s, gen):
    """What the axes and append cases have in hand: a projection's rows and the layer's norms and angles."""
    b, n, hq, h, d = c["batch"], c["n"], c["q_heads"], c["kv_heads"], c["head_dim"]
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    rnd = lambda *t: torch.randn(t, generator=gen, device="cuda")  # noqa: E731
    count, first = _lens(c)
    scale = torch.cat([_spectrum(hq + h, d, gen), _spectrum(h, d, gen)])
    shift = torch.cat([torch.zeros((hq, d), device="cuda"), 0.5 * rnd(h, d), torch.zeros((h, d), device="cuda")])
    x = torch.empty((b, n, hq + 2 * h, d), dtype=dt, device="cuda")
    for i in range(b):
        x[i] = rnd(n, hq + 2 * h, d) * scale + shift
    s["q"], s["k"], s["v"] = x[:, :, :hq], x[:, :, hq:hq + h], x[:, :, hq + h:]
    if not c["fused"]:
        s["q"], s["k"], s["v"] = (t.contiguous() for t in (s["q"], s["k"], s["v"]))
    s["start"] = torch.tensor(first, dtype=torch.int32, device="cuda")
    s["positions"] = _positions(c, first)
    s["new_lens"] = torch.tensor(count, dtype=torch.int32, device="cuda") if c["ragged"] else None
    s["q_norm"], s["k_norm"] = ((1 + 0.2 * rnd(d)) for _ in range(2)) if c["norm"] else (None, None)
    angle = torch.arange(max(first) + n, dtype=torch.float64, device="cuda")[:, None] * _frequencies(c)
    s["cos_sin"] = torch.cat([angle.cos(), angle.sin()], 1).float()
    s["pair_axis"] = _axis_of(c)
    s["axis"] = torch.tensor(s["pair_axis"], device="cuda")
    s["q_out"] = torch.zeros((b, n, hq, d), dtype=dt, device="cuda")


def _params(c, s, gen):
    """A layer's stored parameters: transforms that keep a random basis and even the falling spectrum of its keys a
    little, and codebooks that are samples of their groups' own distributions."""
    h, d = c["kv_heads"], c["head_dim"]
    host = torch.Generator().manual_seed(int(torch.randint(0, 1 << 30, (1,), generator=gen, device="cuda")))
    rnd = lambda *t: torch.randn(t, generator=host, dtype=torch.float64)  # noqa: E731
    qk, qv = (torch.linalg.qr(rnd(h, d, d))[0] for _ in range(2))
    lam = torch.arange(1, d + 1, dtype=torch.float64) ** -0.6
    sigma = (lam * (d / lam.sum())).sqrt()
    even = sigma ** -0.25
    wide = torch.bfloat16 if c["bf16_transforms"] else torch.float32
    s["kbar"] = (0.3 * rnd(h, d)).float().cuda()
    for name, t in (("t_k", qk * even), ("t_k_inv_t", qk / even), ("t_v", qv)):
        s[name] = t.float().to(wide).cuda()
    for name, std in (("cb_k", sigma * even), ("cb_v", sigma)):
        book = 0.92 * rnd(h, d // G, K, G) * std.reshape(1, d // G, 1, G)
        s[name] = (book.float().to(torch.float8_e4m3fn).view(torch.uint8) if c["fp8"] else book.half()).cuda()


def _cache2(c, s, gen):
    """A filled 2-bit cache."""
    b, h, d = c["batch"], c["kv_heads"], c["head_dim"]
    _params(c, s, gen)
    shape = (s["blocks"], h, s["rows"])
    for name in ("k_codes", "v_codes"):
        s[name] = torch.randint(0, 256, shape + (d // G,), generator=gen, device="cuda", dtype=torch.uint8)
    s["k_scales"] = s["v_sq"] = s["band_k"] = s["band_v"] = None
    if c["key_scale"]:
        s["k_scales"] = torch.randn(shape, generator=gen, device="cuda").mul_(0.25).exp_().to(torch.bfloat16)
    if c["sq"]:  # a token's grid: four levels about its mean
        step = 1.2 + 0.4 * torch.rand(shape, generator=gen, device="cuda")
        low = -1.5 * step + 0.1 * torch.randn(shape, generator=gen, device="cuda")
        s["v_sq"] = torch.stack((step, low), -1).to(torch.bfloat16)
    if c["band"]:
        rows = lambda: torch.randn((b, h, sum(BAND), d), generator=gen, device="cuda")  # noqa: E731
        s["band_k"] = (rows() + s["kbar"][:, None]).to(torch.bfloat16)
        s["band_v"] = rows().to(torch.bfloat16)


def _cache4(c, s, gen):
    """A filled 4-bit cache, a part at a time."""
    h, d = c["kv_heads"], c["head_dim"]
    per = max(1, (1 << 22) // (h * s["rows"]))
    for side in ("k", "v"):
        std = _spectrum(h, d, gen)
        codes = torch.empty((s["blocks"], h, s["rows"], d // 2), dtype=torch.uint8, device="cuda")
        sq = torch.empty((s["blocks"], h, s["rows"], 2), dtype=torch.bfloat16, device="cuda")
        for i in range(0, s["blocks"], per):
            part = slice(i, i + per)
            x = torch.randn((*codes[part].shape[:3], d), generator=gen, device="cuda") * std[:, None]
            lo, hi = x.amin(-1), x.amax(-1)
            sq[part] = torch.stack(((hi - lo) / 15, lo), -1).to(torch.bfloat16)
            step, low = sq[part].float().unbind(-1)
            q = ((x - low[..., None]) / step[..., None]).round_().clamp_(0, 15).to(torch.uint8)
            codes[part] = q[..., ::2] | (q[..., 1::2] << 4)
        s[side + "_codes"], s[side + "_sq"] = codes, sq


def _inputs(c, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    b, n, hq, h, d = c["batch"], c["n"], c["q_heads"], c["kv_heads"], c["head_dim"]
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    count, first = _lens(c)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    s = {"case": c}
    if c["op"] != "axes":
        s["rows"], s["per_seq"], s["table"], s["blocks"] = _pages(c, gen)
    if c["op"] in ("axes", "append"):
        _new_rows(c, s, gen)
        if c["op"] == "append":
            for side in ("k", "v"):
                s[side + "_codes"] = torch.zeros((s["blocks"], h, s["rows"], d // 2), dtype=torch.uint8, device="cuda")
                s[side + "_sq"] = torch.zeros((s["blocks"], h, s["rows"], 2), dtype=torch.bfloat16, device="cuda")
    elif c["op"] == "read4":
        _cache4(c, s, gen)
    else:
        _cache2(c, s, gen)
    if c["op"] == "chunk":
        s["q"] = (2.0 * torch.randn((b, n, hq, d), generator=gen, device="cuda")).to(dt)
        s["sinks"] = torch.randn(hq, generator=gen, device="cuda") if c["sinks"] else None
        s["out"] = torch.zeros((b, n, hq, d), dtype=dt, device="cuda")
        s["lens"] = i32(count) if c["ragged"] or count[0] < n else None
    else:
        s["k_out"], s["v_out"] = (torch.zeros((b, n, h, d), dtype=dt, device="cuda") for _ in range(2))
    if c["op"] in ("read", "read4"):
        s["start"] = i32([_place(m, size) for m, size in zip(count, first)])
        s["lens"] = i32(count) if c["ragged"] or count[0] < n else None
    if c["op"] in ("chunk", "read"):
        s["seq_lens"] = i32(first)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        s["call"] = _handle(s)
    return s


def _handle(s):
    """The call as a serving loop keeps it: arguments marshalled once, the workspace allocated."""
    import paper_2608_04074_amd as nk
    c = s["case"]
    if c["op"] in ("axes", "append"):
        rot = nk.Rotary(c["q_heads"], c["kv_heads"], c["head_dim"], cos_sin=s["cos_sin"], interleaved=c["interleaved"],
                        q_norm=s["q_norm"], k_norm=s["k_norm"], eps=EPS)
        axes = nk.RotaryAxes(s["pair_axis"], num_axes=c["axes"])
        if c["op"] == "axes":
            return nk.prepare_rotate_qkv_axes(rot, axes, s["q"], s["k"], s["v"], s["positions"], s["q_out"], s["k_out"],
                                              s["v_out"], new_lens=s["new_lens"])
    layout = nk.CacheLayout(s["rows"], s["per_seq"], s["table"])
    if c["op"] in ("append", "read4"):
        cache = nk.Q4Cache(layout, s["k_codes"], s["v_codes"], s["k_sq"], s["v_sq"])
        if c["op"] == "read4":
            return nk.prepare_q4_read(cache, s["start"], s["k_out"], s["v_out"], lens=s["lens"])
        return nk.prepare_q4_append_axes(rot, axes, cache, s["q"], s["k"], s["v"], s["start"], s["positions"], s["q_out"],
                                         new_lens=s["new_lens"], k_held=s["k_out"], v_held=s["v_out"])
    dense = [s[name].contiguous() for name in ("t_k", "t_k_inv_t", "t_v")]
    params = nk.NovaKVParams(s["kbar"], *dense, s["cb_k"], None if c["sq"] else s["cb_v"], key_scale=c["key_scale"],
                             sq_values=c["sq"])
    more = {"k_scales": s["k_scales"], "v_sq": s["v_sq"],
            "band": nk.Band(*BAND, s["band_k"], s["band_v"]) if c["band"] else None}
    if c["op"] == "read":
        return nk.prepare_read(params, layout, s["k_codes"], s["v_codes"], s["start"], s["k_out"], s["v_out"], lens=s["lens"],
                               seq_lens=s["seq_lens"], **more)
    need = nk.chunk_attn_workspace_bytes(params, c["batch"], c["n"], c["q_heads"], c["seq"])
    ws = torch.zeros(need, dtype=torch.uint8, device="cuda") if need else None
    return nk.prepare_chunk_attn(params, layout, s["q"], s["k_codes"], s["v_codes"], s["seq_lens"], c["seq"], s["out"], ws,
                                 q_lens=s["lens"], window=c["window"], sinks=s["sinks"], **more)


# ------------------------------------------------------------------ one pass

def _valid(lens, n, device):
    """[B][n][1][1]: whether a row is one of its sequence's own."""
    i = torch.arange(n, device=device)
    return (i < lens[:, None])[:, :, None, None]


def _keep(s, name, new, valid):
    """`new` in the rows of `valid`, what was there elsewhere."""
    s[name].copy_(new if valid is None else torch.where(valid, new.to(s[name].dtype), s[name]))


def _norm_rotate(s, x, weight, wide):
    """The norm and rotation of heads [B][n][H][D], in 32 bits (64 for what is quantized, where a value may lie next to a border)."""
    c, r = s["case"], s["case"]["rotary"]
    x = x.to(wide)
    if weight is not None:
        x = x * (x.square().mean(-1, keepdim=True) + EPS).rsqrt() * weight.to(wide)
    at = s["positions"].long()[s["axis"]].permute(1, 2, 0)  # [B][n][pairs]: each pair's own position
    pair = torch.arange(r // 2, device=x.device)
    cos, sin = (s["cos_sin"][at, pair + i].to(wide)[:, :, None] for i in (0, r // 2))
    if c["interleaved"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((turned, x[..., r:]), -1) if r < c["head_dim"] else turned


def _rows_at(s, b, at):
    """Block and row of sequence b's tokens `at`."""
    page, row = at // s["rows"], at % s["rows"]
    return (b * s["per_seq"] + page if s["table"] is None else s["table"][b].long()[page]), row


def _plain_append(s, side, x, valid):
    """Rows x [B][n][H][D] in 64 bits, quantized and stored at their places."""
    c = s["case"]
    lo, hi = x.amin(-1), x.amax(-1)
    sq = torch.stack(((hi - lo) / 15, lo), -1).to(torch.bfloat16)
    step, low = sq.unbind(-1)
    codes = ((x - low.double()[..., None]) / step.double()[..., None]).round()
    codes = torch.where(step[..., None] == 0, 0.0, codes).clamp(0, 15).to(torch.uint8)
    _keep(s, side + "_out", codes.float() * step.float()[..., None] + low.float()[..., None], valid)
    packed = codes[..., ::2] | (codes[..., 1::2] << 4)
    for b, m in enumerate(_lens(c)[0]):
        page, row = _rows_at(s, b, s["start"][b].long() + torch.arange(m, device=x.device))
        s[side + "_codes"][page, :, row] = packed[b, :m]
        s[side + "_sq"][page, :, row] = sq[b, :m]


def _codewords(book, codes):
    """Coefficients [m][H][D] of code rows [m][H][L], in 32 bits."""
    h, L = book.shape[:2]
    flat = (book.view(torch.float8_e4m3fn) if book.dtype == torch.uint8 else book).float().reshape(-1, G)
    first = (torch.arange(h * L, device=codes.device, dtype=torch.int32) * K).reshape(h, L)
    return flat[(codes.int() + first).flatten()].reshape(codes.shape[0], h, L * G)


def _back(x, t):
    """x [m][H][D] times the transposed transforms t [H][D][D]."""
    return torch.matmul(x.transpose(0, 1), t.float().transpose(1, 2).contiguous()).transpose(0, 1)


def _plain_cached(s, b, at, size):
    """Keys and values [m][H][D] of sequence b's tokens `at` (of `size`) in 32 bits."""
    c = s["case"]
    page, row = _rows_at(s, b, at)
    x = _codewords(s["cb_k"], s["k_codes"][page, :, row])
    if c["key_scale"]:
        x = x * s["k_scales"][page, :, row].float()[..., None]
    k = _back(x, s["t_k_inv_t"]) + s["kbar"]
    codes = s["v_codes"][page, :, row]
    if c["sq"]:
        levels = torch.stack([(codes >> i) & 3 for i in (0, 2, 4, 6)], -1).flatten(-2).float()
        grid = s["v_sq"][page, :, row].float()
        x = levels * grid[..., :1] + grid[..., 1:]
    else:
        x = _codewords(s["cb_v"], codes)
    v = _back(x, s["t_v"])
    if c["band"]:
        held = ((at < BAND[0]) | (at >= size - BAND[1]))[:, None, None]
        slot = torch.where(at < BAND[0], at, BAND[0] + at % BAND[1])
        k = torch.where(held, s["band_k"][b][:, slot].transpose(0, 1).float(), k)
        v = torch.where(held, s["band_v"][b][:, slot].transpose(0, 1).float(), v)
    return k, v


def _plain_read(s):
    c = s["case"]
    for b, (m, size) in enumerate(zip(*_lens(c))):
        at = s["start"][b].long() + torch.arange(m, device="cuda")
        if c["op"] == "read":
            k, v = _plain_cached(s, b, at, size)
        else:
            page, row = _rows_at(s, b, at)
            k, v = ((torch.stack((codes & 15, codes >> 4), -1).flatten(-2).float() * sq[..., :1] + sq[..., 1:])
                    for codes, sq in ((s[side + "_codes"][page, :, row], s[side + "_sq"][page, :, row].float()) for side in "kv"))
        s["k_out"][b, :m] = k
        s["v_out"][b, :m] = v


def _plain_chunk(s):
    c = s["case"]
    hq, h, d = c["q_heads"], c["kv_heads"], c["head_dim"]
    per = hq // h
    for b, (m, size) in enumerate(zip(*_lens(c))):
        if not m:
            continue
        first = max(0, size - m + 1 - c["window"]) if c["window"] else 0
        key = torch.arange(first, size, device="cuda")
        k, v = _plain_cached(s, b, key, size)
        q = s["q"][b, :m].float().reshape(m, h, per, d).permute(1, 0, 2, 3).reshape(h, m * per, d)
        z = torch.matmul(q, k.permute(1, 2, 0).contiguous()).reshape(h, m, per, -1) / math.sqrt(d)
        at = torch.arange(size - m, size, device="cuda")[:, None]
        seen = key <= at
        if c["window"]:
            seen &= key > at - c["window"]
        z = z.masked_fill_(~seen[:, None], -math.inf)
        top = z.amax(-1, keepdim=True)
        if s["sinks"] is not None:
            sink = s["sinks"].reshape(h, 1, per, 1)
            top = torch.maximum(top, sink)
        p = z.sub_(top).exp_()
        total = p.sum(-1, keepdim=True)
        if s["sinks"] is not None:
            total = total + (sink - top).exp()
        out = torch.matmul(p.reshape(h, m * per, -1), v.transpose(0, 1).contiguous()).reshape(h, m, per, d) / total
        s["out"][b, :m] = out.permute(1, 0, 2, 3).reshape(m, hq, d)


def _outputs(s):
    if s["case"]["op"] == "chunk":
        return {"out": s["out"]}
    o = {"k": s["k_out"], "v": s["v_out"]}
    if s["case"]["op"] in ("axes", "append"):
        o["q"] = s["q_out"]
    if s["case"]["op"] == "append":
        o.update((name, s[name]) for name in ("k_codes", "v_codes", "k_sq", "v_sq"))
    return o


def run(state):
    s, c = state, state["case"]
    if own:
        s["call"]()
    elif c["op"] == "chunk":
        _plain_chunk(s)
    elif c["op"] in ("read", "read4"):
        _plain_read(s)
    else:
        valid = None if s["new_lens"] is None else _valid(s["new_lens"], c["n"], s["q"].device)
        _keep(s, "q_out", _norm_rotate(s, s["q"], s["q_norm"], torch.float32), valid)
        if c["op"] == "axes":
            _keep(s, "k_out", _norm_rotate(s, s["k"], s["k_norm"], torch.float32), valid)
            _keep(s, "v_out", s["v"], valid)
        else:
            _plain_append(s, "k", _norm_rotate(s, s["k"], s["k_norm"], torch.float64), valid)
            _plain_append(s, "v", s["v"].double(), valid)
    return _outputs(s)


# ------------------------------------------------------------------ the definition in 64 bits

def _exact_heads(s, b, x, weight):
    """Heads of sequence b [m][H][D]: x / rms * w, then each pair times cos + i sin of its axis' angle."""
    c, x, m, r = s["case"], x.double(), len(x), s["case"]["rotary"]
    if weight is not None:
        x = weight.double() * x / (torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / c["head_dim"] + EPS).sqrt()
    turn = torch.stack([torch.complex(s["cos_sin"][:, j].double(), s["cos_sin"][:, j + r // 2].double())[s["positions"][a, b, :m].long()]
                        for j, a in enumerate(s["pair_axis"])], -1)[:, None]
    pairs = ((0, r, 2), (1, r, 2)) if c["interleaved"] else ((0, r // 2, 1), (r // 2, r, 1))
    first, second = (slice(*p) for p in pairs)
    z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * turn
    x = x.clone()
    x[..., first], x[..., second] = z.real, z.imag
    return x


def _exact_held(x):
    low = x.min(-1, keepdim=True).values
    step = ((x.max(-1, keepdim=True).values - low) / 15).to(torch.bfloat16).double()
    low = low.to(torch.bfloat16).double()
    return low + step * torch.where(step > 0, ((x - low) / step).round().clamp(0, 15), 0.0)


def _exact_pool(s, b, name):
    """Sequence b's part of a pool [H][capacity][...]."""
    pages = torch.arange(s["per_seq"], device="cuda") + b * s["per_seq"] if s["table"] is None else s["table"][b].long()
    return s[name][pages].transpose(0, 1).flatten(1, 2)


def _exact_cached(s, b, first, last, size):
    """Keys and values [H][last - first][D] of the 2-bit cache: codewords (scales, grids), back through the transforms."""
    c, d = s["case"], s["case"]["head_dim"]
    sides = []
    for side, book, back in (("k", "cb_k", "t_k_inv_t"), ("v", "cb_v", "t_v")):
        codes = _exact_pool(s, b, side + "_codes")[:, first:last]
        if side == "v" and c["sq"]:
            step, low = _exact_pool(s, b, "v_sq")[:, first:last].double().unbind(-1)
            x = torch.stack([low[..., None] + step[..., None] * ((codes.long() // 4 ** i) % 4) for i in range(G)], -1)
            x = x.reshape(c["kv_heads"], -1, d)
        else:
            words = s[book].view(torch.float8_e4m3fn).double() if c["fp8"] else s[book].double()
            x = torch.stack([words[:, g].gather(1, codes[:, :, g].long()[..., None].expand(-1, -1, G))
                             for g in range(d // G)], 2).reshape(c["kv_heads"], -1, d)
        if side == "k" and c["key_scale"]:
            x = _exact_pool(s, b, "k_scales")[:, first:last].double()[..., None] * x
        x = torch.bmm(x, s[back].double().transpose(1, 2).contiguous())
        if side == "k":
            x = x + s["kbar"].double()[:, None]
        if c["band"]:
            for p in (p for p in range(first, last) if p < BAND[0] or p >= size - BAND[1]):
                x[:, p - first] = s["band_" + side][b, :, p if p < BAND[0] else BAND[0] + p % BAND[1]].double()
        sides.append(x)
    return sides


def exact(case, seed):
    c, s = case, _inputs(case, seed)
    count, first = _lens(c)
    b, n, hq, h, d = c["batch"], c["n"], c["q_heads"], c["kv_heads"], c["head_dim"]
    wide = lambda heads: torch.zeros((b, n, heads, d), dtype=torch.float64, device="cuda")  # noqa: E731
    if c["op"] in ("axes", "append"):
        o = {"k": wide(h), "v": wide(h), "q": wide(hq)}
        for i in range(b):
            m = count[i]
            o["q"][i, :m] = _exact_heads(s, i, s["q"][i, :m], s["q_norm"])
            o["k"][i, :m] = _exact_heads(s, i, s["k"][i, :m], s["k_norm"])
            o["v"][i, :m] = s["v"][i, :m].double()
            if c["op"] == "append":
                o["k"][i, :m], o["v"][i, :m] = _exact_held(o["k"][i, :m]), _exact_held(o["v"][i, :m])
        if c["op"] == "append":
            o.update(k_codes=None, v_codes=None, k_sq=None, v_sq=None)
        return o
    if c["op"] == "read4":
        o = {"k": wide(h), "v": wide(h)}
        for i in range(b):
            for side in ("k", "v"):
                part = slice(_place(count[i], first[i]), _place(count[i], first[i]) + count[i])
                byte = _exact_pool(s, i, side + "_codes")[:, part].double()
                high = torch.floor(byte / 16)
                sq = _exact_pool(s, i, side + "_sq")[:, part].double()
                value = sq[..., 1:] + sq[..., :1] * torch.stack((byte - 16 * high, high), -1).reshape(h, -1, d)
                o[side][i, :count[i]] = value.transpose(0, 1)
        return o
    if c["op"] == "read":
        o = {"k": wide(h), "v": wide(h)}
        for i in range(b):
            m = count[i]
            if m:
                lo = _place(m, first[i])
                k, v = _exact_cached(s, i, lo, lo + m, first[i])
                o["k"][i, :m], o["v"][i, :m] = k.transpose(0, 1), v.transpose(0, 1)
        return o
    out = wide(hq)
    for i in range(b):
        m, size = count[i], first[i]
        if not m:
            continue
        lo = max(0, size - m + 1 - c["window"]) if c["window"] else 0
        k, v = _exact_cached(s, i, lo, size, size)
        behind = torch.arange(size - m, size, device="cuda")[:, None] - torch.arange(lo, size, device="cuda")  # how far a key is behind
        hidden = behind < 0
        if c["window"]:
            hidden = hidden | (behind >= c["window"])
        for g in range(hq // h):  # the query heads g, g + hq/h, ... share no KV head
            q = s["q"][i, :m, g::hq // h].double().transpose(0, 1).contiguous()
            z = torch.bmm(q, k.transpose(1, 2).contiguous()) / d ** 0.5
            z = z.masked_fill(hidden, -math.inf)
            if s["sinks"] is not None:
                z = torch.cat([z, s["sinks"][g::hq // h].double()[:, None, None].expand(h, m, 1)], -1)
            p = torch.softmax(z, -1)[..., :size - lo].contiguous()
            out[i, :m, g::hq // h] = torch.bmm(p, v).transpose(0, 1)
    return {"out": out}


def _token_bytes(c):
    """Of a cached token and KV head in the 2-bit cache: codes, and what the formats keep beside them."""
    return 2 * (c["head_dim"] // G) + (2 if c["key_scale"] else 0) + (4 if c["sq"] else 0)


def _layer_bytes(c):
    """Codebooks and the way back out of the transforms' domain, of all KV heads."""
    d = c["head_dim"]
    books = (1 if c["sq"] else 2) * d * K * (1 if c["fp8"] else 2)
    return c["kv_heads"] * (books + 2 * d * d * (2 if c["bf16_transforms"] else 4) + 4 * d)


def work(case):
    c = case
    count, first = _lens(c)
    hq, h, d = c["q_heads"], c["kv_heads"], c["head_dim"]
    e = 2 if c["dtype"] == "bf16" else 4
    t = sum(count)
    if c["op"] in ("axes", "append"):
        heads = hq + 2 * h
        moved = 2 * t * heads * d * e + 4 * t * c["axes"]
        if c["op"] == "append":  # the codes, scales and offsets, beside the values that they stand for
            moved += t * 2 * h * (d // 2 + 4)
        table = 4 * c["rotary"] * (max(f + m for f, m in zip(first, count)) - min(first))
        per = (4 if c["norm"] else 0) + (3 * c["rotary"] / d)
        return {"bytes": moved + table, "flops": int(t * (hq + h) * d * per) + (t * 2 * h * d * 6 if c["op"] == "append" else 0)}
    if c["op"] == "read4":
        return {"bytes": t * h * (2 * (d // 2 + 4) + 2 * d * e), "flops": t * 2 * h * d * 2}
    banded = lambda lo, hi, size: len([p for p in range(lo, hi) if p < BAND[0] or p >= size - BAND[1]]) if c["band"] else 0  # noqa: E731
    if c["op"] == "read":
        held = sum(banded(_place(m, size), _place(m, size) + m, size) for m, size in zip(count, first))
        return {"bytes": (t - held) * h * _token_bytes(c) + held * h * 4 * d + t * h * 2 * d * e + _layer_bytes(c),
                "flops": (t - held) * h * 4 * d * d}
    pairs = read = held = 0
    for m, size in zip(count, first):
        w = c["window"] or size
        pairs += sum(min(size - m + i + 1, w) for i in range(m))
        span = min(size, w + m - 1) if m else 0
        read += span
        held += banded(size - span, size, size)
    return {"bytes": (read - held) * h * _token_bytes(c) + held * h * 4 * d + 2 * t * hq * d * e + _layer_bytes(c),
            "flops": 4 * d * hq * pairs + 4 * d * d * hq * t}
