"""The operators around a 4-bit cache and in front of both caches, as cases that can be timed and checked.

A decoder layer projects its hidden states to queries, keys and values, norms
each query and key head, rotates it by its position, appends keys and values
to the layer's cache and attends over that cache.  ``rotate_qkv`` is the norm
and rotation in front of the 2-bit cache's calls (nova_kv_encode and the step),
``q4_append`` the same with the append to a cache held in 4 bits, and
``q4_attn`` the attention over that cache.  The listed cases stand for one user
with a short context up to 64 sequences of 32K tokens, prompts, chunks of
prompts and drafted tokens, both head sizes, paged and contiguous caches.

A case is a dict: ``op`` ("rotate", "append" or "attn"), ``batch``, ``n``
(tokens per sequence: new ones, or queries), ``q_heads``, ``kv_heads``,
``head_dim``, ``dtype`` ("bf16" or "f32"), ``ragged`` (lengths and positions
differ per sequence, rows behind a sequence's own are padding); for rotate and
append ``norm``, ``rotary`` (coordinates rotated), ``interleaved`` (pairs of
neighbours, not of halves), ``fused`` (q, k and v are slices of one projection),
``start`` (the first new position); for append and attn ``block`` (tokens per
cache block, 0 = contiguous with ``capacity`` rows per sequence); for attn
``seq`` (cached tokens of the longest sequence, the queries' own included),
``window`` and ``sinks``.
"""
import math

import torch

own = False

EPS = 1e-6        # of the norms
THETA = 1e6       # base of the rotation's angles


def _case(name, op, batch, n, q_heads, kv_heads, head_dim, **more):
    c = {"name": name, "op": op, "batch": batch, "n": n, "q_heads": q_heads, "kv_heads": kv_heads, "head_dim": head_dim,
         "dtype": "bf16", "ragged": False}
    if op == "attn":
        c.update(seq=0, window=0, sinks=False)
    else:
        c.update(norm=True, rotary=head_dim, interleaved=False, fused=True, start=0)
    if op != "rotate":
        c.update(block=0, capacity=0)
    c.update(more)
    return c


def listed():
    return [
        # one user's decode step at 2000 tokens, in front of the 2-bit cache's step: the smallest call
        _case("rotate_one_token", "rotate", 1, 1, 32, 8, 128, start=1999),
        # prompts of 32 sequences of 4096 tokens, in front of the encoder
        _case("rotate_prompt", "rotate", 32, 4096, 32, 8, 128),
        # a ragged chunk in fp32 of a model that rotates half of a 64-wide head by neighbours and has no norms
        _case("rotate_partial_f32", "rotate", 3, 613, 64, 8, 64, dtype="f32", ragged=True, norm=False, rotary=32,
              interleaved=True, fused=False, start=70001),
        # the decode step of a busy server, 16-token pages
        _case("append_64_tokens", "append", 64, 1, 32, 8, 128, ragged=True, block=16, start=3000, capacity=4096),
        # prompts of 32 sequences written to pages
        _case("append_prompt", "append", 32, 4096, 32, 8, 128, block=16, capacity=4096),
        # a chunk of a few tokens behind ragged contexts, fp32, head size 64, a cache of odd capacity
        _case("append_chunk_f32", "append", 8, 24, 64, 8, 64, dtype="f32", ragged=True, norm=False, start=577,
              capacity=613),
        # one user, a short chat: launch and set-up time
        _case("attn_one_user_2k", "attn", 1, 1, 32, 8, 128, seq=2000, capacity=2048),
        # the largest cache: 64 sequences of 32K tokens on 16-token pages
        _case("attn_64x32k_paged", "attn", 64, 1, 32, 8, 128, seq=32768, block=16, capacity=32768),
        # one sequence of 128K tokens
        _case("attn_one_128k", "attn", 1, 1, 32, 8, 128, seq=131072, capacity=131072),
        # a sliding-window layer with learned sinks, ragged, eight query heads per KV head of 64
        _case("attn_window_sinks", "attn", 16, 1, 64, 8, 64, seq=6000, ragged=True, capacity=8192, window=128, sinks=True),
        # a chunk of two prompts over what is cached already
        _case("attn_chunk_2k", "attn", 2, 2048, 32, 8, 128, seq=8192, block=16, capacity=8192),
        # drafted tokens in fp32 over ragged contexts, an odd capacity
        _case("attn_drafted_f32", "attn", 5, 5, 16, 8, 128, dtype="f32", seq=5003, ragged=True, capacity=5003),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("rotate", "append", "attn", "attn"))
    d = rng.choice((128, 128, 64))
    kv = rng.choice((8, 8, 8, 4, 2, 1, 5))
    hq = kv * rng.choice((1, 2, 3, 4, 4, 4, 5, 6, 7, 8, 8))
    block = rng.choice((0, 0, 16, 16, 32, 64, 24))
    batch = _log(rng, 1, 64)
    more = dict(dtype=rng.choice(("bf16", "bf16", "f32")), ragged=rng.random() < 0.6)
    if op == "attn":
        # at most the largest listed case's cached token-heads, and the listed chunk's logits
        s = _log(rng, 1, max(1, min(131072, (1 << 24) // (batch * kv))))
        n = rng.choice((1, 1, 1, _log(rng, 2, 16), _log(rng, 16, 2048)))
        n = max(1, min(n, s, (1 << 28) // (batch * hq * s)))
        c = _case("", op, batch, n, hq, kv, d, seq=s, window=rng.choice((0, 0, 0, 128, _log(rng, 1, 4096))),
                  sinks=rng.random() < 0.3, block=block, capacity=s + rng.randint(0, 200), **more)
    else:
        # at most the listed prompts' projected heads
        n = rng.choice((1, _log(rng, 2, 64), _log(rng, 64, 8192)))
        n = max(1, min(n, (1 << 22) // (batch * (hq + 2 * kv))))
        more.update(norm=rng.random() < 0.6, rotary=rng.choice((d, d, d, d // 2, d // 4, 0)),
                    interleaved=rng.random() < 0.3, fused=rng.random() < 0.7, start=_log(rng, 1, 100000) - 1)
        if op == "append":
            # positions in front of the new tokens are cache too: a pool of at most 2^18 rows
            more["start"] %= max(1, (1 << 18) // batch - n)
            more.update(block=block, capacity=more["start"] + n + rng.randint(0, 200))
        c = _case("", op, batch, n, hq, kv, d, **more)
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs

def _lens(c):
    """Tokens (queries) of each sequence, and the position of its first one."""
    b, n = c["batch"], c["n"]
    if c["op"] == "attn":
        seq = [c["seq"]] * b
        if c["ragged"]:  # from half to all of the longest, the last of several sequences an idle one
            seq = [c["seq"] - (c["seq"] // 2) * i // b for i in range(b)]
            if b > 3:
                seq[-1] = 0
        count = [min(n, s) if not c["ragged"] or n == 1 else min(max(1, n - i % n), s) for i, s in enumerate(seq)]
        return count, seq
    start = [c["start"]] * b
    count = [n] * b
    if c["ragged"]:
        start = [max(0, c["start"] - 37 * i) for i in range(b)]
        count = [max(1, n - i * (n // 2) // b) for i in range(b)]
    return count, start


def _spectrum(h, d, gen):
    """Standard deviations of a layer's channels: most alike, a few of them several times as large."""
    s = torch.randn((h, d), generator=gen, device="cuda").mul_(0.3).exp_()
    return s * (1 + 3 * (torch.rand((h, d), generator=gen, device="cuda") < 0.04))


def _pages(c, gen):
    """(rows of a block, blocks per sequence, block table or None, blocks of the pool)"""
    b = c["batch"]
    if not c["block"]:
        return c["capacity"], 1, None, b
    bps = -(-c["capacity"] // c["block"])
    table = torch.randperm(b * bps, generator=gen, device="cuda").to(torch.int32).reshape(b, bps)
    return c["block"], bps, table, b * bps


def _inputs(c, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    b, n, hq, h, d = c["batch"], c["n"], c["q_heads"], c["kv_heads"], c["head_dim"]
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    count, first = _lens(c)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    s = {"case": c}
    if c["op"] == "attn":
        s["q"] = (1.5 * rnd(b, n, hq, d)).to(dt)
        s["seq_lens"] = i32(first)
        s["q_lens"] = i32(count) if c["ragged"] and n > 1 else None
        s["sinks"] = rnd(hq) if c["sinks"] else None
        s["out"] = torch.zeros((b, n, hq, d), dtype=dt, device="cuda")
        s["rows"], s["per_seq"], s["table"], s["blocks"] = _pages(c, gen)
        for side in ("k", "v"):  # a cache of such a layer's rows, filled a part at a time
            std, mean = _spectrum(h, d, gen), 0.5 * rnd(h, d) if side == "k" else 0.0
            codes = torch.empty((s["blocks"], h, s["rows"], d // 2), dtype=torch.uint8, device="cuda")
            sq = torch.empty((s["blocks"], h, s["rows"], 2), dtype=torch.bfloat16, device="cuda")
            for i in range(0, s["blocks"], max(1, (1 << 22) // (h * s["rows"]))):
                part = slice(i, i + max(1, (1 << 22) // (h * s["rows"])))
                x = rnd(*codes[part].shape[:3], d) * std[:, None] + (mean[:, None] if side == "k" else 0.0)
                lo, hi = x.amin(-1), x.amax(-1)
                sq[part] = torch.stack(((hi - lo) / 15, lo), -1).to(torch.bfloat16)
                step, low = sq[part].float().unbind(-1)
                q = ((x - low[..., None]) / step[..., None]).round_().clamp_(0, 15).to(torch.uint8)
                codes[part] = q[..., ::2] | (q[..., 1::2] << 4)
            s[side + "_codes"], s[side + "_sq"] = codes, sq
        return s
    heads = hq + 2 * h
    scale = torch.cat([_spectrum(heads - h, d, gen), _spectrum(h, d, gen)])
    shift = torch.cat([torch.zeros((hq, d), device="cuda"), 0.5 * rnd(h, d), torch.zeros((h, d), device="cuda")])
    x = torch.empty((b, n, heads, d), dtype=dt, device="cuda")
    for i in range(b):
        x[i] = rnd(n, heads, d) * scale + shift
    s["qkv"] = x
    s["q"], s["k"], s["v"] = x[:, :, :hq], x[:, :, hq:hq + h], x[:, :, hq + h:]
    if not c["fused"]:
        s["q"], s["k"], s["v"] = (t.contiguous() for t in (s["q"], s["k"], s["v"]))
        del s["qkv"]
    s["start"] = i32(first)
    s["new_lens"] = i32(count) if c["ragged"] else None
    s["q_norm"], s["k_norm"] = ((1 + 0.2 * rnd(d)) for _ in range(2)) if c["norm"] else (None, None)
    r = c["rotary"]
    s["cos_sin"] = None
    if r:
        freq = THETA ** (-torch.arange(0, r, 2, dtype=torch.float64, device="cuda") / r)
        angle = torch.arange(c["start"] + n, dtype=torch.float64, device="cuda")[:, None] * freq
        s["cos_sin"] = torch.cat([angle.cos(), angle.sin()], 1).float()
    s["q_out"] = torch.zeros((b, n, hq, d), dtype=dt, device="cuda")
    s["k_out"], s["v_out"] = (torch.zeros((b, n, h, d), dtype=dt, device="cuda") for _ in range(2))
    if c["op"] == "append":
        s["rows"], s["per_seq"], s["table"], s["blocks"] = _pages(c, gen)
        for side in ("k", "v"):
            s[side + "_codes"] = torch.zeros((s["blocks"], h, s["rows"], d // 2), dtype=torch.uint8, device="cuda")
            s[side + "_sq"] = torch.zeros((s["blocks"], h, s["rows"], 2), dtype=torch.bfloat16, device="cuda")
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
    if c["op"] != "rotate":
        cache = nk.Q4Cache(nk.CacheLayout(s["rows"], s["per_seq"], s["table"]), s["k_codes"], s["v_codes"], s["k_sq"], s["v_sq"])
    if c["op"] == "attn":
        ws = torch.zeros(nk.q4_attn_workspace_bytes(cache, c["batch"], c["n"], c["q_heads"], c["seq"]), dtype=torch.uint8, device="cuda")
        return nk.prepare_q4_attn(cache, s["q"], s["seq_lens"], c["seq"], s["out"], ws, q_lens=s["q_lens"], window=c["window"],
                                  sinks=s["sinks"])
    rot = nk.Rotary(c["q_heads"], c["kv_heads"], c["head_dim"], cos_sin=s["cos_sin"], interleaved=c["interleaved"],
                    q_norm=s["q_norm"], k_norm=s["k_norm"], eps=EPS)
    if c["op"] == "rotate":
        return nk.prepare_rotate_qkv(rot, s["q"], s["k"], s["v"], s["start"], s["q_out"], s["k_out"], s["v_out"],
                                     new_lens=s["new_lens"])
    return nk.prepare_q4_append(rot, cache, s["q"], s["k"], s["v"], s["start"], s["q_out"], new_lens=s["new_lens"],
                                k_held=s["k_out"], v_held=s["v_out"])


# ------------------------------------------------------------------ one pass

def _valid(lens, n, device):
    """[B][n][1][1]: whether a row is one of its sequence's own."""
    i = torch.arange(n, device=device)
    return (i < lens[:, None])[:, :, None, None]


def _norm_rotate(s, x, weight, wide):
    """The norm and rotation of heads [B][n][H][D], in 32 bits (64 for what is quantized, where a value may lie next to a border)."""
    c = s["case"]
    x = x.to(wide)
    if weight is not None:
        x = x * (x.square().mean(-1, keepdim=True) + EPS).rsqrt() * weight.to(wide)
    r = c["rotary"]
    if not r:
        return x
    at = s["start"].long()[:, None] + torch.arange(c["n"], device=x.device)
    row = s["cos_sin"][at.clamp(max=len(s["cos_sin"]) - 1)].to(wide)[:, :, None]
    cos, sin = row[..., :r // 2], row[..., r // 2:]
    if c["interleaved"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((turned, x[..., r:]), -1) if r < c["head_dim"] else turned


def _keep(s, name, new, valid):
    """`new` in the rows of `valid`, what was there elsewhere."""
    s[name].copy_(new if valid is None else torch.where(valid, new.to(s[name].dtype), s[name]))


def _plain_append(s, side, x, valid):
    """Rows x [B][n][H][D] in 64 bits, quantized and stored at their positions."""
    c = s["case"]
    lo, hi = x.amin(-1), x.amax(-1)
    sq = torch.stack(((hi - lo) / 15, lo), -1).to(torch.bfloat16)
    step, low = sq.unbind(-1)
    codes = ((x - low.double()[..., None]) / step.double()[..., None]).round()
    codes = torch.where(step[..., None] == 0, 0.0, codes).clamp(0, 15).to(torch.uint8)
    held = codes.float() * step.float()[..., None] + low.float()[..., None]
    _keep(s, side + "_out", held, valid)
    at = s["start"].long()[:, None] + torch.arange(c["n"], device=x.device)
    page, row = at // s["rows"], at % s["rows"]
    page = page + torch.arange(c["batch"], device=x.device)[:, None] * s["per_seq"]
    if s["table"] is not None:
        page = s["table"].flatten()[page.clamp(max=s["table"].numel() - 1)].long()
    if valid is not None:
        mine = valid[..., 0, 0]
        page, row, codes, sq = page[mine], row[mine], codes[mine], sq[mine]
    packed = codes[..., ::2] | (codes[..., 1::2] << 4)
    s[side + "_codes"][page, :, row] = packed
    s[side + "_sq"][page, :, row] = sq


def _plain_cache(s, side):
    """The cache's values [B][H][seq][D] in 32 bits."""
    c = s["case"]
    pool = lambda t: (t if s["table"] is None else t[s["table"].flatten().long()])  # noqa: E731
    by_seq = lambda t: pool(t).unflatten(0, (c["batch"], s["per_seq"])).transpose(1, 2).flatten(2, 3)[:, :, :c["seq"]]  # noqa: E731
    codes, sq = by_seq(s[side + "_codes"]), by_seq(s[side + "_sq"]).float()
    values = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).float()
    return values * sq[..., :1] + sq[..., 1:]


def _plain_attn(s):
    c = s["case"]
    b, n, hq, h, d = c["batch"], c["n"], c["q_heads"], c["kv_heads"], c["head_dim"]
    q = s["q"].float().reshape(b, n, h, hq // h, d).permute(0, 2, 1, 3, 4).reshape(b, h, n * (hq // h), d)
    z = torch.matmul(q, _plain_cache(s, "k").transpose(2, 3).contiguous()).reshape(b, h, n, hq // h, c["seq"]) / math.sqrt(d)
    at = (s["seq_lens"] - (n if s["q_lens"] is None else s["q_lens"]))[:, None] + torch.arange(n, device=q.device)
    key = torch.arange(c["seq"], device=q.device)
    seen = key <= at[..., None]
    if c["window"]:
        seen &= key > at[..., None] - c["window"]
    z = z.masked_fill_(~seen[:, None, :, None], -math.inf)
    top = z.amax(-1, keepdim=True)
    sink = None
    if s["sinks"] is not None:
        sink = s["sinks"].reshape(1, h, 1, hq // h, 1)
        top = torch.maximum(top, sink)
    top = torch.where(top == -math.inf, 0.0, top)
    p = z.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    if sink is not None:
        total = total + (sink - top).exp()
    out = torch.matmul(p.reshape(b, h, -1, c["seq"]), _plain_cache(s, "v")).reshape(b, h, n, hq // h, d)
    out = torch.where(total > 0, out / total, 0.0).permute(0, 2, 1, 3, 4).reshape(b, n, hq, d)
    _keep(s, "out", out, None if s["q_lens"] is None else _valid(s["q_lens"], n, q.device))


def _outputs(s):
    c = s["case"]
    if c["op"] == "attn":
        return {"out": s["out"]}
    o = {"q": s["q_out"], "k": s["k_out"], "v": s["v_out"]}
    if c["op"] == "append":
        o.update((name, s[name]) for name in ("k_codes", "v_codes", "k_sq", "v_sq"))
    return o


def run(state):
    s, c = state, state["case"]
    if own:
        s["call"]()
        return _outputs(s)
    if c["op"] == "attn":
        _plain_attn(s)
        return _outputs(s)
    valid = None if s["new_lens"] is None else _valid(s["new_lens"], c["n"], s["q"].device)
    _keep(s, "q_out", _norm_rotate(s, s["q"], s["q_norm"], torch.float32), valid)
    if c["op"] == "rotate":
        _keep(s, "k_out", _norm_rotate(s, s["k"], s["k_norm"], torch.float32), valid)
        _keep(s, "v_out", s["v"], valid)
    else:
        _plain_append(s, "k", _norm_rotate(s, s["k"], s["k_norm"], torch.float64), valid)
        _plain_append(s, "v", s["v"].double(), valid)
    return _outputs(s)


# ------------------------------------------------------------------ the definition in 64 bits

def _exact_heads(s, x, weight, at):
    """Heads of one sequence [m][H][D]: x / rms * w, then each pair times cos + i sin."""
    c, x = s["case"], x.double()
    if weight is not None:
        x = weight.double() * x / (torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / c["head_dim"] + EPS).sqrt()
    r = c["rotary"]
    if r:
        turn = torch.complex(*s["cos_sin"][at].double().chunk(2, dim=1))[:, None]
        pairs = (0, r, 2), (1, r, 2)
        if not c["interleaved"]:
            pairs = (0, r // 2, 1), (r // 2, r, 1)
        a, b = (slice(*p) for p in pairs)
        z = torch.complex(x[..., a].contiguous(), x[..., b].contiguous()) * turn
        x = x.clone()
        x[..., a], x[..., b] = z.real, z.imag
    return x


def _exact_held(x):
    low = x.min(-1, keepdim=True).values
    step = ((x.max(-1, keepdim=True).values - low) / 15).to(torch.bfloat16).double()
    low = low.to(torch.bfloat16).double()
    return low + step * torch.where(step > 0, ((x - low) / step).round().clamp(0, 15), 0.0)


def exact(case, seed):
    c, s = case, _inputs(case, seed)
    count, first = _lens(c)
    b, n, hq, h, d = c["batch"], c["n"], c["q_heads"], c["kv_heads"], c["head_dim"]
    wide = lambda heads: torch.zeros((b, n, heads, d), dtype=torch.float64, device="cuda")  # noqa: E731
    if c["op"] != "attn":
        o = {"q": wide(hq), "k": wide(h), "v": wide(h)}
        for i in range(b):
            m = count[i]
            at = torch.arange(first[i], first[i] + m, device="cuda")
            o["q"][i, :m] = _exact_heads(s, s["q"][i, :m], s["q_norm"], at)
            o["k"][i, :m] = _exact_heads(s, s["k"][i, :m], s["k_norm"], at)
            o["v"][i, :m] = s["v"][i, :m].double()
            if c["op"] == "append":
                o["k"][i, :m], o["v"][i, :m] = _exact_held(o["k"][i, :m]), _exact_held(o["v"][i, :m])
        if c["op"] == "append":
            o.update(k_codes=None, v_codes=None, k_sq=None, v_sq=None)
        return o
    out = wide(hq)
    for i in range(b):
        m, size = count[i], first[i]
        if not m or not size:
            continue
        pages = torch.arange(s["per_seq"], device="cuda") + i * s["per_seq"]
        if s["table"] is not None:
            pages = s["table"][i].long()
        both = []
        for side in ("k", "v"):
            byte = s[side + "_codes"][pages].transpose(0, 1).reshape(h, -1, d // 2)[:, :size].double()
            high = torch.floor(byte / 16)
            value = torch.stack((byte - 16 * high, high), -1).reshape(h, size, d)
            sq = s[side + "_sq"][pages].transpose(0, 1).reshape(h, -1, 2)[:, :size].double()
            both.append(sq[..., 1:] + sq[..., :1] * value)
        behind = torch.arange(size - m, size, device="cuda")[:, None] - torch.arange(size, device="cuda")  # how far a key is behind
        hidden = behind < 0
        if c["window"]:
            hidden = hidden | (behind >= c["window"])
        for g in range(hq // h):  # the query heads g, g + hq/h, ... share no KV head
            q = s["q"][i, :m, g::hq // h].double().transpose(0, 1).contiguous()
            z = torch.bmm(q, both[0].transpose(1, 2).contiguous()) / d ** 0.5
            z = z.masked_fill(hidden, -math.inf)
            if s["sinks"] is not None:
                z = torch.cat([z, s["sinks"][g::hq // h].double()[:, None, None].expand(h, m, 1)], -1)
            p = torch.softmax(z, -1)[..., :size].contiguous()
            out[i, :m, g::hq // h] = torch.bmm(p, both[1]).transpose(0, 1)
    return {"out": out}


def work(case):
    c = case
    count, first = _lens(c)
    hq, h, d = c["q_heads"], c["kv_heads"], c["head_dim"]
    e = 2 if c["dtype"] == "bf16" else 4
    if c["op"] != "attn":
        t = sum(count)
        heads = hq + 2 * h
        written = t * heads * d * e
        if c["op"] == "append":  # the codes, scales and offsets, beside the values that they stand for
            written += t * 2 * h * (d // 2 + 4)
        table = 4 * c["rotary"] * (max(f + m for f, m in zip(first, count)) - min(first)) if c["rotary"] else 0
        per = (4 if c["norm"] else 0) + (3 * c["rotary"] / d)
        return {"bytes": t * heads * d * e + written + table,
                "flops": int(t * (hq + h) * d * per) + (t * 2 * h * d * 6 if c["op"] == "append" else 0)}
    pairs = read = 0
    for m, size in zip(count, first):
        w = c["window"] or size
        each = [min(size - m + i + 1, w) for i in range(m)]
        pairs += sum(each)
        read += min(size, w + m - 1) if m else 0
    return {"bytes": read * h * (d + 8) + 2 * sum(count) * hq * d * e, "flops": 4 * d * hq * pairs}
