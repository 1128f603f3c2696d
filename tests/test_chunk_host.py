"""Argument checks of chunk attention, of reading caches back and of positions on several axes that need
no GPU: every call here is rejected by the host-side checks (or is a no-op) before any HIP call."""

import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

import paper_2608_04074_amd as nk
from oracle import chunk as oracle
from paper_2608_04074_amd import _native as nat
from test_q4_host import FUSED, INVALID, MB, OK, UNSUPPORTED, WORKSPACE, cache, ref, rotary, rows


def params(**kw):
    a = dict(num_kv_heads=8, head_dim=128, group_dim=4, codebook_size=256, flags=0, kbar=MB, t_k=2 * MB, t_k_inv_t=3 * MB,
             t_v=4 * MB, cb_k=5 * MB, cb_v=6 * MB)
    a.update(kw)
    return nat.Params(**a)


def layout(**kw):
    return nat.Layout(**dict(dict(block_size=16, blocks_per_seq=256, block_table=7 * MB), **kw))


def attend(p=None, lay=None, **kw):
    a = dict(q=1 << 33, dtype=nat.NOVA_KV_BF16, batch=2, n=3, hq=32, q_lens=None, k=1 << 30, v=2 << 30, ks=None, sq=None, band=None,
             seq=8 * MB, max_seq=4096, window=0, sinks=None, scale=0.0, out=2 << 33, ws=3 << 33, ws_bytes=1 << 32)
    a.update(kw)
    band = None if a["band"] is None else nat.Band(*a["band"])
    return nat.lib().nova_kv_chunk_attn(ref(params() if p is None else p), ref(layout() if lay is None else lay), a["q"], a["dtype"],
                                        a["batch"], a["n"], a["hq"], a["q_lens"], a["k"], a["v"], a["ks"], a["sq"], ref(band), a["seq"],
                                        a["max_seq"], a["window"], a["sinks"], a["scale"], a["out"], a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=9), INVALID), (dict(batch=-1), INVALID), (dict(n=-1), INVALID), (dict(batch=70000), INVALID),
    (dict(hq=0), INVALID), (dict(hq=12), INVALID), (dict(max_seq=0), INVALID), (dict(max_seq=4097), INVALID),
    (dict(window=-1), INVALID), (dict(scale=-0.5), INVALID), (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID),
    (dict(q=None), INVALID), (dict(seq=None), INVALID), (dict(out=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID),
    (dict(q=(1 << 33) + 8), INVALID), (dict(out=(2 << 33) + 4), INVALID), (dict(k=(1 << 30) + 8), INVALID), (dict(v=(2 << 30) + 4), INVALID),
    (dict(n=1 << 23), UNSUPPORTED), (dict(ws=None), WORKSPACE), (dict(ws_bytes=100), WORKSPACE), (dict(ws=(3 << 33) + 16), WORKSPACE),
    (dict(band=(0, 0, MB, MB)), INVALID), (dict(band=(-1, 5, MB, MB)), INVALID), (dict(band=(1000, 25, MB, MB)), INVALID),
    (dict(band=(4, 4, None, MB)), INVALID), (dict(band=(4, 4, MB, MB + 8)), INVALID),
])
def test_attention_refusals(kw, status):
    assert attend(**kw) == status
    assert nat.lib().nova_kv_last_error()


def test_attention_refuses_bad_layers_and_layouts():
    for kw, status in ((dict(head_dim=96), UNSUPPORTED), (dict(group_dim=8), INVALID), (dict(codebook_size=128), UNSUPPORTED), (dict(flags=16), UNSUPPORTED),
                       (dict(t_k_inv_t=None), INVALID), (dict(t_v=None), INVALID), (dict(cb_k=None), INVALID), (dict(cb_v=5 * MB + 8), INVALID),
                       (dict(kbar=MB + 4), INVALID), (dict(flags=nat.NOVA_KV_KEY_SCALE), INVALID), (dict(flags=nat.NOVA_KV_SQ_VALUES), INVALID)):
        assert attend(params(**kw)) in ((status, UNSUPPORTED) if "group_dim" in kw else (status,)), kw
    assert attend(params(flags=nat.NOVA_KV_KEY_SCALE), ks=MB + 1) == INVALID
    assert attend(params(flags=nat.NOVA_KV_SQ_VALUES), sq=MB + 2) == INVALID
    for kw in (dict(block_size=0), dict(blocks_per_seq=0), dict(block_size=1 << 16, blocks_per_seq=1 << 16)):
        assert attend(lay=layout(**kw)) == INVALID
    assert nat.lib().nova_kv_chunk_attn(None, *[None] * 2, 1, 1, 1, 8, *[None] * 7, 1, 0, None, 0.0, None, None, 0, None) == INVALID


def test_workspace_query():
    lib = nat.lib()
    size = lambda *a, **kw: lib.nova_kv_chunk_attn_workspace_bytes(ref(params(**kw)), *a)  # noqa: E731
    assert size(1, 1, 32, 4096) > 0 and size(1, 1, 32, 4096) % 256 == 0
    assert size(0, 1, 32, 4096) == size(1, 0, 32, 4096) == size(1, 1, 12, 4096) == size(1, 1, 32, 0) == 0
    assert size(1, 1, 32, (1 << 30) + 1) == size(1, 2 ** 31 - 1, 32, 4096) == size(65536, 1, 32, 4096) == size(1, 1, 32, 4096, head_dim=96) == 0
    assert lib.nova_kv_chunk_attn_workspace_bytes(None, 1, 1, 32, 4096) == 0
    for shape in ((1, 1), (3, 5), (1, 300)):
        got = [size(*shape, 32, s) for s in (1, 64, 300, 1000, 4096, 100000)]
        assert got == sorted(got)


def read(p=None, lay=None, **kw):
    a = dict(k=1 << 30, v=2 << 30, ks=None, sq=None, band=None, seq=None, dtype=nat.NOVA_KV_BF16, batch=2, n=100, start=8 * MB, lens=None,
             k_out=1 << 33, v_out=2 << 33)
    a.update(kw)
    band = None if a["band"] is None else nat.Band(*a["band"])
    return nat.lib().nova_kv_read(ref(params() if p is None else p), ref(layout() if lay is None else lay), a["k"], a["v"], a["ks"], a["sq"],
                                  ref(band), a["seq"], a["dtype"], a["batch"], a["n"], a["start"], a["lens"], a["k_out"], a["v_out"], None)


def read4(c=None, **kw):
    a = dict(dtype=nat.NOVA_KV_BF16, batch=2, n=100, start=8 * MB, lens=None, k_out=1 << 33, v_out=2 << 33)
    a.update(kw)
    return nat.lib().nova_kv_q4_read(ref(cache() if c is None else c), a["dtype"], a["batch"], a["n"], a["start"], a["lens"], a["k_out"],
                                     a["v_out"], None)


@pytest.mark.parametrize("call", (read, read4))
@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), INVALID), (dict(batch=-1), INVALID), (dict(n=-1), INVALID), (dict(batch=65536), INVALID), (dict(start=None), INVALID),
    (dict(k_out=(1 << 33) + 8), INVALID), (dict(v_out=(2 << 33) + 2), INVALID), (dict(v_out=(1 << 33) + 4096), INVALID),
    (dict(k_out=(2 << 33) + 2 * 100 * 8 * 128 * 2 - 16), INVALID), (dict(n=1 << 30), UNSUPPORTED),
])
def test_read_refusals(call, kw, status):
    assert call(**kw) == status
    assert nat.lib().nova_kv_last_error()


def test_read_refuses_more_heads_than_a_round_holds():
    more = dict(n=1, k_out=1 << 40, v_out=2 << 40)
    assert read(params(num_kv_heads=4097), **more) == UNSUPPORTED and "4096" in nat.lib().nova_kv_last_error().decode()


def test_read_refuses_bad_caches():
    assert read(k=None) == read(v=None) == read(k=(1 << 30) + 8) == INVALID
    assert read(params(flags=nat.NOVA_KV_KEY_SCALE)) == read(params(flags=nat.NOVA_KV_SQ_VALUES)) == INVALID
    assert read(band=(4, 4, MB, MB)) == INVALID                        # without lengths
    assert read(band=(0, 0, MB, MB), seq=MB) == INVALID and read(params(head_dim=32)) == UNSUPPORTED
    assert read(lay=layout(block_size=0)) == INVALID and read4(cache(head_dim=256)) == UNSUPPORTED and read4(cache(k_sq=None)) == INVALID
    assert nat.lib().nova_kv_q4_read(None, 1, 1, 1, None, None, None, None, None) == INVALID


def axes_call(append, ax=None, r=None, **kw):
    a = dict(positions=9 * MB, batch=2, n=100, start=5 * MB, axes=nat.Axes(3, (ctypes.c_uint8 * 64)(*[0, 1, 2] * 21)) if ax is None else ax)
    a.update(kw)
    r = rotary() if r is None else r
    x = [ref(t) for t in (rows(FUSED), rows(FUSED + 8192), rows(FUSED + 8192 + 2048))]
    outs = (6 << 30, 7 << 30, 8 << 30)
    if append:
        return nat.lib().nova_kv_q4_append_axes(ref(r), ref(a["axes"]), ref(cache()), *x, 1, a["batch"], a["n"], None, a["start"],
                                                a["positions"], *outs, None)
    return nat.lib().nova_kv_rotate_qkv_axes(ref(r), ref(a["axes"]), *x, 1, a["batch"], a["n"], None, a["positions"], *outs, None)


@pytest.mark.parametrize("append", (False, True))
def test_axes_refusals(append):
    of = lambda m, *pairs: nat.Axes(m, (ctypes.c_uint8 * 64)(*pairs))  # noqa: E731
    for kw in (dict(ax=of(0)), dict(ax=of(5)), dict(ax=of(-1)), dict(ax=of(2, *[0] * 63, 2)), dict(ax=of(1, 0, 255)), dict(positions=None),
               dict(r=rotary(rotary_dim=0, cos_sin=None)), dict(r=rotary(rotary_dim=136)), dict(batch=-1), dict(batch=70000)):
        assert axes_call(append, **kw) == INVALID, kw
    null = [None] * 3
    if append:
        assert axes_call(True, start=None) == INVALID
        assert nat.lib().nova_kv_q4_append_axes(ref(rotary()), None, ref(cache()), *[ref(rows(FUSED))] * 3, 1, 2, 5, None, MB, MB, 6 << 30,
                                                7 << 30, 8 << 30, None) == INVALID
    else:
        assert nat.lib().nova_kv_rotate_qkv_axes(ref(rotary()), None, ref(rows(FUSED)), None, None, 1, 2, 5, None, MB, 6 << 30, None, None, None) == INVALID
        assert nat.lib().nova_kv_rotate_qkv_axes(ref(rotary()), None, *null, 1, 2, 5, None, None, *null, None) == OK


def test_no_ops():
    assert attend(batch=0, q=None) == OK and attend(n=0, out=None) == OK
    for call in (read, read4):
        assert call(batch=0, start=None) == call(n=0) == call(k_out=None, v_out=None, start=None) == OK
    assert axes_call(False, batch=0, positions=None) == axes_call(True, n=0, positions=None) == OK


def test_binding_refusals():
    """Shapes, types and devices, before any pointer is handed over (CPU tensors are refused)."""
    for make in (lambda: nk.RotaryAxes([]), lambda: nk.RotaryAxes([0] * 65), lambda: nk.RotaryAxes([0, 4]), lambda: nk.RotaryAxes([0, -1]),
                 lambda: nk.RotaryAxes([0, 1], num_axes=1), lambda: nk.RotaryAxes([0], num_axes=5)):
        with pytest.raises(ValueError):
            make()
    assert nk.RotaryAxes.cycle((3, 1, 2)).pair_axis == (0, 1, 2, 0, 2, 0) and nk.RotaryAxes.blocks((1, 2)).pair_axis == (0, 1, 1)
    assert list(nk.RotaryAxes.blocks((1, 2)).c.pair_axis)[:3] == [0, 1, 1] and nk.RotaryAxes([0, 0], num_axes=3).num_axes == 3
    x = torch.zeros(2, 3, 8, 128)
    with pytest.raises((ValueError, TypeError)):
        nk.rotate_qkv_axes(nk.Rotary(32, 8, 128), nk.RotaryAxes([0]), None, x, None, torch.zeros(1, 2, 3, dtype=torch.int32))


def test_oracle_formulas():
    """The oracle's parts against the same sums written out one by one."""
    rng = np.random.default_rng(0)
    L, S = 3, 5
    book = rng.standard_normal((L, 256, 4))
    codes = rng.integers(0, 256, (S, L)).astype(np.uint8)
    words, lev = oracle.codewords(book, codes), oracle.levels(codes)
    for t in range(S):
        for i in range(4 * L):
            assert words[t, i] == book[i // 4, codes[t, i // 4], i % 4]
            assert lev[t, i] == (codes[t, i // 4] // 4 ** (i % 4)) % 4
    head = {"cb_k": book, "cb_v": book, "kbar": rng.standard_normal(12), "t_k_inv_t": rng.standard_normal((12, 12)), "t_v": rng.standard_normal((12, 12))}
    rho, grid = rng.random(S), rng.standard_normal((S, 2))
    k, v, r, s = oracle.cached_rows(head, codes, codes, rho, grid)
    for t in range(S):
        for i in range(12):
            assert abs(k[t, i] - sum(rho[t] * words[t, j] * head["t_k_inv_t"][i, j] for j in range(12)) - head["kbar"][i]) < 1e-12
            assert abs(v[t, i] - sum((grid[t, 1] + grid[t, 0] * lev[t, j]) * head["t_v"][i, j] for j in range(12))) < 1e-12
    # a logit through the transform's coordinates is the logit over the row that is read back
    q = rng.standard_normal(12)
    assert np.allclose(r @ (q @ head["t_k_inv_t"]) + q @ head["kbar"], k @ q)
    out = oracle.attend(q[None, None], k, v, np.array([3]), window=2, sinks=np.array([0.3]))
    z = np.array([q @ k[j] / np.sqrt(12) for j in (2, 3)])
    w = np.exp(z) / (np.exp(z).sum() + np.exp(0.3))
    assert np.allclose(out[0, 0], w @ v[2:4]) and not oracle.attend(q[None, None], k, v, np.array([-1])).any()
    table = rng.standard_normal((7, 4))
    pos = rng.integers(0, 7, (2, 3))
    rows_of = oracle.axis_angles(table, (1, 0), pos)
    for i in range(3):
        assert rows_of[i].tolist() == [table[pos[1, i], 0], table[pos[0, i], 1], table[pos[1, i], 2], table[pos[0, i], 3]]


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ is not installed")
def test_checks_under_sanitizers(tmp_path):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    exe = tmp_path / "read_checks"
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", "-fsanitize=address,undefined",
                    "-fno-sanitize-recover=all", "-I", os.path.join(root, "include"),
                    os.path.join(root, "paper_2608_04074_amd", "csrc", "host_checks.cpp"),
                    os.path.join(root, "tests", "asan", "read_checks_driver.cpp"), "-o", str(exe)], check=True)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0:verify_asan_link_order=0", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([str(exe)], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0, r.stderr[-4000:]
