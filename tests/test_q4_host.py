"""Argument checks of the norm, rotation and 4-bit cache calls that need no GPU.

Every call here is rejected by the host-side checks (or is a no-op) before any
HIP call, so nothing touches a device."""

import ctypes
import os
import shutil
import subprocess

import pytest
import torch

import paper_2608_04074_amd as nk
from paper_2608_04074_amd import _native as nat

OK, INVALID, UNSUPPORTED, WORKSPACE = (nat.NOVA_KV_OK, nat.NOVA_KV_ERR_INVALID_ARG, nat.NOVA_KV_ERR_UNSUPPORTED,
                                       nat.NOVA_KV_ERR_WORKSPACE)
MB = 1 << 20


def rotary(**kw):
    a = dict(num_q_heads=32, num_kv_heads=8, head_dim=128, rotary_dim=128, interleaved=0, num_positions=4096,
             cos_sin=MB, q_norm=2 * MB, k_norm=3 * MB, q_norm_per_head=0, k_norm_per_head=1, eps=1e-6)
    a.update(kw)
    return nat.Rotary(**a)


def cache(**kw):
    lay = dict(block_size=16, blocks_per_seq=256, block_table=4 * MB)
    lay.update({k: kw.pop(k) for k in list(kw) if k in lay})
    a = dict(num_kv_heads=8, head_dim=128, num_blocks=1024, layout=nat.Layout(**lay), k_codes=1 << 30, v_codes=2 << 30,
             k_sq=3 << 30, v_sq=4 << 30)
    a.update(kw)
    return nat.Q4Cache(**a)


def rows(data, bs=100 * 6144, ts=6144):
    return nat.Rows(data, bs, ts)


def ref(x):
    return None if x is None else ctypes.byref(x)


FUSED = 5 << 30


def tokens(append, r=None, c=None, **kw):
    """nova_kv_q4_append (append) or nova_kv_rotate_qkv with one argument changed."""
    a = dict(q=rows(FUSED), k=rows(FUSED + 8192), v=rows(FUSED + 8192 + 2048), dtype=nat.NOVA_KV_BF16, batch=2, n=100, lens=None,
             start=5 * MB, q_out=6 << 30, k_out=7 << 30, v_out=8 << 30)
    a.update(kw)
    r = rotary() if r is None else r
    tail = [ref(a["q"]), ref(a["k"]), ref(a["v"]), a["dtype"], a["batch"], a["n"], a["lens"], a["start"], a["q_out"], a["k_out"], a["v_out"], None]
    if append:
        return nat.lib().nova_kv_q4_append(ref(r), ref(cache() if c is None else c), *tail)
    return nat.lib().nova_kv_rotate_qkv(ref(r), *tail)


@pytest.mark.parametrize("append", (False, True))
@pytest.mark.parametrize("kw,status", [
    (dict(num_q_heads=0), INVALID), (dict(num_kv_heads=0), INVALID), (dict(num_q_heads=12), INVALID),
    (dict(num_q_heads=1 << 20), UNSUPPORTED), (dict(head_dim=96), UNSUPPORTED), (dict(rotary_dim=-8), INVALID),
    (dict(rotary_dim=136), INVALID), (dict(rotary_dim=20), UNSUPPORTED), (dict(interleaved=2), INVALID),
    (dict(cos_sin=None), INVALID), (dict(num_positions=0), INVALID), (dict(cos_sin=MB + 4), INVALID),
    (dict(q_norm=MB + 4), INVALID), (dict(k_norm=MB + 8), INVALID), (dict(k_norm_per_head=2), INVALID),
    (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID),
])
def test_rotary_refusals(append, kw, status):
    assert tokens(append, r=rotary(**kw)) == status
    assert nat.lib().nova_kv_last_error()


@pytest.mark.parametrize("append", (False, True))
@pytest.mark.parametrize("kw,status", [
    (dict(batch=-1), INVALID), (dict(n=-1), INVALID), (dict(batch=65536), INVALID), (dict(dtype=2), INVALID),
    (dict(batch=60000, n=1000), UNSUPPORTED), (dict(start=None), INVALID),
    (dict(q=rows(None)), INVALID), (dict(k=rows(FUSED + 1)), INVALID), (dict(v=rows(FUSED, -6144)), INVALID),
    (dict(v=rows(FUSED, 1 << 41)), INVALID), (dict(q=rows(FUSED, 0, -1)), INVALID),
    (dict(q_out=None), INVALID), (dict(q=None), INVALID), (dict(q_out=(6 << 30) + 8), INVALID), (dict(v_out=(8 << 30) + 2), INVALID),
    (dict(dtype=nat.NOVA_KV_F32, k=rows(FUSED + 2)), INVALID),
    # outputs over each other, over other rows, over their own strided rows
    (dict(k_out=(6 << 30) + 4096), INVALID), (dict(v_out=(7 << 30) + 16 * 128), INVALID),
    (dict(q_out=FUSED), INVALID), (dict(k_out=FUSED + 16), INVALID),
    (dict(q=rows(6 << 30, 100 * 4096, 4096), q_out=(6 << 30) + 16), INVALID),
])
def test_token_refusals(append, kw, status):
    assert tokens(append, **kw) == status


def test_append_refusals():
    for kw, status in ((dict(num_kv_heads=4), INVALID), (dict(head_dim=64), INVALID), (dict(num_blocks=0), INVALID),
                       (dict(head_dim=32), UNSUPPORTED), (dict(block_size=0), INVALID), (dict(blocks_per_seq=0), INVALID),
                       (dict(k_codes=None), INVALID), (dict(v_sq=None), INVALID), (dict(v_codes=(2 << 30) + 8), INVALID),
                       (dict(k_sq=(3 << 30) + 2), INVALID), (dict(num_blocks=1 << 26), UNSUPPORTED),
                       (dict(block_size=1 << 16, blocks_per_seq=1 << 16), INVALID)):
        assert tokens(True, c=cache(**kw)) == status, kw
    assert tokens(True, k=None, k_out=None) == INVALID
    assert tokens(True, v=None, v_out=None) == INVALID
    assert nat.lib().nova_kv_q4_append(ref(rotary()), None, *[None] * 3, 1, 1, 1, *[None] * 6) == INVALID
    assert tokens(False, r=nat.Rotary()) == INVALID


def test_no_ops():
    assert tokens(False, batch=0, q=None, q_out=None) == OK and tokens(True, n=0, k=None, k_out=None) == OK
    assert tokens(False, q=None, k=None, v=None, q_out=None, k_out=None, v_out=None) == OK
    assert attn(batch=0, q=None) == OK and attn(n=0, out=None) == OK


def attn(c=None, **kw):
    a = dict(q=1 << 33, dtype=nat.NOVA_KV_BF16, batch=2, n=3, hq=32, q_lens=None, seq=5 * MB, max_seq=4096, window=0, sinks=None,
             scale=0.0, out=2 << 33, ws=3 << 33, ws_bytes=1 << 32)
    a.update(kw)
    return nat.lib().nova_kv_q4_attn(ref(cache() if c is None else c), a["q"], a["dtype"], a["batch"], a["n"], a["hq"], a["q_lens"],
                                     a["seq"], a["max_seq"], a["window"], a["sinks"], a["scale"], a["out"], a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=9), INVALID), (dict(batch=-1), INVALID), (dict(n=-1), INVALID), (dict(batch=70000), INVALID),
    (dict(hq=0), INVALID), (dict(hq=12), INVALID), (dict(max_seq=0), INVALID), (dict(max_seq=4097), INVALID),
    (dict(window=-1), INVALID), (dict(scale=-0.5), INVALID), (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID),
    (dict(q=None), INVALID), (dict(seq=None), INVALID), (dict(out=None), INVALID), (dict(q=(1 << 33) + 8), INVALID),
    (dict(out=(2 << 33) + 4), INVALID), (dict(n=1 << 23), UNSUPPORTED), (dict(ws=None), WORKSPACE), (dict(ws_bytes=100), WORKSPACE),
    (dict(ws=(3 << 33) + 16), WORKSPACE),
])
def test_attn_refusals(kw, status):
    assert attn(**kw) == status


def test_attn_refuses_bad_caches():
    assert nat.lib().nova_kv_q4_attn(None, *[None] * 1, 1, 1, 1, 8, None, None, 1, 0, None, 0.0, None, None, 0, None) == INVALID
    for kw, status in ((dict(head_dim=256), UNSUPPORTED), (dict(k_sq=None), INVALID), (dict(num_kv_heads=0), INVALID)):
        assert attn(cache(**kw)) == status


def test_workspace_query():
    lib = nat.lib()
    size = lambda *a: lib.nova_kv_q4_attn_workspace_bytes(ref(cache()), *a)  # noqa: E731
    assert size(1, 1, 32, 4096) > 0 and size(1, 1, 32, 4096) % 256 == 0
    assert size(0, 1, 32, 4096) == size(1, 0, 32, 4096) == size(1, 1, 12, 4096) == size(1, 1, 32, 0) == 0
    assert lib.nova_kv_q4_attn_workspace_bytes(None, 1, 1, 32, 4096) == 0
    for shape in ((1, 1), (3, 5), (1, 300)):
        got = [size(*shape, 32, s) for s in (1, 64, 300, 1000, 4096)]
        assert got == sorted(got)


def test_binding_refusals():
    """Shapes, types and devices, before any pointer is handed over (CPU tensors are refused)."""
    x = torch.zeros(2, 3, 8, 128)
    r = nk.Rotary(32, 8, 128)
    for call in (lambda: nk.rotate_qkv(r, None, x, None, None), lambda: nk.rotate_qkv(r, None, None, None, None),
                 lambda: nk.rotate_qkv(r, None, x[0], None, None), lambda: nk.Rotary(32, 8, 128, cos_sin=x[0, 0]),
                 lambda: nk.Rotary(32, 8, 128, q_norm=torch.zeros(128)),
                 lambda: nk.Q4Cache.zeros(nk.CacheLayout.contiguous(16), 1, 8, 128, device="cpu")):
        with pytest.raises((ValueError, TypeError)):
            call()
    assert nk.q4_code_shape(8, 128, nk.CacheLayout(16, 4), 2) == (8, 8, 16, 64)
    assert nk.q4_sq_shape(8, nk.CacheLayout(16, 4), 2, 11) == (11, 8, 16, 2)


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ is not installed")
def test_checks_under_sanitizers(tmp_path):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    exe = tmp_path / "q4_checks"
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", "-fsanitize=address,undefined",
                    "-fno-sanitize-recover=all", "-I", os.path.join(root, "include"),
                    os.path.join(root, "paper_2608_04074_amd", "csrc", "host_checks.cpp"),
                    os.path.join(root, "tests", "asan", "q4_checks_driver.cpp"), "-o", str(exe)], check=True)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0:verify_asan_link_order=0", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([str(exe)], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0, r.stderr[-4000:]


def test_workspace_query_of_refused_calls():
    """The workspace query returns 0 for calls of too many rows, of lengths past any capacity and of other heads."""
    size = lambda *a, **kw: nat.lib().nova_kv_q4_attn_workspace_bytes(ref(cache(**kw)), *a)  # noqa: E731
    assert size(1, 1, 32, 1 << 30) > 0
    assert size(1, 1, 32, (1 << 30) + 1) == size(1, 2 ** 31 - 1, 32, 4096) == 0
    assert size(65536, 1, 32, 4096) == size(65535, 65535, 32, 4096) == size(1, 1, 32, 4096, head_dim=96) == 0
