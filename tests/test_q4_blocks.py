"""Debug mode of the 4-bit cache's calls: negative block-table entries hold nothing and pass, entries past the pool
are reported."""

import os
import shutil
import subprocess

import pytest


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ is not installed")
def test_metadata_check_under_sanitizers(tmp_path):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    exe = tmp_path / "q4_blocks"
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", "-fsanitize=address,undefined",
                    "-fno-sanitize-recover=all", "-I", os.path.join(root, "include"),
                    os.path.join(root, "paper_2608_04074_amd", "csrc", "host_checks.cpp"),
                    os.path.join(root, "tests", "asan", "q4_blocks_driver.cpp"), "-o", str(exe)], check=True)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0:verify_asan_link_order=0", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([str(exe)], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0, r.stderr[-4000:]


@pytest.mark.gpu
def test_blocks_not_held_pass_debug_mode():
    import torch
    import paper_2608_04074_amd as nk
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    table = i32([[-1, 0, 1], [4, 5, -1]])      # a block released in front of the window, and one not held yet
    cache = nk.Q4Cache.zeros(nk.CacheLayout(16, 3, table), 2, 2, 64, num_blocks=6)
    k = torch.randn((2, 4, 2, 64), dtype=torch.bfloat16, device="cuda")
    q = torch.randn((2, 4, 4, 64), dtype=torch.bfloat16, device="cuda")
    call = lambda: (nk.q4_append(nk.Rotary(4, 2, 64), cache, q, k, k, i32([40, 30])),  # noqa: E731
                    nk.q4_attn(cache, q, i32([44, 34]), 48, window=8))
    want = call()
    try:
        nk.set_debug(True)
        got = call()
        table[1, 1] = 6
        with pytest.raises(nk.NovaKVError, match="physical block 6"):
            call()
    finally:
        nk.set_debug(False)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
