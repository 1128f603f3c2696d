"""Debug mode of chunk attention passes what the call does not look up: table entries in front of a window, of
positions that only a band holds, and of sequences without queries."""

import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from chunk_cases import Cache


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ is not installed")
def test_attended_blocks_under_sanitizers(tmp_path):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    exe = tmp_path / "attended_checks"
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", "-fsanitize=address,undefined",
                    "-fno-sanitize-recover=all", "-I", os.path.join(root, "include"),
                    os.path.join(root, "paper_2608_04074_amd", "csrc", "host_checks.cpp"),
                    os.path.join(root, "tests", "asan", "attended_checks_driver.cpp"), "-o", str(exe)], check=True)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0:verify_asan_link_order=0", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([str(exe)], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0, r.stderr[-4000:]


@pytest.mark.gpu
@pytest.mark.parametrize("n", (2, 20, 70))
def test_debug_mode_passes_released_blocks(n):
    import paper_2608_04074_amd as nk
    c = Cache(nk, 6, [700, 400, 90], 2, 64, 16, "band")
    q = torch.as_tensor(np.random.default_rng(n).standard_normal((3, n, 8, 64))).to(torch.bfloat16).cuda()
    q_lens = torch.tensor([n, n - 1, 0], dtype=torch.int32, device="cuda")
    run = lambda w: nk.chunk_attn(c.params, c.layout, q, c.k_codes, c.v_codes, c.seq_lens, c.top, q_lens=q_lens, window=w, **c.more)  # noqa: E731
    want = [run(w) for w in (90, 0)]
    table, blocks = c.layout.block_table, c.k_codes.shape[0]
    kept = table.clone()
    try:
        nk.set_debug(True, blocks)
        for w, ref in zip((90, 0), want):
            table.copy_(kept)
            for b, S in enumerate(c.seqs[:2]):
                low = max(0, S - (n - b) + 1 - w) if w else 5
                table[b, :max(low, 5) // 16] = -5
                table[b, -(-(S - 40) // 16):] = 2 ** 30
            table[2] = -1
            assert torch.equal(run(w), ref)
            for b, S in enumerate(c.seqs[:2]):  # the first and the last block that are attended
                low = max(0, S - (n - b) + 1 - w) if w else 5
                for block in (max(low, 5) // 16, (S - 41) // 16):
                    held = table[b, block].clone()
                    table[b, block] = blocks
                    with pytest.raises(nk.NovaKVError, match=f"sequence {b}: block {block} maps to physical block {blocks}"):
                        run(w)
                    table[b, block] = held
    finally:
        nk.set_debug(False)
