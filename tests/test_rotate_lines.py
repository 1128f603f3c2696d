"""Which layouts of a rotated row's stores may be streamed, enumerated on the host: those of whole lines."""

import os
import shutil
import subprocess

import pytest


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ is not installed")
def test_streamed_stores_write_whole_lines(tmp_path):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    exe = tmp_path / "rotate_lines"
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", os.path.join(root, "tests", "asan", "rotate_lines_driver.cpp"), "-o", str(exe)],
                   check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout[-2000:]
