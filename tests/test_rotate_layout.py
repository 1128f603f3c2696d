"""Stores of a row's 4-bit codes, enumerated on the host for every rotary_dim: aligned, and each byte once."""

import os
import shutil
import subprocess

import pytest


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ is not installed")
def test_code_stores(tmp_path):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    exe = tmp_path / "rotate_layout"
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", os.path.join(root, "tests", "asan", "rotate_layout_driver.cpp"), "-o", str(exe)],
                   check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout[-2000:]
