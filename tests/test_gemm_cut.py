"""The tiles that the operators' products take (host code built with g++, no GPU)."""
from __future__ import annotations

import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("g++ not available")
    exe = str(tmp_path_factory.mktemp("cut") / "gemm_cut_test")
    subprocess.run(["g++", "-O1", "-g", "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                    "-I", os.path.join(ROOT, "paper_2603_11438_amd", "csrc"),
                    os.path.join(ROOT, "tests", "native", "gemm_cut_test.cpp"), "-o", exe],
                   check=True, capture_output=True, text=True)
    return exe


def test_forward_takes_the_cheapest_shape_there_is(exe):
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "gemm cut: ok" in r.stdout, r.stdout + r.stderr
