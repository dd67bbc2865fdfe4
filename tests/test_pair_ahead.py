"""Which of the 256 x 256 tiles the gated feed-forward block's forward takes (host code
built with g++, no GPU)."""
from __future__ import annotations

import os
import shutil
import subprocess

import pytest

from gemm_shapes_ahead import BOTH

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LARGE = 3


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("g++ not available")
    exe = str(tmp_path_factory.mktemp("ahead") / "pair_ahead_test")
    subprocess.run(["g++", "-O1", "-g", "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                    "-I", os.path.join(ROOT, "paper_2603_11438_amd", "csrc"), os.path.join(ROOT, "tests", "native", "pair_ahead_test.cpp"), "-o", exe],
                   check=True, capture_output=True, text=True)
    return exe


def taken(exe, t, d, f, saved):
    tile, ahead = map(int, subprocess.run([exe, *map(str, (t, d, f, int(saved)))], capture_output=True, text=True, check=True).stdout.split())
    return tile, bool(ahead)


@pytest.mark.parametrize("saved,size,ahead", [
    # measured, us with two buffers and with three: 357, 367; 416, 424; 616, 636
    (False, (8192, 1024, 11264), False), (False, (4096, 4096, 8192), False), (False, (6144, 4096, 8192), False), (False, (16384, 2048, 4096), False),
    # 1212, 1180; 487, 459; 881, 850; 1080, 1018
    (False, (8192, 4096, 11264), True), (False, (2048, 6144, 11264), True), (False, (8192, 4096, 8192), True), (False, (16384, 2304, 8192), True),
    # 470, 458; 170, 162
    (True, (8192, 1024, 11264), True), (True, (4096, 768, 8192), True)])
def test_as_measured(exe, saved, size, ahead):
    assert taken(exe, *size, saved) == (LARGE, ahead)


def test_tested_sizes_reach_both(exe):
    for _, *size in BOTH:
        assert taken(exe, *size, False) == (LARGE, False) and taken(exe, *size, True) == (LARGE, True)
