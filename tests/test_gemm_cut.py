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


def products(exe, *call):
    """{(product, tile, whether k is split)} of a call."""
    out = subprocess.run([exe, *map(str, call)], capture_output=True, text=True, check=True).stdout
    return {(name, int(tile), int(runs) > 1) for name, tile, runs in map(str.split, out.splitlines())}


def test_tested_sizes_reach_every_tile(exe):
    """Every kernel that the rule can choose is run by a test: the sizes of
    tests/gemm_shapes.py, on the GPU against 64 bits."""
    from gemm_shapes import FFN, ORTHO

    both = (False, True)
    found = set().union(*(products(exe, "ffn", *s) for s in FFN))
    wanted = {(name, tile, split) for name in ("dx", "dw") for tile in range(5) for split in both}
    wanted |= {("forward", tile, split) for tile in (-1, 1, 4) for split in both} | {("forward", 3, False)}
    assert not wanted - found, sorted(wanted - found)
    for planes in (1, 2):
        found = set().union(*(products(exe, "ortho", planes, min(m, n), max(m, n), b) for p, m, n, b in ORTHO if p == planes))
        wanted = {("a", tile, split) for tile in range(4) for split in both} | {(name, tile, False) for name in "bx" for tile in range(4)}
        assert not wanted - found, (planes, sorted(wanted - found))
