"""The tiles that the vocabulary loss's products take (host code built with g++, no GPU)."""
from __future__ import annotations

import os
import shutil
import subprocess

import pytest

from loss_shapes import SIZES

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("g++ not available")
    exe = str(tmp_path_factory.mktemp("cut") / "vocab_cut_test")
    subprocess.run(["g++", "-O1", "-g", "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                    "-I", os.path.join(ROOT, "paper_2603_11438_amd", "csrc"), os.path.join(ROOT, "tests", "native", "vocab_cut_test.cpp"), "-o", exe],
                   check=True, capture_output=True, text=True)
    return exe


def products(exe, size):
    """{(product, tile, whether k is split)}."""
    out = subprocess.run([exe, *map(str, size)], capture_output=True, text=True, check=True).stdout
    return {(name, int(tile), int(runs) > 1) for name, tile, runs in map(str.split, out.splitlines())}


def test_tested_sizes_reach_every_tile(exe):
    """Every kernel that the rule can choose is run by a test against 64 bits."""
    both = (False, True)
    found = set().union(*(products(exe, s) for s in SIZES))
    wanted = {(name, tile, False) for name in ("stats", "dz") for tile in range(-1, 5)}
    wanted |= {(name, tile, split) for name in ("dx", "dw") for tile in range(5) for split in both}
    # a product of several pieces has many rows of dz: tiles of 64 only with k in runs
    wanted |= {(name, tile, split) for name in ("dx_first", "dx_more") for tile in range(1, 5) for split in both}
    wanted |= {(name, 0, True) for name in ("dx_first", "dx_more")}
    assert not wanted - found, sorted(wanted - found)


def test_a_large_training_step_takes_tiles_that_are_tested(exe):
    """4096 tokens of 4096 over 131072 classes: 256 x 256 throughout, in two pieces."""
    taken = products(exe, (4096, 4096, 131072))
    assert taken == {(name, 3, False) for name in ("stats", "dz", "dx_first", "dx_more", "dw")}
    assert taken <= set().union(*(products(exe, s) for s in SIZES))
