"""Launch attributes are set for each device, and a failure to set one is not
remembered (host code built with g++, no GPU)."""
from __future__ import annotations

import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2603_11438_amd", "csrc")


def test_once_per_device(tmp_path):
    if not shutil.which("g++"):
        pytest.skip("g++ not available")
    exe = str(tmp_path / "once_per_device_test")
    subprocess.run(["g++", "-O1", "-g", "-std=c++17", "-pthread", "-fsanitize=thread", "-I", CSRC,
                    os.path.join(ROOT, "tests", "native", "once_per_device_test.cpp"), "-o", exe],
                   check=True, capture_output=True, text=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "once per device: ok" in r.stdout, r.stdout + r.stderr


def test_no_attribute_is_set_once_for_all_devices():
    for name in sorted(os.listdir(CSRC)):
        if name.endswith((".hip", ".h", ".cpp")):
            text = open(os.path.join(CSRC, name)).read()
            assert not re.search(r"static\b[^;]*=\s*hipFuncSetAttribute", text), name
