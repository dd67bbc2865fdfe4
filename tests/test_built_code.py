"""What the device code of the built library may rely on, held against its
disassembly (no GPU)."""
from __future__ import annotations

import os
import re
import shutil
import subprocess

import pytest

import paper_2603_11438_amd as ar

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"


@pytest.fixture(scope="module")
def listings(tmp_path_factory):
    """The instructions of each of the library's code objects, one a line."""
    if not os.path.exists(OBJDUMP):
        pytest.skip("llvm-objdump not available")
    if not os.path.exists(ar.LIB_PATH):
        import __graft_entry__

        __graft_entry__.build()
    at = tmp_path_factory.mktemp("code")
    shutil.copy(ar.LIB_PATH, at / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=at, check=True, capture_output=True)
    objects = sorted(p for p in at.iterdir() if "gfx950" in p.name and p.stat().st_size)
    assert objects
    found = []
    for p in objects:
        r = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", str(p)], check=True, capture_output=True, text=True)
        found.append([re.sub(r"\s*//.*", "", line).strip() for line in r.stdout.splitlines()])
    return found


SET = re.compile(r"s_mov_b32 m0, s\d+")


def test_m0_is_the_loads_to_lds_alone(listings):
    """The loads into LDS set m0 in assembly that cannot say so to the compiler: no
    other instruction may write it or read it."""
    loads = 0
    for lines in listings:
        for k, line in enumerate(lines):
            if re.search(r"\bm0\b", line):
                assert SET.fullmatch(line), line
                assert lines[k + 1] == "s_nop 0" and re.fullmatch(r"buffer_load_dwordx4 .* offen lds", lines[k + 2]), lines[k:k + 3]
                loads += 1
        # readers that do not name it
        hidden = [line for line in lines if re.match(r"s_sendmsg|s_movrel|v_movrel|ds_gws|s_ttracedata|ds_\w*addtid|v_interp", line)]
        assert not hidden, hidden[:3]
        assert sum(line.endswith(" lds") for line in lines) == sum(bool(SET.fullmatch(line)) for line in lines)
    assert loads, "no load sets m0 any more: this test has nothing to hold"
