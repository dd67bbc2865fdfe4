"""The native part of the operators' binding is a shortcut: without it, or with
one built against another torch, the checks in Python run instead, with a
warning (no GPU)."""
from __future__ import annotations

import pytest
import torch

import paper_2603_11438_amd as ar
from paper_2603_11438_amd import ops


@pytest.fixture
def fresh(monkeypatch):
    monkeypatch.setattr(ops, "_native_path", None)
    return monkeypatch


def _refused_in_python():
    x = torch.ones(4, 16)
    for call in (lambda: ar.residual_norm(x, x), lambda: ar.residual_norm_backward(x, x, None, x),
                 lambda: ar.gated_ffn(x.bfloat16(), x.bfloat16(), x.bfloat16()), lambda: ar.orthogonalize(x)):
        with pytest.raises(ValueError):
            call()


def test_built_against_the_loaded_torch(fresh):
    ops._native()  # None without a device context, but loaded
    assert ops._native_path
    _refused_in_python()


def test_not_built(fresh, tmp_path):
    fresh.setattr(ops, "OPS_ARGS_PATH", str(tmp_path / "absent.so"))
    with pytest.warns(RuntimeWarning, match="not built"):
        assert ops._native() is None
    _refused_in_python()


def test_built_against_another_torch(fresh):
    fresh.setattr(torch, "__version__", "0.0.1")
    with pytest.warns(RuntimeWarning, match="0.0.1"):
        assert ops._native() is None
    _refused_in_python()


def test_cannot_be_loaded(fresh, tmp_path):
    bad = tmp_path / "_ops_args.so"
    bad.write_bytes(b"not a library")
    fresh.setattr(ops, "OPS_ARGS_PATH", str(bad))
    with pytest.warns(RuntimeWarning):
        assert ops._native() is None
    _refused_in_python()
