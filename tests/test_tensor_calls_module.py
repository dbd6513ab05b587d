"""The extension module that marshals torch tensors for the operators between the linear layers: who needs it, when it is
built (no GPU, nothing is compiled here)."""
import subprocess
import sys

import pytest
import torch

from paper_2508_18182_b200 import binding as A
from paper_2508_18182_b200 import build as B

NAME = "paper_2508_18182_b200._tensor_calls"


class _NoDevice:
    """A library whose contexts cannot be created."""

    def adloco_create(self, handle, device):
        return A.ERR_CUDA

    def adloco_status_string(self, rc):
        return b"no device"


def test_a_context_does_not_need_the_module(monkeypatch):
    monkeypatch.setitem(sys.modules, NAME, None)                 # an import of it fails
    monkeypatch.delattr(sys.modules["paper_2508_18182_b200"], "_tensor_calls", raising=False)
    monkeypatch.setattr(A, "load_library", _NoDevice)
    with pytest.raises(A.AdlocoError) as e:                      # not an ImportError
        A.Context(0)
    assert e.value.status == A.ERR_CUDA


def test_the_operators_say_what_is_missing(monkeypatch):
    monkeypatch.setitem(sys.modules, NAME, None)
    monkeypatch.delattr(sys.modules["paper_2508_18182_b200"], "_tensor_calls", raising=False)
    ctx = A.Context.__new__(A.Context)
    ctx.h, ctx.device = None, torch.device("cuda", 0)
    with pytest.raises(ImportError, match="paper_2508_18182_b200.build"):
        ctx.calls


def test_torch_without_cuda_does_not_fail_the_build(monkeypatch, tmp_path, capsys):
    monkeypatch.setattr(torch.version, "cuda", None)
    monkeypatch.setattr(B, "CALLS", str(tmp_path / "_tensor_calls.so"))
    monkeypatch.setattr(B, "_stale", lambda: False)
    monkeypatch.setattr(subprocess, "run", lambda *a, **k: pytest.fail("nothing to compile"))
    assert B.build() == B.LIB
    assert "torch with CUDA" in capsys.readouterr().err


def test_the_module_is_rebuilt_for_another_torch(monkeypatch, tmp_path):
    """Its age says nothing about the torch it was compiled against; a stamp beside it does."""
    built = []

    def compiler(cmd, **kw):
        built.append(cmd)
        open(cmd[cmd.index("-o") + 1], "w").close()
        return subprocess.CompletedProcess(cmd, 0, "", "")
    monkeypatch.setattr(B, "CALLS", str(tmp_path / "_tensor_calls.so"))
    monkeypatch.setattr(B, "_stale", lambda: False)
    monkeypatch.setattr(subprocess, "run", compiler)
    B.build()
    B.build()
    assert len(built) == 1
    monkeypatch.setattr(torch, "__version__", "0.0.1+other")
    B.build()
    B.build()
    assert len(built) == 2
