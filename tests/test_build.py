"""What the build needs: hipcc for the library; hipcc, torch and the headers of both torch and Python for the operators' extension."""
import importlib.util
import os

import pytest

from paper_2310_14423_amd import build as b
import paper_2310_14423_amd.operators as ops


@pytest.fixture
def recorded(monkeypatch, tmp_path):
    """Builds into an empty folder with a compiler that writes an empty file."""
    commands = []

    def compiler(cmd):
        commands.append(cmd)
        open(cmd[cmd.index("-o") + 1], "w").close()
    monkeypatch.setattr(b.subprocess, "check_call", compiler)
    monkeypatch.setattr(b, "LIB", str(tmp_path / "libqsr.so"))
    monkeypatch.setattr(b, "CALLS", str(tmp_path / "_calls.so"))
    return commands


def test_one_compiler(recorded):
    assert b.build() == b.LIB and os.path.exists(b.LIB) and os.path.exists(b.CALLS)
    assert [c[0] for c in recorded] == ["hipcc", "hipcc"]


def test_without_torch(recorded, monkeypatch, capsys):
    """The library is built and said to be; an extension for another library does not stay."""
    find = importlib.util.find_spec
    monkeypatch.setattr(importlib.util, "find_spec", lambda name, *a: None if name == "torch" else find(name, *a))
    open(b.CALLS, "w").close()
    assert b.build() == b.LIB and os.path.exists(b.LIB) and not os.path.exists(b.CALLS) and len(recorded) == 1
    assert "not built" in capsys.readouterr().err


@pytest.mark.parametrize("missing", ["Python.h", "python_variable.h"])
def test_without_headers(recorded, monkeypatch, capsys, missing):
    exists = os.path.exists
    monkeypatch.setattr(os.path, "exists", lambda p: exists(p) and os.path.basename(p) != missing)
    assert b.build() == b.LIB and exists(b.LIB) and not exists(b.CALLS) and len(recorded) == 1
    assert "not built" in capsys.readouterr().err


def test_operators_without_their_extension(monkeypatch):
    """Loud, with the way out of it."""
    import sys
    import torch
    import paper_2310_14423_amd as qsr
    monkeypatch.setattr(ops, "_calls", None)
    monkeypatch.setattr(ops, "_torch", None)
    monkeypatch.setitem(sys.modules, "paper_2310_14423_amd._calls", None)
    monkeypatch.delattr(qsr, "_calls", raising=False)
    with pytest.raises(RuntimeError, match="paper_2310_14423_amd.build"):
        qsr.rmsnorm(torch.zeros(2, 4), torch.ones(4))
