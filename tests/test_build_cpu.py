"""What the build runs, and when: the library needs nothing of torch, the reader of lists is built anew for another torch.  No compiler is called."""
import os
import sys

import pytest
import torch

import paper_1706_07191_amd as B
from paper_1706_07191_amd import build as builder


@pytest.fixture
def ran(tmp_path, monkeypatch):
    """The commands of builds into a folder of their own, whose results are empty files."""
    monkeypatch.setattr(builder, "OBJ", str(tmp_path / "_build"))
    monkeypatch.setattr(builder, "LIB", str(tmp_path / "libbrsvd.so"))
    monkeypatch.setattr(builder, "LISTS", str(tmp_path / "_lists.so"))
    commands = []

    def run(cmd):
        commands.append(cmd)
        open(cmd[cmd.index("-o") + 1], "w").close()
        return ""
    monkeypatch.setattr(builder, "_run", run)
    return commands


def results(commands):
    return sorted(os.path.basename(c[c.index("-o") + 1]) for c in commands)


ALL = sorted([s.replace(".hip", ".o") for s in builder.SOURCES] + ["libbrsvd.so"])


def test_library_without_torch(ran, monkeypatch, capsys):
    monkeypatch.setitem(sys.modules, "torch", None)
    assert builder.build() == builder.LIB and os.path.exists(builder.LIB)
    assert results(ran) == ALL and not os.path.exists(builder.LISTS)
    assert "_lists.so" in capsys.readouterr().out


def test_library_where_the_reader_of_lists_does_not_compile(ran, monkeypatch):
    run = builder._run

    def fails(cmd):
        if cmd[0] == "g++":
            raise RuntimeError("command failed")
        return run(cmd)
    monkeypatch.setattr(builder, "_run", fails)
    with pytest.raises(RuntimeError):
        builder.build()
    assert results(ran) == ALL and os.path.exists(builder.LIB)


@pytest.mark.parametrize("what,value", [("__version__", "0.1+other"), ("compiled_with_cxx11_abi", lambda: not torch._C._GLIBCXX_USE_CXX11_ABI)])
def test_reader_of_lists_is_of_this_torch(ran, monkeypatch, what, value):
    builder.build()
    assert results(ran) == sorted(ALL + ["_lists.so"])
    ran.clear()
    builder.build()
    assert ran == []
    monkeypatch.setattr(torch, what, value)
    builder.build()
    assert results(ran) == ["_lists.so"]
    ran.clear()
    builder.build()
    assert ran == []


def test_reader_of_lists_of_another_torch_is_not_used(monkeypatch):
    monkeypatch.setattr(B, "_tables", None)
    monkeypatch.setattr(torch, "__version__", "0.1+other")
    with pytest.raises(ImportError, match="0.1.other"):
        B._tensors([])
    monkeypatch.undo()
    assert B._tensors([]) == (b"",)
