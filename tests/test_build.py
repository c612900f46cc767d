"""What is built, for what, and in which order (no compiler runs here)."""
import os
import sys

import pytest
import torch

from paper_2604_06836_b200 import build, clip


@pytest.fixture
def commands(monkeypatch, tmp_path):
    """Takes the place of the compilers: what they are called with, and an empty file for each result."""
    calls = []

    def call(cmd):
        calls.append(cmd)
        open(cmd[cmd.index("-o") + 1], "w").close()
    monkeypatch.setattr(build.subprocess, "check_call", call)
    monkeypatch.setattr(build, "HERE", str(tmp_path))
    monkeypatch.setattr(build, "LIB", str(tmp_path / "libstq.so"))
    return calls


def test_the_library_needs_no_torch(commands, monkeypatch, capsys):
    monkeypatch.setitem(sys.modules, "torch", None)
    assert build.build() == build.LIB and os.path.exists(build.LIB)
    assert len(commands) == 1 and "sm_100a" in " ".join(commands[0])
    assert "torch" in capsys.readouterr().err


def test_the_module_is_built_for_each_torch(commands, monkeypatch):
    build.build()
    assert len(commands) == 2 and any(c.endswith("stq_lists.cpp") for c in commands[1])
    build.build()
    assert len(commands) == 2                      # neither is out of date
    monkeypatch.setattr(torch, "__version__", "9.9.0a1+git-1234")
    build.build()
    name = "_lists_torch_9_9_0a1_git_1234"
    assert len(commands) == 3 and f"-DSTQ_LISTS={name}" in commands[2]
    assert f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}" in commands[2]
    assert len([f for f in os.listdir(build.HERE) if f.startswith(name + ".")]) == 1


def test_a_module_for_another_torch_is_not_taken(stq_lib, monkeypatch):
    monkeypatch.setattr(clip, "_fn", None)
    monkeypatch.setattr(torch, "__version__", "9.9.0")
    with pytest.raises(RuntimeError, match="paper_2604_06836_b200.build"):
        clip._lib()
    monkeypatch.undo()
    assert clip._lib() is not None
