"""What the build makes, and for whom (no GPU needed)."""
import os
import subprocess
import sys

import pytest

from paper_2510_26771_b200 import build as stamp_build


def test_the_library_builds_without_torch(monkeypatch, capsys):
    stamp_build.build()
    monkeypatch.setitem(sys.modules, "torch", None)          # `import torch` raises ImportError
    monkeypatch.setattr(subprocess, "check_call", lambda *a, **k: pytest.fail("nothing is out of date"))
    assert stamp_build.build() == stamp_build.LIB_PATH
    assert "torch" in capsys.readouterr().err


def test_the_library_builds_without_pythons_headers(monkeypatch, capsys, tmp_path):
    import sysconfig
    stamp_build.build()
    paths = dict(sysconfig.get_paths(), include=str(tmp_path))
    monkeypatch.setattr(sysconfig, "get_paths", lambda *a, **k: paths)
    monkeypatch.setattr(subprocess, "check_call", lambda *a, **k: pytest.fail("nothing can be compiled"))
    assert stamp_build.build() == stamp_build.LIB_PATH
    assert "Python.h" in capsys.readouterr().err


def test_another_torch_gets_a_module_of_its_own(monkeypatch):
    import torch
    stamp_build.build()
    here = stamp_build.calls_path()
    assert os.path.exists(here) and here.endswith(".so")
    monkeypatch.setattr(torch, "__version__", "2.99.0+other")
    there = stamp_build.calls_path()
    assert there != here and not os.path.exists(there)
    commands = []
    monkeypatch.setattr(subprocess, "check_call", lambda command, *a, **k: commands.append(command))
    monkeypatch.setattr(os, "replace", lambda *a: None)
    assert stamp_build.build_calls() == there and len(commands) == 1


def test_a_failed_compilation_leaves_no_file(monkeypatch):
    import torch
    stamp_build.build()
    monkeypatch.setattr(torch, "__version__", "2.99.0+other")

    def fail(command, *a, **k):
        open(command[command.index("-o") + 1], "w").close()
        raise subprocess.CalledProcessError(1, command)

    monkeypatch.setattr(subprocess, "check_call", fail)
    before = sorted(os.listdir(os.path.dirname(stamp_build.LIB_PATH)))
    with pytest.raises(subprocess.CalledProcessError):
        stamp_build.build_calls()
    assert sorted(os.listdir(os.path.dirname(stamp_build.LIB_PATH))) == before


def test_the_entry_point_loads_the_marshalling_module(monkeypatch):
    import __graft_entry__
    from oracle import stamp_oracle
    from paper_2510_26771_b200 import binding
    stamp_build.build()
    monkeypatch.setattr(stamp_build, "build", lambda **k: None)
    monkeypatch.setattr(stamp_oracle, "build", lambda **k: None)
    monkeypatch.setattr(binding, "_calls", None)
    __graft_entry__.build()
    assert binding._calls is not None
