"""The compiled call path is optional: the library builds without it, and a module made for another torch is not used."""
import os
import sys
import types

import pytest

from paper_2505_23725_b200 import binding, build


def test_the_library_builds_where_the_call_path_does_not(monkeypatch, tmp_path, capsys):
    stale = tmp_path / "_fastcall.so"
    stale.write_bytes(b"made for something else")
    def broken(force=False):
        raise RuntimeError("Python.h: No such file or directory")
    monkeypatch.setattr(build, "build_fastcall", broken)
    monkeypatch.setattr(build, "FASTCALL", str(stale))
    assert build.build_library(force=False) == build.LIB and os.path.exists(build.LIB)
    assert not stale.exists()
    assert "Python.h" in capsys.readouterr().err


def test_the_call_path_is_made_again_for_another_torch(monkeypatch, tmp_path):
    so, stamp = tmp_path / "_fastcall.so", tmp_path / "_build" / "fastcall.torch"
    monkeypatch.setattr(build, "FASTCALL", str(so))
    monkeypatch.setattr(build, "FASTCALL_TORCH", str(stamp))
    made = []
    def compiler(cmd, **kw):
        made.append(cmd)
        so.write_bytes(b"module")
        return types.SimpleNamespace(returncode=0, stdout="")
    monkeypatch.setattr(build.subprocess, "run", compiler)
    assert build.build_fastcall() == str(so) and len(made) == 1
    build.build_fastcall()
    assert len(made) == 1                              # up to date
    stamp.write_text("1.0.0")
    build.build_fastcall()
    assert len(made) == 2
    build.build_fastcall(force=True)
    assert len(made) == 3
    monkeypatch.setattr(build.subprocess, "run", lambda cmd, **kw: types.SimpleNamespace(returncode=1, stdout="no"))
    with pytest.raises(RuntimeError, match="g\\+\\+"):
        build.build_fastcall(force=True)


def test_a_module_for_another_torch_is_not_used(monkeypatch):
    import torch
    name = binding.__package__ + "._fastcall"
    package = sys.modules[binding.__package__]
    for version, used in ((torch.__version__, True), ("1.0.0", False), (None, False)):
        m = types.ModuleType(name)
        if version is not None:
            m.TORCH = version
        monkeypatch.setitem(sys.modules, name, m)
        monkeypatch.setattr(package, "_fastcall", m, raising=False)
        assert (binding._load_fastcall() is m) == used


def test_the_built_module_is_for_this_torch():
    build.build_fastcall()
    import importlib.util
    import torch
    spec = importlib.util.spec_from_file_location("_fastcall", build.FASTCALL)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    assert m.TORCH == torch.__version__
