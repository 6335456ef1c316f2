"""The C library is built where the Python extension beside it cannot be (no compiler runs here)."""
from __future__ import annotations

import os
import sys
import sysconfig

import pytest

from paper_2607_15621_gb300 import build as b
from paper_2607_15621_gb300 import fsx


@pytest.fixture
def stub(monkeypatch, tmp_path):
    """build() into a folder of its own, every command of which writes its output; those that name `stub.fails` fail."""
    def run(cmd):
        if stub.fails and any(stub.fails in x for x in cmd):
            raise RuntimeError("command failed: " + " ".join(cmd))
        with open(cmd[cmd.index("-o") + 1], "w") as f:
            f.write("built")
        return ""
    stub = lambda: None
    stub.fails, stub.lib, stub.calls = "", str(tmp_path / "lib" / "libfsx.so"), str(tmp_path / "lib" / "_calls.so")
    for name, value in (("OUT_DIR", str(tmp_path / "lib")), ("BUILD_DIR", str(tmp_path / "obj")), ("LIB", stub.lib), ("CALLS", stub.calls),
                        ("_run", run), ("nvcc", lambda: "nvcc")):
        monkeypatch.setattr(b, name, value)
    monkeypatch.setattr(fsx, "CALLS_PATH", stub.calls)
    return stub


def test_both_are_built(stub):
    assert b.build() == stub.lib and os.path.exists(stub.lib) and os.path.exists(stub.calls)


@pytest.mark.parametrize("lacking", ["torch", "Python.h", "compiler"])
def test_the_library_needs_neither_torch_nor_headers(stub, monkeypatch, lacking, tmp_path, capsys):
    b.build()  # an extension of an earlier build
    os.remove(stub.lib)
    if lacking == "torch":
        monkeypatch.setitem(sys.modules, "torch", None)
    elif lacking == "Python.h":
        paths = dict(sysconfig.get_paths(), include=str(tmp_path))
        monkeypatch.setattr(sysconfig, "get_paths", lambda *a, **k: paths)
    else:
        monkeypatch.setenv("CXX", str(tmp_path / "none"))
    assert b.build() == stub.lib and os.path.exists(stub.lib)
    assert not os.path.exists(stub.calls)  # it does not go with this library
    said = {"torch": "torch", "Python.h": "Python.h", "compiler": "none"}[lacking]
    assert said in capsys.readouterr().err
    monkeypatch.setattr(fsx, "_calls", None)
    monkeypatch.setattr(fsx, "lib", lambda: None)
    if lacking != "torch":  # the binding's callers have torch
        with pytest.raises(RuntimeError, match=said):
            fsx._native()


def test_an_extension_that_does_not_compile_is_an_error_but_the_library_is_there(stub):
    stub.fails = "calls.cpp"
    with pytest.raises(RuntimeError, match="calls.cpp"):
        b.build()
    assert os.path.exists(stub.lib) and not os.path.exists(stub.calls)


def test_a_source_that_does_not_compile_leaves_no_library(stub):
    stub.fails = "rotary.cu"
    with pytest.raises(RuntimeError, match="rotary.cu"):
        b.build()
    assert not os.path.exists(stub.lib)
