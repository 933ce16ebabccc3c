"""The build: the library is made of the HIP sources alone, whether the Python binding on top of it can be built or not.
The compilers are stand-ins that write empty files."""
import os
import sys

import pytest

import __graft_entry__ as graft
from paper_2407_09577_amd import build


@pytest.fixture
def tree(tmp_path, monkeypatch):
    hipcc = tmp_path / "hipcc"
    hipcc.write_text('#!/bin/sh\nwhile [ "$1" != -o ]; do shift; done\n: > "$2"\n')
    hipcc.chmod(0o755)
    for name, value in (("HIPCC", str(hipcc)), ("CXX", "false"), ("BUILD_DIR", str(tmp_path / "_build")),
                        ("LIB_PATH", str(tmp_path / "lib.so")), ("BINDING_PATH", str(tmp_path / "binding.so"))):
        monkeypatch.setattr(build, name, value)
    return tmp_path


@pytest.mark.parametrize("cxx", ["false", "/nowhere/c++"])
def test_the_library_stands_without_the_binding(tree, monkeypatch, cxx):
    monkeypatch.setattr(build, "CXX", cxx)
    (tree / "binding.so").write_text("of another library")
    with pytest.raises((RuntimeError, FileNotFoundError)):
        build.build(verbose=False)
    assert (tree / "lib.so").exists() and not (tree / "binding.so").exists()


def test_no_torch(tree, monkeypatch, capsys):
    monkeypatch.setitem(sys.modules, "torch", None)
    assert build.build() == str(tree / "lib.so")
    assert (tree / "lib.so").exists() and "without the binding" in capsys.readouterr().err


def test_ensure_built(tree, monkeypatch, capsys):
    monkeypatch.setattr("oracle.build", lambda *a, **k: None)
    graft.ensure_built()
    assert (tree / "lib.so").exists() and "the binding is not built" in capsys.readouterr().err
    stamp = os.stat(tree / "lib.so").st_mtime_ns
    (tree / "binding.so").write_text("built")
    graft.ensure_built()
    assert os.stat(tree / "lib.so").st_mtime_ns == stamp and capsys.readouterr().err == ""


def test_a_library_that_does_not_build(tree, monkeypatch):
    monkeypatch.setattr(build, "HIPCC", "false")
    with pytest.raises(RuntimeError):
        build.build(verbose=False)
    assert not (tree / "lib.so").exists()
