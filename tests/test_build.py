"""The build: libicv.so needs hipcc alone, whatever happens to the module that checks torch tensors.  The compilers are stand-ins
that write their output file."""
import importlib.util
import os

import pytest

from paper_1907_02129_amd import build


@pytest.fixture
def paths(tmp_path, monkeypatch):
    (tmp_path / "csrc").mkdir()
    for name in ("a.hip", "b.hip"):
        (tmp_path / "csrc" / name).write_text("")
    hipcc = tmp_path / "hipcc"
    hipcc.write_text('#!/bin/sh\nwhile [ "$1" != -o ]; do shift; done\necho made > "$2"\n')
    hipcc.chmod(0o755)
    for name, at in (("CSRC", "csrc"), ("OBJ", "obj"), ("LIB", "lib.so"), ("PYTHON_MODULE", "module.so"), ("HIPCC", "hipcc")):
        monkeypatch.setattr(build, name, str(tmp_path / at))
    return tmp_path


@pytest.mark.parametrize("what", ["torch", "headers", "Python.h", "compiler"])
def test_the_library_is_built_without_what_only_the_module_needs(paths, monkeypatch, capsys, what):
    (paths / "module.so").write_text("an old one")
    if what == "torch":
        monkeypatch.setattr(importlib.util, "find_spec", lambda name, *a: None)
    elif what == "compiler":
        monkeypatch.setenv("CXX", "no-such-compiler")
    else:
        exists = os.path.exists
        end = "python_variable.h" if what == "headers" else "Python.h"
        monkeypatch.setattr(os.path, "exists", lambda p: not str(p).endswith(end) and exists(p))
    assert build.missing_for_python_module()
    assert build.build() == str(paths / "lib.so") and (paths / "lib.so").exists()
    assert not (paths / "module.so").exists()                       # it would check against another description
    assert "_icv_python.so" in capsys.readouterr().err


def test_the_library_is_linked_where_the_module_fails(paths, monkeypatch):
    def fails(*_):
        raise RuntimeError("g++ failed")

    monkeypatch.setattr(build, "missing_for_python_module", lambda: "", raising=False)
    monkeypatch.setattr(build, "build_python_module", fails)
    with pytest.raises(RuntimeError, match="g.. failed"):
        build.build()
    assert (paths / "lib.so").exists()
