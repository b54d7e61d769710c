"""The library needs hipcc alone; the attention operators' binding to torch is built
where torch, a C++ compiler and Python's headers are there.  (The compile and link
steps are stand-ins here.)"""
import os
import sys
import sysconfig

import pytest

from paper_2509_25689_amd import build


@pytest.fixture
def steps(tmp_path, monkeypatch):
    """build with its files under tmp_path and its steps recorded."""
    done = []
    for name in ("BUILD", "LIB", "PEAKS_LIB", "BINDING_LIB"):
        monkeypatch.setattr(build, name, str(tmp_path / name))
    open(build.BINDING_LIB, "w").close()                     # an earlier build's

    def compile_one(src):
        done.append(src)
        return src + ".o"

    def link(objs, lib):
        done.append(lib)
        open(lib, "w").close()
    monkeypatch.setattr(build, "_compile", compile_one)
    monkeypatch.setattr(build, "_link", link)
    return done


def _without_torch(monkeypatch, tmp_path):
    monkeypatch.setitem(sys.modules, "torch", None)          # (import torch raises ImportError)


def _without_compiler(monkeypatch, tmp_path):
    monkeypatch.setenv("PATH", str(tmp_path))


def _without_python_headers(monkeypatch, tmp_path):
    monkeypatch.setattr(sysconfig, "get_paths", lambda: {"include": str(tmp_path)})


@pytest.mark.parametrize("without,named", [(_without_torch, "torch"), (_without_compiler, "g++"), (_without_python_headers, "Python.h")])
def test_library_builds_without_what_the_binding_needs(steps, monkeypatch, tmp_path, capsys, without, named):
    without(monkeypatch, tmp_path)
    assert build.build() == build.LIB
    assert build.LIB in steps and build.PEAKS_LIB in steps
    assert not os.path.exists(build.BINDING_LIB)             # none rather than one of other sources
    assert named in capsys.readouterr().out


def test_binding_that_does_not_compile_is_an_error(steps, monkeypatch, tmp_path):
    bad = tmp_path / "bad.cpp"
    bad.write_text("#error no")
    monkeypatch.setattr(build, "BINDING", str(bad))
    with pytest.raises(RuntimeError, match="compile failed"):
        build.build()
