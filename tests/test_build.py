"""What is built where the host code of the binding cannot be, with compilers that only leave their output (no GPU)."""
import os
import stat
import sys

import pytest

from paper_2409_10516_amd import binding as B, build as M


@pytest.fixture
def tree(tmp_path, monkeypatch):
    """A tree of one source. hipcc, as g++ if asked, writes what -o names."""
    fake = tmp_path / "fake"
    fake.write_text('#!/bin/sh\nwhile [ "$1" != -o ]; do shift; done\necho built > "$2"\n')
    fake.chmod(fake.stat().st_mode | stat.S_IXUSR)
    for name, at in (("CSRC", tmp_path), ("LIB", tmp_path / "libra.so"), ("CALLS", tmp_path / "_calls.so"), ("SOURCES", ["a.hip"])):
        monkeypatch.setattr(M, name, str(at) if name != "SOURCES" else at)
    monkeypatch.setenv("HIPCC", str(fake))
    monkeypatch.setenv("CXX", str(fake))
    return tmp_path


def test_all_is_built(tree, capsys):
    assert M.build(verbose=False) == str(tree / "libra.so")
    assert (tree / "libra.so").exists() and (tree / "_calls.so").exists() and capsys.readouterr().out == ""


def test_the_library_is_built_without_a_host_compiler(tree, monkeypatch, capsys):
    monkeypatch.setenv("CXX", str(tree / "none"))
    (tree / "_calls.so").write_text("of other sources")
    assert M.build(verbose=False) == str(tree / "libra.so")
    assert (tree / "libra.so").exists() and not (tree / "_calls.so").exists() and "_calls.so" in capsys.readouterr().out


def test_the_library_is_built_without_pythons_headers(tree, monkeypatch, capsys):
    monkeypatch.setattr(M.sysconfig, "get_paths", lambda: {"include": str(tree / "none")})
    assert M.build(verbose=False) == str(tree / "libra.so")
    assert (tree / "libra.so").exists() and not (tree / "_calls.so").exists() and "Python.h" in capsys.readouterr().out


def test_the_library_is_built_without_torch(tree, monkeypatch, capsys):
    monkeypatch.setitem(sys.modules, "torch", None)
    assert M.build(verbose=False) == str(tree / "libra.so")
    assert (tree / "libra.so").exists() and not (tree / "_calls.so").exists() and "torch" in capsys.readouterr().out


def test_a_host_compiler_with_arguments(tree, monkeypatch):
    monkeypatch.setenv("CXX", f"{tree / 'fake'} -std=c++17")
    M.build(verbose=False)
    assert (tree / "_calls.so").exists()


def test_a_mistake_in_the_host_code_is_one_of_the_build(tree, monkeypatch):
    """The library is linked all the same."""
    broken = tree / "broken"
    broken.write_text("#!/bin/sh\necho a mistake\nexit 1\n")
    broken.chmod(broken.stat().st_mode | stat.S_IXUSR)
    monkeypatch.setenv("CXX", str(broken))
    (tree / "_calls.so").write_text("of other sources")
    with pytest.raises(RuntimeError, match="a mistake"):
        M.build(verbose=False)
    assert (tree / "libra.so").exists() and not (tree / "_calls.so").exists()


def test_a_mistake_in_a_kernel_is_one_of_the_build(tree, monkeypatch):
    broken = tree / "broken"
    broken.write_text("#!/bin/sh\necho a mistake\nexit 1\n")
    broken.chmod(broken.stat().st_mode | stat.S_IXUSR)
    monkeypatch.setenv("HIPCC", str(broken))
    with pytest.raises(RuntimeError, match="a mistake"):
        M.build(verbose=False)


def test_compiled_checks_are_used_where_they_are_built(monkeypatch, tmp_path):
    monkeypatch.setattr(B, "_short", None)
    assert os.path.exists(B.CALLS_PATH) and B._calls() is not None
    monkeypatch.setattr(B, "_short", None)
    monkeypatch.setattr(B, "CALLS_PATH", str(tmp_path / "_calls.so"))
    assert B._calls() is None
