"""The build: the library by itself, and the calls on torch tensors for the PyTorch that is there."""

import os

import pytest

from paper_2608_11152_gb300 import build as b


@pytest.fixture
def small(tmp_path, monkeypatch):
    """A build of one small file into a folder of its own."""
    monkeypatch.setattr(b, "BUILD", str(tmp_path))
    monkeypatch.setattr(b, "LIB", str(tmp_path / "libmisat.so"))
    monkeypatch.setattr(b, "CALLS", str(tmp_path / "_calls.so"))
    monkeypatch.setattr(b, "CALLS_FOR", str(tmp_path / "calls_for.txt"), raising=False)
    monkeypatch.setattr(b, "SOURCES", ["kv.cu"])
    return tmp_path


def _no_torch(monkeypatch):
    monkeypatch.setattr(b.importlib.util, "find_spec", lambda name: None)


def _no_compiler(monkeypatch):
    which = b.shutil.which
    monkeypatch.setattr(b.shutil, "which", lambda name: None if name == "g++" else which(name))


def _no_headers(monkeypatch):
    monkeypatch.setattr(b.sysconfig, "get_paths", lambda: {"include": "/nonexistent"})


@pytest.mark.parametrize("without", [_no_torch, _no_compiler, _no_headers])
def test_the_library_needs_neither_torch_nor_a_host_compiler_of_its_own(small, monkeypatch, capsys, without):
    pytest.importorskip("torch")
    without(monkeypatch)
    assert b.build() == b.LIB
    assert os.path.exists(b.LIB) and not os.path.exists(b.CALLS)
    assert "without the calls" in capsys.readouterr().err
    made = os.path.getmtime(b.LIB)
    b.build()
    assert os.path.getmtime(b.LIB) == made


def test_calls_that_do_not_compile_leave_the_library(small, monkeypatch):
    pytest.importorskip("torch")

    def fails():
        raise RuntimeError("g++ failed")

    monkeypatch.setattr(b, "_compile_calls", fails)
    with pytest.raises(RuntimeError, match="failed"):
        b.build()
    assert os.path.exists(b.LIB) and not os.path.exists(b.CALLS)


def test_calls_are_built_again_for_another_torch_and_the_library_is_not(small, monkeypatch):
    pytest.importorskip("torch")
    b.build()
    assert os.path.exists(b.LIB) and os.path.exists(b.CALLS)
    lib, calls = os.path.getmtime(b.LIB), os.path.getmtime(b.CALLS)
    b.build()
    assert (os.path.getmtime(b.LIB), os.path.getmtime(b.CALLS)) == (lib, calls)
    text = b._calls_for()
    monkeypatch.setattr(b, "_calls_for", lambda: text + "another")
    b.build()
    assert os.path.getmtime(b.LIB) == lib and os.path.getmtime(b.CALLS) > calls
