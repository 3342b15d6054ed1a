"""What build() needs: the library builds without torch, a C++ compiler of its own or
Python's headers, and before an error of the binding is raised.  (A library of one
small source stands for the real one.)"""
import os
import sys

import pytest

from paper_2609_02514_gb300 import build as b


@pytest.fixture
def small(tmp_path, monkeypatch):
    src = tmp_path / "one.cu"
    src.write_text('extern "C" int one() { return 1; }\n')
    monkeypatch.setattr(b, "HERE", str(tmp_path))
    monkeypatch.setattr(b, "LIB", str(tmp_path / "libone.so"))
    monkeypatch.setattr(b, "_sources", lambda: [str(src)])
    return tmp_path


def _no_torch(monkeypatch, tmp_path):
    monkeypatch.setitem(sys.modules, "torch", None)       # an import of it raises


def _no_headers(monkeypatch, tmp_path):
    import sysconfig
    paths = dict(sysconfig.get_paths(), include=str(tmp_path))
    monkeypatch.setattr(sysconfig, "get_paths", lambda: paths)


def _no_compiler(monkeypatch, tmp_path):
    monkeypatch.delenv("CXX", raising=False)
    which = b.shutil.which
    monkeypatch.setattr(b.shutil, "which", lambda name: None if name in ("g++", "c++") else which(name))


@pytest.mark.parametrize("without", [_no_torch, _no_headers, _no_compiler])
def test_the_library_builds_without(small, monkeypatch, capfd, without):
    without(monkeypatch, small)
    assert b.build() == b.LIB and os.path.exists(b.LIB)
    assert not list(small.glob("_binding*"))
    assert "is not built" in capfd.readouterr().err


def test_the_library_is_there_when_the_binding_does_not_compile(small, monkeypatch):
    pytest.importorskip("torch")
    bad = small / "binding.cpp"
    bad.write_text("this is not C++\n")
    monkeypatch.setattr(b, "BINDING_SRC", str(bad))
    with pytest.raises(RuntimeError, match="the binding does not compile"):
        b.build()
    assert os.path.exists(b.LIB) and not list(small.glob("_binding*.so"))


def test_a_binding_of_other_versions_is_not_loaded(monkeypatch):
    torch = pytest.importorskip("torch")
    import paper_2609_02514_gb300 as A
    b.build()
    monkeypatch.setattr(A, "_native_module", None)
    assert A._native().__file__ == b.binding_path(torch.__version__)
    monkeypatch.setattr(A, "_native_module", None)
    monkeypatch.setattr(torch, "__version__", "0.0.1")
    with pytest.raises(RuntimeError, match="build it with"):
        A._native()


def test_a_built_binding_needs_no_compiler(small, monkeypatch, capfd):
    torch = pytest.importorskip("torch")
    with open(b.binding_path(torch.__version__), "w"):
        pass
    _no_compiler(monkeypatch, small)
    b.build()
    assert "is not built" not in capfd.readouterr().err
