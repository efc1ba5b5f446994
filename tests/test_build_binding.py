"""The build of the operators' Python module where a compiler or Python's headers are
missing: nothing else of the package needs them."""
import importlib.util
import os
import shutil
import sysconfig

import pytest

from paper_2202_11836_amd import build as B

HEADERS = os.path.exists(os.path.join(sysconfig.get_paths()["include"], "Python.h"))


@pytest.fixture
def package(tmp_path, monkeypatch):
    monkeypatch.setattr(B, "PKG", str(tmp_path))
    monkeypatch.delenv("CXX", raising=False)
    return tmp_path


def test_without_pythons_headers(package, monkeypatch, capsys):
    old = package / "_attn_call.so"
    old.write_bytes(b"of an earlier source")
    monkeypatch.setattr(sysconfig, "get_paths", lambda: {"include": str(package)})
    assert B.build_binding() is None and not old.exists()
    assert "Python.h" in capsys.readouterr().err


@pytest.mark.skipif(not HEADERS or not os.path.exists(B.HIPCC), reason="needs hipcc and Python.h")
def test_without_gxx(package, monkeypatch):
    which = shutil.which
    monkeypatch.setattr(shutil, "which", lambda n, *a, **k: None if n == "g++" else which(n, *a, **k))
    monkeypatch.setenv("PATH", os.path.dirname(B.HIPCC))
    path = B.build_binding()
    spec = importlib.util.spec_from_file_location("_attn_call", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    assert {"setup", "forward", "backward"} <= set(dir(m))


@pytest.mark.skipif(not HEADERS, reason="needs Python.h")
def test_a_failed_compilation_is_one(package, monkeypatch):
    monkeypatch.setenv("CXX", shutil.which("false") or "/bin/false")
    with pytest.raises(RuntimeError):
        B.build_binding()
