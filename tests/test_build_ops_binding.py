"""The build of the Python module that uses torch's objects where torch's headers are missing."""
import os
import sysconfig

import pytest

from paper_2202_11836_amd import build as B


@pytest.mark.skipif(not os.path.exists(os.path.join(sysconfig.get_paths()["include"], "Python.h")),
                    reason="needs Python.h")
@pytest.mark.parametrize("torch", ["absent", "without headers"])
def test_without_torchs_headers(torch, tmp_path, monkeypatch, capsys):
    import importlib.machinery
    import importlib.util
    spec = importlib.machinery.ModuleSpec("torch", None, is_package=True)
    spec.submodule_search_locations = [str(tmp_path)]
    monkeypatch.setattr(importlib.util, "find_spec", lambda name: None if torch == "absent" else spec)
    monkeypatch.setattr(B, "PKG", str(tmp_path))
    old = tmp_path / "_ops_call.so"
    old.write_bytes(b"of an earlier source")
    path = B.build_binding()
    assert path == str(tmp_path / "_attn_call.so") and os.path.exists(path) and not old.exists()
    assert "torch" in capsys.readouterr().err
