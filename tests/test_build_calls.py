"""The Python extension of the losses is built beside the library where a CUDA build of torch is installed, anew for another
torch or Python; the library needs neither."""
import importlib.util
import os

import pytest

from paper_2403_06988_gb300 import build as build_mod


@pytest.fixture
def elsewhere(tmp_path, monkeypatch):
    """Everything built goes to a folder of its own."""
    monkeypatch.setattr(build_mod, "CALLS", str(tmp_path / "_loss_calls.so"))
    compiled = []

    def run(cmd, **kw):
        compiled.append(cmd)
        open(cmd[cmd.index("-o") + 1], "w").close()
        return type("Done", (), {"returncode": 0, "stdout": "", "stderr": ""})
    monkeypatch.setattr(build_mod.subprocess, "run", run)
    return compiled


def test_without_torch_the_library_is_built_alone(elsewhere, monkeypatch, capsys):
    find = importlib.util.find_spec
    monkeypatch.setattr(importlib.util, "find_spec", lambda name, *a: None if name == "torch" else find(name, *a))
    monkeypatch.setattr(build_mod, "up_to_date", lambda lib=None: True)
    assert build_mod.build() == build_mod.LIB
    assert build_mod.build_calls() is None and not elsewhere
    assert "torch" in capsys.readouterr().err


def test_with_a_torch_without_cuda_too(elsewhere, monkeypatch, tmp_path):
    (tmp_path / "torch" / "lib").mkdir(parents=True)
    spec = type("Spec", (), {"submodule_search_locations": [str(tmp_path / "torch")]})
    find = importlib.util.find_spec
    monkeypatch.setattr(importlib.util, "find_spec", lambda name, *a: spec if name == "torch" else find(name, *a))
    assert build_mod.build_calls() is None and not elsewhere


def test_built_again_for_another_torch(elsewhere, monkeypatch):
    pytest.importorskip("torch")
    assert build_mod.build_calls() == build_mod.CALLS and len(elsewhere) == 1
    assert build_mod.build_calls() == build_mod.CALLS and len(elsewhere) == 1
    monkeypatch.setattr(build_mod, "_torch_version", lambda *a: "another")
    assert build_mod.build_calls() == build_mod.CALLS and len(elsewhere) == 2
    assert build_mod.build_calls() == build_mod.CALLS and len(elsewhere) == 2
    os.utime(build_mod.CALLS, (1, 1))     # older than its source
    build_mod.build_calls()
    assert len(elsewhere) == 3


def test_a_missing_or_foreign_extension_says_how_to_get_it(elsewhere, monkeypatch):
    pytest.importorskip("torch")
    import paper_2403_06988_gb300 as p
    monkeypatch.setattr(p, "_CALLS", None)
    with pytest.raises(ImportError, match="build"):
        p._calls()
    build_mod.build_calls()
    monkeypatch.setattr(build_mod, "_torch_version", lambda *a: "another")
    with pytest.raises(ImportError, match="build"):
        p._calls()
