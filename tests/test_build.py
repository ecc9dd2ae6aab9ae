"""The build script: what it makes where torch is missing or does not compile."""
import importlib
import os
import time

import pytest

import paper_2608_14575_gb300  # noqa: F401  (the package's attribute `build` is the function)

build = importlib.import_module("paper_2608_14575_gb300.build")


@pytest.fixture
def small(monkeypatch, tmp_path):
    """One translation unit, into a folder of its own."""
    monkeypatch.setattr(build, "OUT_DIR", str(tmp_path))
    monkeypatch.setattr(build, "SOURCES", {"hwr_noalloc.cu": []})


def test_library_without_torch(small, monkeypatch):
    find = importlib.util.find_spec
    monkeypatch.setattr(build.importlib.util, "find_spec", lambda name, *a: None if name == "torch" else find(name, *a))
    out = build.build()
    assert out == build.lib_path() and os.path.exists(out)
    assert not os.path.exists(build.torch_path())
    made = os.path.getmtime(out)
    time.sleep(0.05)
    assert build.build() == out and os.path.getmtime(out) == made       # nothing is stale


def test_library_beside_a_broken_binding(small, monkeypatch):
    pytest.importorskip("torch")
    real = build._torch_commands
    monkeypatch.setattr(build, "_torch_commands", lambda *a: (["false"], real(*a)[1]))
    with pytest.raises(RuntimeError):
        build.build()
    assert os.path.exists(build.lib_path()) and not os.path.exists(build.torch_path())
