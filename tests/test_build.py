"""The build script: what it makes where torch is missing or does not compile."""
import importlib
import os
import shutil
import subprocess
import sys
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


def test_binding_moves_with_its_library(tmp_path):
    """A copy of the package loads the copy's own library, also where the first is gone."""
    pytest.importorskip("torch")
    build.build()
    there = tmp_path / "moved"
    there.mkdir()
    for f in (build.lib_path(), build.torch_path()):
        shutil.copy(f, there)
    lib, binding = (str(there / os.path.basename(f)) for f in (build.lib_path(), build.torch_path()))
    program = f"""
import ctypes, importlib.util, torch
ctypes.CDLL({lib!r})
spec = importlib.util.spec_from_file_location("hwr_torch", {binding!r})
spec.loader.exec_module(importlib.util.module_from_spec(spec))
print(sorted({{l.split()[-1] for l in open("/proc/self/maps") if "libhwr_" in l}}))
"""
    out = subprocess.run([sys.executable, "-c", program], capture_output=True, text=True, check=True).stdout
    assert eval(out) == [lib]
