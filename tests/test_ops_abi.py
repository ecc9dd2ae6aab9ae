"""The operators' C ABI at its boundary, without a GPU."""
import ctypes as ct
import os
import re
import subprocess

import pytest

import paper_2608_14575_gb300 as H
from paper_2608_14575_gb300 import _hwr, _ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    H.build()
    return _ops.load_ops()


def header():
    return re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "hwr_ops.h")).read(), flags=re.S)


def test_every_declared_function_is_exported(lib):
    names = set(re.findall(r"\b(hwr_[a-z_]+)\s*\(", header()))
    out = subprocess.run(["nm", "-D", "--defined-only", H.lib_path()], capture_output=True, text=True, check=True).stdout
    exported = {l.split()[-1] for l in out.splitlines() if l.strip()}
    assert names <= exported and names == set(_ops.OPS_EXPORTS)


def test_constants_match_the_header():
    text = open(os.path.join(ROOT, "include", "hwr_ops.h")).read()
    for name in ("HWR_OPS_MAX_GROUPS", "HWR_OPS_MAX_RANK"):
        assert int(re.search(rf"#define {name} (\d+)", text).group(1)) == getattr(H, name)


def test_calls_without_a_context(lib):
    bad = _hwr.HWR_ERR_INVALID_ARG
    r, a, f = _ops.hwr_rows(), _ops.hwr_adapters(), ct.c_float()
    assert lib.hwr_ops_create(None, None) == bad
    assert lib.hwr_ops_synchronize(None) == bad
    assert lib.hwr_ops_reserve(None, 1) == bad
    assert lib.hwr_ops_after(None, None) == bad and lib.hwr_ops_before(None, None) == bad
    assert lib.hwr_dispatch(None, 1, 1, None, None, None) == bad
    assert lib.hwr_grouped_forward(None, ct.byref(r), None, 0) == bad
    assert lib.hwr_grouped_backward(None, ct.byref(r), None, 0, None, 0, None) == bad
    assert lib.hwr_adapter_forward(None, ct.byref(r), ct.byref(a), None, 0) == bad
    assert lib.hwr_adapter_backward(None, ct.byref(r), ct.byref(a), None, 0, None, 0, None, None) == bad
    assert lib.hwr_clip_gradients(None, 0, None, 1.0, ct.byref(f)) == bad
    assert lib.hwr_gradients_create(None, 0, None, None) == bad
    assert lib.hwr_gradients_clip(None, None, 1.0, ct.byref(f)) == bad
    assert lib.hwr_gradients_destroy(None, None) == _hwr.HWR_OK
    assert lib.hwr_ops_destroy(None) == _hwr.HWR_OK


def test_routing_contexts_refuse_half_precision():
    import workload as W
    p = W.make_config(0, Q=4)
    lib = H.load()
    pr = _hwr.hwr_predictor()
    pr.dtype = H.HWR_F16
    t = _hwr.hwr_deployment_table()
    ctx = ct.c_void_p()
    assert lib.hwr_create(ct.byref(t), ct.byref(pr), None, p["E"], H.HWR_F16, None, ct.byref(ctx)) \
        == _hwr.HWR_ERR_INVALID_ARG and ctx.value is None
