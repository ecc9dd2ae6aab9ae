"""The layer of experts, token log probabilities and AdamW at their C boundary, without a GPU."""
import ctypes as ct
import os
import re

import pytest

import paper_2608_14575_gb300 as H
from paper_2608_14575_gb300 import _hwr, _ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    H.build()
    return _ops.load_ops()


def test_constants_match_the_header():
    text = open(os.path.join(ROOT, "include", "hwr_ops.h")).read()
    for name in ("HWR_EXPERTS_MAX_ROWS", "HWR_EXPERTS_MAX_TOP", "HWR_EXPERTS_MAX_OUT", "HWR_EXPERTS_MAX_WIDTH",
                 "HWR_TOKENS_MAX_TOP", "HWR_ADAMW_BLOCK"):
        assert int(re.search(rf"#define {name} (\d+)", text).group(1)) == getattr(H, name)
    for name, value in _ops.ACTIVATIONS.items():
        assert int(re.search(rf"HWR_ACT_{name.upper()} = (\d+)", text).group(1)) == value


def test_structures_match_the_header():
    """Fields of the same names in the same order."""
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "hwr_ops.h")).read(), flags=re.S)
    for name in ("hwr_adamw_tensor", "hwr_adamw_options", "hwr_experts", "hwr_logits"):
        body = re.search(r"typedef struct \{([^}]*)\} " + name + ";", text).group(1)
        fields = [re.sub(r".*[ *]", "", f.strip()) for line in body.split(";") if line.strip()
                  for f in line.split(",")]
        assert fields == [f for f, _ in getattr(_ops, name)._fields_], name


def test_calls_without_a_context(lib):
    bad = _hwr.HWR_ERR_INVALID_ARG
    e, z, o = _ops.hwr_experts(), _ops.hwr_logits(), _ops.hwr_adamw_options()
    assert lib.hwr_expert_layer(None, ct.byref(e), None, 0) == bad
    assert lib.hwr_token_logprobs(None, ct.byref(z), 0, None, None, None, None, None) == bad
    assert lib.hwr_token_logprobs_backward(None, ct.byref(z), None, None, None, None, None, 0) == bad
    assert lib.hwr_adamw_create(None, 0, None, 32, None, None) == bad
    assert lib.hwr_adamw_step(None, None, ct.byref(o), None, None) == bad
    assert lib.hwr_adamw_destroy(None, None) == _hwr.HWR_OK
