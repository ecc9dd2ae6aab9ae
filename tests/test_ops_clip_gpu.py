"""Gradient clipping over many chunks and long tensors."""
import math

import pytest

torch = pytest.importorskip("torch")

import paper_2608_14575_gb300 as H

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    H.build()
    return H.Operators()


def test_norm_over_many_chunks(ops):
    """300 chunks a block.  A thread's share of a chunk is 16 fp32 squares, exact sums of
    this value's; an fp32 sum over the chunks would round it the same way each time, 29
    units of 2^-24 off in the norm.  What may be off: 16 roundings of a share (half of
    that in the norm), and the norm's own."""
    nsm = torch.cuda.get_device_properties(0).multi_processor_count
    g = torch.full((nsm * 8 * 300 * 4096,), 981 / 1024, device="cuda")
    norm = float(ops.clip_gradients([g], float("inf")))
    want = 981 / 1024 * math.sqrt(g.numel())
    assert abs(norm - want) <= want * 9 * 2.0 ** -24


def test_more_than_2_31_elements(ops):
    """Offsets beyond 32 bits: a tensor of 2^31 + 4,099 values, the last ones among them."""
    n = (1 << 31) + 4099
    g = torch.zeros(n, device="cuda", dtype=torch.bfloat16)
    at = torch.tensor([0, 4095, (1 << 31) - 1, 1 << 31, n - 1], device="cuda")
    g[at] = 3.0
    norm = ops.clip_gradients([g], 1.0)
    assert abs(float(norm) - math.sqrt(45)) <= 1e-6 * math.sqrt(45)
    want = torch.tensor(3.0 / (math.sqrt(45) + 1e-6)).to(torch.bfloat16)
    assert (g[at].cpu() == want).all()
    assert int((g != 0).sum()) == 5
