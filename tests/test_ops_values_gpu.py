"""Values at the ends of their types: infinities, small gradients, large inner products."""
import pytest

torch = pytest.importorskip("torch")

import paper_2608_14575_gb300 as H
import ops_ref as R
from test_ops_gpu import BF, HF, choices, ints, make

pytestmark = pytest.mark.gpu
INF = float("inf")


@pytest.fixture(scope="module")
def ops():
    H.build()
    return H.Operators()


def same(got, want, dt):
    """Equal, infinities and NaN among the values."""
    want = want.to(dt)
    bad = ~((got == want) | (got.isnan() & want.isnan()))
    assert not bad.any(), (int(bad.sum()), bad.numel(), torch.nonzero(bad)[:4].tolist(), got[bad][:4].tolist(),
                           want[bad][:4].tolist())


@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("T", [1, 5, 40])
def test_padding_meets_no_infinite_adapter(ops, dt, T):
    """A group's rows are padded to whole 16s with zeros; times an infinite value of the
    adapter these are NaN, which no gradient may see."""
    G, K, N, r = 2, 64, 72, 8
    c = torch.arange(T, device="cuda", dtype=torch.int32) % 2
    x, dy = torch.full((T, K), 2.0, device="cuda", dtype=dt), torch.ones(T, N, device="cuda", dtype=dt)
    w, s = torch.zeros(N, K, device="cuda", dtype=dt), torch.ones(G, device="cuda")
    a, b = torch.ones(G, r, K, device="cuda", dtype=dt), torch.ones(G, N, r, device="cuda", dtype=dt)
    a[0, 3, 5], b[0, 7, 2] = INF, INF
    _, da, db = ops.adapter_backward(dy, x, w, a, b, s, ops.dispatch(c, G))
    n = (c == 0).sum().item()
    want = torch.full((r, K), 2.0 * N * n, device="cuda", dtype=torch.float64)
    want[2] = INF
    same(da[0], want, dt)
    want = torch.full((N, r), 2.0 * K * n, device="cuda", dtype=torch.float64)
    want[:, 3] = INF
    same(db[0], want, dt)
