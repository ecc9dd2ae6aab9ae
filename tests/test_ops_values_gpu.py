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


# Inner products at any magnitude.  Their sums are fp32; beside a shared projection they
# are two bf16 terms (at most 2^-16 off, relatively), in the gradients two terms of the
# rows' type, of fp16 scaled by the group's largest (2^-22 of the value, 2^-38 of the
# largest).  What is left is the outputs' own rounding.

def inner(p, mags, terms):
    return (terms + 64) * R.ADD * mags + p.abs() * 2.0 ** -22


def ends(x, w, a, b, s, dy, c):
    """(y, dx, da, db) with their bounds."""
    dt, (N, K), r = x.dtype, w.shape, a.shape[1]
    xx, d, ww = x.double(), dy.double(), w.double()
    low = 2.0 ** -16 if dt is BF else 2.0 ** -21
    y, dx = xx @ ww.T, d @ ww
    my, mx = xx.abs() @ ww.abs().T, d.abs() @ ww.abs()
    ey, ex = torch.zeros_like(y), torch.zeros_like(dx)
    da, db = torch.zeros(a.shape, device="cuda").double(), torch.zeros(b.shape, device="cuda").double()
    ea, eb = torch.zeros_like(da), torch.zeros_like(db)
    for g, t in enumerate(R.rows_of(c, a.shape[0])):
        if not t.numel():
            continue
        A, B, sg = a[g].double(), b[g].double(), s[g].double()
        u, v = sg * (xx[t] @ A.T), sg * (d[t] @ B)
        iu = inner(u, sg.abs() * (xx[t].abs() @ A.abs().T), K)
        iv = inner(v, sg.abs() * (d[t].abs() @ B.abs()), N)
        y[t] += u @ B.T
        dx[t] += v @ A
        my[t] += u.abs() @ B.abs().T
        mx[t] += v.abs() @ A.abs()
        ey[t] = (iu + u.abs() * 2.0 ** -16) @ B.abs().T
        ex[t] = (iv + v.abs() * 2.0 ** -16) @ A.abs()
        da[g], db[g] = v.T @ xx[t], d[t].T @ u
        T = t.numel()
        lu, lv = iu + u.abs() * low + u.abs().max() * 2.0 ** -38, iv + v.abs() * low + v.abs().max() * 2.0 ** -38
        ea[g] = (lv + v.abs() * (T + 64) * R.ADD).T @ xx[t].abs()
        eb[g] = d[t].abs().T @ (lu + u.abs() * (T + 64) * R.ADD)
    def rounded(v, e):
        return v, R.UNIT[dt] * (v.abs() + e) + e + R.FLOOR[dt]
    return [rounded(y, ey + (K + 2 * r + 64) * R.ADD * my), rounded(dx, ex + (N + 2 * r + 64) * R.ADD * mx),
            rounded(da, ea), rounded(db, eb)]


def inside(got, want, name):
    """A value beyond the type's range is infinite; the others are within their bounds."""
    exact, err = want
    over = exact.abs() > torch.finfo(got.dtype).max + err
    assert torch.equal(got[over].double(), torch.sign(exact[over]) * INF), name
    R.inside(torch.where(over, torch.zeros_like(got), got), (torch.where(over, torch.zeros_like(exact), exact), err), name)


def check_ends(ops, x, w, a, b, s, dy, c):
    plan = ops.dispatch(c, a.shape[0])
    want = ends(x, w, a, b, s, dy, c)
    inside(ops.adapter_forward(x, w, a, b, s, plan), want[0], "y")
    dx, da, db = ops.adapter_backward(dy, x, w, a, b, s, plan)
    inside(dx, want[1], "dx")
    inside(da, want[2], "da")
    inside(db, want[3], "db")
    alone, _, _ = ops.adapter_backward(dy, x, w, a, b, s, plan, need_dab=False)
    inside(alone, want[1], "dx alone")
    _, *both = ops.adapter_backward(dy, x, w, a, b, s, plan, need_dx=False)
    assert torch.equal(both[0], da) and torch.equal(both[1], db)


@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("T,G,K,N,r", [(17, 2, 64, 72, 8), (300, 5, 200, 136, 24), (5000, 3, 264, 256, 16),
                                       (3000, 7, 512, 300, 100), (900, 2, 128, 64, 33)])
def test_small_gradients(ops, dt, T, G, K, N, r):
    """dy of 1e-4 and a B near zero, as in an adapter's first steps: inner products of 1e-6,
    whose gradients are well inside fp16; a row of one group is far larger than the rest."""
    c = choices(T, G, "holes")
    x, w = make(T, K, dt=dt), make(N, K, std=K ** -0.5, dt=dt)
    a, b = make(G, r, K, std=1.0, dt=dt, seed=1), make(G, N, r, std=1e-3, dt=dt, seed=2)
    dy = make(T, N, std=1e-4, dt=dt, seed=3)
    check_ends(ops, x, w, a, b, torch.full((G,), 0.5, device="cuda"), dy, c)
    dy[T // 2] = 0.5
    check_ends(ops, x, w, a, b, torch.full((G,), 0.5, device="cuda"), dy, c)
    x[T // 3:] *= 2.0 ** -12
    check_ends(ops, x, w, a, b, torch.linspace(1e-3, 4, G, device="cuda"), dy, c)


@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("T", [1, 16, 17, 300, 5000])
def test_inner_products_beyond_half_precision(ops, dt, T):
    """Inner products of 1e6 beside small matrices on the other side: finite results,
    whatever the number of rows."""
    G, K, N, r = 2, 72, 136, 8
    c = choices(T, G, "any")
    x, w = make(T, K, std=100.0, dt=dt), make(N, K, std=K ** -0.5, dt=dt)
    a, b = make(G, r, K, std=200.0, dt=dt, seed=1), make(G, N, r, std=1e-4, dt=dt, seed=2)
    dy = make(T, N, std=0.01 / T, dt=dt, seed=3)
    s = torch.tensor([1.0, 8.0], device="cuda")
    assert float((x.double() @ a[1].double().T).abs().max()) * 8 > 65504
    check_ends(ops, x, w, a, b, s, dy, c)


@pytest.mark.parametrize("dt", [BF, HF])
def test_inner_products_beyond_half_precision_backward(ops, dt):
    """The same for those of the backward pass."""
    T, G, K, N, r = 400, 2, 136, 72, 8
    c = choices(T, G, "any")
    x, w = make(T, K, std=1e-5, dt=dt), make(N, K, std=K ** -0.5, dt=dt)
    a, b = make(G, r, K, std=1e-5, dt=dt, seed=1), make(G, N, r, std=200.0, dt=dt, seed=2)
    dy, s = make(T, N, std=50.0, dt=dt, seed=3), torch.tensor([1.0, 8.0], device="cuda")
    assert float((dy.double() @ b[1].double()).abs().max()) * 8 > 65504
    check_ends(ops, x, w, a, b, s, dy, c)


@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("T,K,N,r", [(5, 64, 72, 8), (16, 72, 64, 24), (40, 72, 64, 24), (300, 65, 130, 40),
                                     (300, 256, 320, 16), (5000, 136, 72, 8), (3000, 264, 200, 70)])
def test_infinities_give_what_they_give_in_64_bits(ops, dt, T, K, N, r):
    """Infinities in adapters, rows and gradients: infinite where the formula is, NaN only
    where it is (0 times an infinity, a difference of two)."""
    G = 7
    c = torch.arange(T, device="cuda", dtype=torch.int32) % (G + 1) - 1
    x, w, a, b, dy = (ints(*s, lo=-1, hi=1, dt=dt, seed=i) for i, s in
                      enumerate(((T, K), (N, K), (G, r, K), (G, N, r), (T, N))))
    s = 2.0 ** torch.randint(-1, 2, (G,), device="cuda").float()
    a[1, 3, 5], a[2, r - 1, K - 1] = INF, -INF
    b[3, 7, 2], b[4, N - 1, r - 1] = INF, -INF
    for g, v in ((5, INF), (6, -INF)):
        t = torch.nonzero(c == g).flatten()
        if t.numel():
            x[t[-1], 4], dy[t[0], 6] = v, -v
    plan = ops.dispatch(c, G)
    same(ops.adapter_forward(x, w, a, b, s, plan), R.adapter_forward(x, w, a, b, s, c)[0], dt)
    for got, (want, _) in zip(ops.adapter_backward(dy, x, w, a, b, s, plan), R.adapter_backward(dy, x, w, a, b, s, c)):
        same(got, want, dt)
    gw = ints(G, N, K, lo=-1, hi=1, dt=dt, seed=7)
    gw[1, 3, 5], gw[2, N - 1, K - 1] = INF, -INF
    same(ops.grouped_forward(x, gw, plan), R.grouped_forward(x, gw, c)[0], dt)
    for got, (want, _) in zip(ops.grouped_backward(dy, x, gw, plan), R.grouped_backward(dy, x, gw, c)):
        same(got, want, dt)
