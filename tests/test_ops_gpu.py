"""The operators after a routing decision against plain 64-bit forms."""
import math

import pytest

torch = pytest.importorskip("torch")

import paper_2608_14575_gb300 as H
import ops_ref as R

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def ops():
    H.build()
    return H.Operators()


def make(*shape, std=1.0, dt=BF, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + 7919 * sum(shape))
    return torch.empty(shape, device="cuda", dtype=dt).normal_(0, std, generator=g)


def ints(*shape, lo=-2, hi=2, dt=BF, seed=0):
    """Small whole numbers: every sum below is exact in fp32."""
    g = torch.Generator(device="cuda").manual_seed(seed + 104729 * sum(shape))
    return torch.randint(lo, hi + 1, shape, device="cuda", generator=g).to(dt)


def choices(T, G, kind, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + 31 * T + G)
    c = torch.randint(0, G, (T,), device="cuda", generator=g, dtype=torch.int32)
    if kind == "none":
        c.fill_(-1)
    elif kind == "one":
        c.fill_(G - 1)
    elif kind == "holes":           # empty groups, and rows without a choice
        c = torch.where(c % 3 == 1, torch.full_like(c, -1), c)
    elif kind == "outside":
        c = torch.where(c % 2 == 0, c + G * 1000, c - 2 * G)
    elif kind == "skew":
        c = (c.double() ** 2 / max(G, 1)).to(torch.int32)
    return c


# ---- dispatch ---------------------------------------------------------------

@pytest.mark.parametrize("T", [0, 1, 31, 32, 33, 255, 256, 257, 4096, 4097, 8191, 8192, 8193, 50_001, 65_536,
                               65_537, 200_001, 1_300_003])
@pytest.mark.parametrize("G", [1, 2, 12, 64, 1023, 1024])
@pytest.mark.parametrize("kind", ["any", "none", "one", "holes", "outside"])
def test_dispatch(ops, T, G, kind):
    if T > 100_000 and kind in ("none", "outside"):
        pytest.skip("covered at smaller sizes")
    c = choices(T, G, kind)
    key = torch.where((c >= 0) & (c < G), c, torch.full_like(c, G)).long().cpu()
    plan = ops.dispatch(c, G)
    order = torch.argsort(key, stable=True)
    assert torch.equal(plan.order.cpu().long(), order)
    counts = torch.bincount(key, minlength=G + 1)[:G]
    assert torch.equal(plan.offsets.cpu().long(), torch.cat([torch.zeros(1, dtype=torch.long), counts.cumsum(0)]))


# ---- grouped products -----------------------------------------------------------

SHAPES = [   # T, G, K, N
    (1, 1, 8, 8), (1, 5, 64, 64), (3, 2, 72, 24), (64, 12, 256, 512), (127, 1, 64, 128),
    (128, 1, 128, 256), (129, 1, 192, 264), (300, 7, 1000, 520), (1000, 3, 128, 1024),
    (2500, 40, 256, 384), (5000, 4, 512, 776), (700, 1000, 64, 48),
    (200, 3, 1, 1), (77, 4, 33, 5), (260, 3, 101, 257), (64, 2, 4104, 40),
    # tiles cut along long contractions: few rows and many
    (100, 3, 4096, 512), (1000, 2, 4096, 256), (1025, 2, 4096, 256), (3000, 3, 2048, 512), (2100, 30, 328, 3000),
]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("kind", ["any", "holes", "skew"])
def test_grouped(ops, shape, dt, kind):
    T, G, K, N = shape
    c = choices(T, G, kind)
    x, w, dy = make(T, K, dt=dt), make(G, N, K, std=K ** -0.5, dt=dt), make(T, N, dt=dt, seed=3)
    plan = ops.dispatch(c, G)
    R.inside(ops.grouped_forward(x, w, plan), R.grouped_forward(x, w, c), "y")
    dx, dw = ops.grouped_backward(dy, x, w, plan)
    ex, ew = R.grouped_backward(dy, x, w, c)
    R.inside(dx, ex, "dx")
    R.inside(dw, ew, "dw")


@pytest.mark.parametrize("shape", [(1, 3, 64, 64), (130, 2, 128, 320), (1111, 9, 520, 200), (4096, 2, 256, 2048),
                                   (9000, 5, 264, 1032)])
@pytest.mark.parametrize("dt", [BF, HF])
def test_grouped_exact(ops, shape, dt):
    """Whole numbers: the one rounding of each output is all that may differ from 64 bits."""
    T, G, K, N = shape
    c = choices(T, G, "holes")
    x, w, dy = ints(T, K, dt=dt), ints(G, N, K, dt=dt), ints(T, N, dt=dt, seed=1)
    plan = ops.dispatch(c, G)
    assert torch.equal(ops.grouped_forward(x, w, plan), R.grouped_forward(x, w, c)[0].to(dt))
    dx, dw = ops.grouped_backward(dy, x, w, plan)
    (ex, _), (ew, _) = R.grouped_backward(dy, x, w, c)
    assert torch.equal(dx, ex.to(dt))
    assert torch.equal(dw, ew.to(dt))


@pytest.mark.parametrize("kind", ["none", "one", "outside"])
def test_grouped_rows_without_choice(ops, kind):
    T, G, K, N = 300, 6, 128, 192
    c = choices(T, G, kind)
    x, w, dy = ints(T, K), ints(G, N, K), ints(T, N, seed=1)
    x[c != G - 1] = float("nan")          # rows that no product may read into another's result
    plan = ops.dispatch(c, G)
    y = ops.grouped_forward(x, w, plan)
    dx, dw = ops.grouped_backward(dy, x, w, plan)
    none = (c < 0) | (c >= G)
    assert (y[none] == 0).all() and (dx[none] == 0).all()
    if kind != "one":
        assert (dw == 0).all()
    else:
        assert (dw[:-1] == 0).all() and torch.equal(y, R.grouped_forward(x, w, c)[0].to(BF))


def test_grouped_keeps_groups_apart(ops):
    """NaN and infinite weights, inputs and gradients of one group leave the others' results."""
    T, G, K, N = 500, 4, 200, 136
    c = choices(T, G, "any")
    x, w, dy = ints(T, K), ints(G, N, K), ints(T, N, seed=1)
    want, (wdx, wdw) = R.grouped_forward(x, w, c)[0].to(BF), [e.to(BF) for e, _ in R.grouped_backward(dy, x, w, c)]
    w[1, 5], x[c == 1] = float("nan"), float("inf")
    dy[c == 1] = float("nan")
    plan = ops.dispatch(c, G)
    keep = c != 1
    assert torch.equal(ops.grouped_forward(x, w, plan)[keep], want[keep])
    dx, dw = ops.grouped_backward(dy, x, w, plan)
    assert torch.equal(dx[keep], wdx[keep])
    for g in (0, 2, 3):
        assert torch.equal(dw[g], wdw[g])
    assert dw[1].isnan().all()


@pytest.mark.parametrize("pad,shift", [(8, 0), (3, 0), (0, 1), (5, 3)])
def test_grouped_strides(ops, pad, shift):
    """Rows apart, and addresses off the 16-byte grid."""
    T, G, K, N = 333, 3, 136, 72

    def wide(*shape, seed=0):
        rows = math.prod(shape[:-1])
        buf = torch.full((shift + rows * (shape[-1] + pad) + 8,), float("nan"), device="cuda", dtype=BF)
        v = buf[shift:shift + rows * (shape[-1] + pad)].view(*shape[:-1], shape[-1] + pad)[..., :shape[-1]]
        v.copy_(ints(*shape, seed=seed))
        return v
    c = choices(T, G, "holes")
    x, w, dy, out = wide(T, K), wide(G, N, K, seed=1), wide(T, N, seed=2), wide(T, N, seed=3)
    plan = ops.dispatch(c, G)
    y = ops.grouped_forward(x, w, plan, out=out)
    assert y is out and torch.equal(y, R.grouped_forward(x, w, c)[0].to(BF))
    dx, dw = ops.grouped_backward(dy, x, w, plan)
    (ex, _), (ew, _) = R.grouped_backward(dy, x, w, c)
    assert torch.equal(dx, ex.to(BF)) and torch.equal(dw, ew.to(BF))
    assert dw.stride() == w.stride()
    if pad:     # nothing beside the rows is written
        raw = out.as_strided((T, N + pad), out.stride())
        assert raw[:-1, N:].isnan().all()


def test_grouped_parts(ops):
    T, G, K, N = 65, 2, 64, 96
    c = choices(T, G, "any")
    x, w, dy = ints(T, K), ints(G, N, K), ints(T, N, seed=1)
    plan = ops.dispatch(c, G)
    dx, dw = ops.grouped_backward(dy, x, w, plan)
    a, none = ops.grouped_backward(dy, x, w, plan, need_dw=False)
    assert none is None and torch.equal(a, dx)
    none, b = ops.grouped_backward(dy, x, w, plan, need_dx=False)
    assert none is None and torch.equal(b, dw)


def test_grouped_differences(ops):
    """Gradients against central differences of the forward pass, which is linear in
    x and in w: the difference over any step is exact but for the outputs' rounding."""
    T, G, K, N = 90, 3, 64, 80
    c = choices(T, G, "holes")
    x, w, dy = ints(T, K), ints(G, N, K), ints(T, N, seed=1)
    plan = ops.dispatch(c, G)
    dx, dw = ops.grouped_backward(dy, x, w, plan)

    def loss(x, w):
        y = ops.grouped_forward(x, w, plan).double()
        return (y * dy.double()).sum(), (y.abs() * dy.double().abs()).sum() * R.UNIT[BF]
    for k in range(3):
        for which, grad in (("x", dx), ("w", dw)):
            d = ints(*grad.shape, lo=-1, hi=1, seed=20 + k)
            up, e0 = loss(x + d, w) if which == "x" else loss(x, w + d)
            down, e1 = loss(x - d, w) if which == "x" else loss(x, w - d)
            slope = (grad.double() * d.double()).sum()
            own = (grad.double().abs() * d.double().abs()).sum() * R.UNIT[BF]
            assert abs((up - down) / 2 - slope) <= (e0 + e1) / 2 + own


# ---- adapters -----------------------------------------------------------------

ADAPTERS = [   # T, G, K, N, rank
    (1, 1, 64, 64, 8), (1, 32, 256, 512, 16), (7, 3, 72, 136, 4), (64, 64, 512, 512, 16),
    (128, 5, 128, 256, 64), (129, 200, 64, 320, 24), (500, 3, 264, 200, 100), (1500, 4, 512, 1032, 32),
    (260, 2, 128, 64, 256), (3000, 12, 256, 512, 128), (90, 4, 33, 57, 5), (50, 2, 1, 3, 1),
    (300, 1000, 128, 64, 16),
    # picked rows on the tensor cores, cut tiles that share out their adapters
    (200, 3, 2048, 64, 128), (64, 40, 2048, 1024, 48), (250, 60, 1024, 2048, 16), (100, 100, 4096, 512, 8),
    (600, 50, 2048, 1024, 40), (17, 9, 1024, 640, 24), (16, 9, 1000, 648, 24), (400, 6, 2048, 2048, 16),
]


def adapter_inputs(T, G, K, N, r, dt):
    return (make(T, K, dt=dt), make(N, K, std=K ** -0.5, dt=dt), make(G, r, K, std=K ** -0.5, dt=dt, seed=1),
            make(G, N, r, std=r ** -0.5, dt=dt, seed=2), 0.5 + torch.rand(G, device="cuda"))


@pytest.mark.parametrize("shape", ADAPTERS)
@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("kind", ["any", "holes", "none"])
def test_adapter(ops, shape, dt, kind):
    T, G, K, N, r = shape
    c = choices(T, G, kind)
    x, w, a, b, s = adapter_inputs(T, G, K, N, r, dt)
    dy = make(T, N, dt=dt, seed=5)
    plan = ops.dispatch(c, G)
    R.inside(ops.adapter_forward(x, w, a, b, s, plan), R.adapter_forward(x, w, a, b, s, c), "y")
    got = ops.adapter_backward(dy, x, w, a, b, s, plan)
    for g, want, name in zip(got, R.adapter_backward(dy, x, w, a, b, s, c), ("dx", "da", "db")):
        R.inside(g, want, name)


@pytest.mark.parametrize("shape", [(1, 2, 64, 64, 16), (200, 3, 128, 320, 40), (1030, 11, 256, 264, 8),
                                   (2000, 2, 64, 128, 200)])
@pytest.mark.parametrize("dt", [BF, HF])
def test_adapter_exact(ops, shape, dt):
    """Whole numbers small enough for the two 16-bit terms of the inner products."""
    T, G, K, N, r = shape
    c = choices(T, G, "holes")
    x, w, a, b = (ints(*s, lo=-1, hi=1, dt=dt, seed=i) for i, s in
                  enumerate(((T, K), (N, K), (G, r, K), (G, N, r))))
    s = 2.0 ** torch.randint(-1, 2, (G,), device="cuda").float()
    dy = ints(T, N, lo=-1, hi=1, dt=dt, seed=9)
    plan = ops.dispatch(c, G)
    assert torch.equal(ops.adapter_forward(x, w, a, b, s, plan), R.adapter_forward(x, w, a, b, s, c)[0].to(dt))
    for g, (want, _) in zip(ops.adapter_backward(dy, x, w, a, b, s, plan),
                            R.adapter_backward(dy, x, w, a, b, s, c)):
        assert torch.equal(g, want.to(dt))


def test_adapter_keeps_groups_apart(ops):
    """A NaN or infinity in one adapter, or in one request's row, stays there, also
    where requests of several adapters share a tile."""
    T, G, K, N, r = 200, 6, 128, 192, 24
    c = choices(T, G, "holes")
    x, w, a, b = (ints(*s, lo=-1, hi=1, seed=i) for i, s in enumerate(((T, K), (N, K), (G, r, K), (G, N, r))))
    s, dy = torch.ones(G, device="cuda"), ints(T, N, lo=-1, hi=1, seed=9)
    want = R.adapter_forward(x, w, a, b, s, c)[0].to(BF)
    wdx, wda, wdb = (e.to(BF) for e, _ in R.adapter_backward(dy, x, w, a, b, s, c))
    a[2, 3], b[3] = float("nan"), float("inf")
    bad = int(torch.nonzero(c == 5)[0])
    x[bad], dy[bad] = float("nan"), float("inf")
    plan = ops.dispatch(c, G)
    keep = (c != 2) & (c != 3)
    keep[bad] = False
    y = ops.adapter_forward(x, w, a, b, s, plan)
    assert torch.equal(y[keep], want[keep]) and y[bad].isnan().all()
    dx, da, db = ops.adapter_backward(dy, x, w, a, b, s, plan)
    assert torch.equal(dx[keep], wdx[keep])
    for g in (0, 1, 4):
        assert torch.equal(da[g], wda[g]) and torch.equal(db[g], wdb[g])
    # what an adapter's gradients do not depend on does not reach them either:
    # dA reads B, not A; dB reads A, not B
    assert torch.equal(da[2], wda[2]) and torch.equal(db[3], wdb[3])


def test_adapter_infinite_inner_product(ops):
    """An inner product beyond the type's range is infinite, not NaN."""
    K, N, r = 64, 64, 8
    x, w = torch.full((1, K), 3e4, device="cuda", dtype=HF), torch.zeros(N, K, device="cuda", dtype=HF)
    a = torch.full((1, r, K), 1.0, device="cuda", dtype=HF)
    b = torch.full((1, N, r), 1.0, device="cuda", dtype=HF)
    y = ops.adapter_forward(x, w, a, b, torch.ones(1, device="cuda"), ops.dispatch(torch.zeros(1, device="cuda", dtype=torch.int32), 1))
    assert (y == float("inf")).all()


def test_adapter_differences(ops):
    """As for the grouped products: the forward pass is linear in x, a and b each."""
    T, G, K, N, r = 70, 3, 64, 96, 8
    c = choices(T, G, "holes")
    x, w, a, b = (ints(*s, lo=-1, hi=1, seed=i) for i, s in enumerate(((T, K), (N, K), (G, r, K), (G, N, r))))
    s, dy = torch.full((G,), 0.5, device="cuda"), ints(T, N, lo=-1, hi=1, seed=9)
    plan = ops.dispatch(c, G)
    grads = dict(zip("xab", ops.adapter_backward(dy, x, w, a, b, s, plan)))

    def loss(**by):
        v = dict(x=x, a=a, b=b) | by
        y = ops.adapter_forward(v["x"], w, v["a"], v["b"], s, plan).double()
        return (y * dy.double()).sum(), (y.abs() * dy.double().abs()).sum() * R.UNIT[BF]
    for name, at in (("x", x), ("a", a), ("b", b)):
        for k in range(2):
            d = ints(*at.shape, lo=-1, hi=1, seed=40 + k)
            (up, e0), (down, e1) = loss(**{name: at + d}), loss(**{name: at - d})
            g = grads[name].double()
            own = (g.abs() * d.double().abs()).sum() * R.UNIT[BF]
            assert abs((up - down) / 2 - (g * d.double()).sum()) <= (e0 + e1) / 2 + own, name


@pytest.mark.parametrize("pad,shift", [(8, 0), (3, 1)])
def test_adapter_strides(ops, pad, shift):
    T, G, K, N, r = 140, 3, 72, 200, 16

    def wide(rows, cols, seed):
        buf = torch.full((shift + rows * (cols + pad) + 8,), float("nan"), device="cuda", dtype=BF)
        v = buf[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
        v.copy_(ints(rows, cols, lo=-1, hi=1, seed=seed))
        return v
    c = choices(T, G, "holes")
    x, w, dy = wide(T, K, 0), wide(N, K, 1), wide(T, N, 2)
    a, b, s = ints(G, r, K, lo=-1, hi=1), ints(G, N, r, lo=-1, hi=1), torch.ones(G, device="cuda")
    plan = ops.dispatch(c, G)
    assert torch.equal(ops.adapter_forward(x, w, a, b, s, plan), R.adapter_forward(x, w, a, b, s, c)[0].to(BF))
    for g, (want, _) in zip(ops.adapter_backward(dy, x, w, a, b, s, plan),
                            R.adapter_backward(dy, x, w, a, b, s, c)):
        assert torch.equal(g, want.to(BF))


@pytest.mark.parametrize("K,N,r", [(72, 264, 8), (68, 300, 12), (66, 302, 6), (65, 301, 7), (300, 68, 36), (301, 65, 33)])
@pytest.mark.parametrize("T", [7, 100, 1500])
def test_results_of_each_alignment(ops, K, N, r, T):
    """Rows of results that are aligned to 16, 8, 4 and 2 bytes; what lies between
    the rows of a strided result stays."""
    G = 5
    c = choices(T, G, "holes")
    x, w, a, b, gw = (ints(*s, lo=-1, hi=1, seed=i) for i, s in
                      enumerate(((T, K), (N, K), (G, r, K), (G, N, r), (G, N, K))))
    dy, s = ints(T, N, lo=-1, hi=1, seed=9), torch.ones(G, device="cuda")
    plan = ops.dispatch(c, G)
    for g, (want, _) in zip(ops.grouped_backward(dy, x, gw, plan), R.grouped_backward(dy, x, gw, c)):
        assert torch.equal(g, want.to(BF))
    for g, (want, _) in zip(ops.adapter_backward(dy, x, w, a, b, s, plan),
                            R.adapter_backward(dy, x, w, a, b, s, c)):
        assert torch.equal(g, want.to(BF))
    for pad in (0, 1, 2, 4, 8):
        buf = torch.full((T, N + pad), 7.0, device="cuda", dtype=BF)
        ops.adapter_forward(x, w, a, b, s, plan, out=buf[:, :N])
        assert torch.equal(buf[:, :N], R.adapter_forward(x, w, a, b, s, c)[0].to(BF)) and (buf[:, N:] == 7).all()
        buf = torch.full((T, N + pad), 7.0, device="cuda", dtype=BF)
        ops.grouped_forward(x, gw, plan, out=buf[:, :N])
        assert torch.equal(buf[:, :N], R.grouped_forward(x, gw, c)[0].to(BF)) and (buf[:, N:] == 7).all()


@pytest.mark.parametrize("T,G,K,N,r", [(5000, 3, 1024, 256, 8), (3000, 40, 2048, 200, 40), (1500, 7, 4096, 96, 96),
                                       (1500, 5, 512, 384, 5), (700, 9, 256, 640, 33), (257, 2, 1536, 72, 16)])
@pytest.mark.parametrize("dt", [BF, HF])
def test_many_rows_of_narrow_products(ops, T, G, K, N, r, dt):
    """Rows of several tiles that are picked by index, tiles in pieces, inner
    products of many rows; also without the gradients that need a copy."""
    c = choices(T, G, "holes")
    x, w, a, b, gw = (ints(*s, lo=-1, hi=1, dt=dt, seed=i) for i, s in
                      enumerate(((T, K), (N, K), (G, r, K), (G, N, r), (G, N, K))))
    dy, s = ints(T, N, lo=-1, hi=1, dt=dt, seed=9), 2.0 ** torch.randint(-1, 2, (G,), device="cuda").float()
    plan = ops.dispatch(c, G)
    assert torch.equal(ops.grouped_forward(x, gw, plan), R.grouped_forward(x, gw, c)[0].to(dt))
    want = R.grouped_backward(dy, x, gw, c)[0][0].to(dt)
    assert torch.equal(ops.grouped_backward(dy, x, gw, plan, need_dw=False)[0], want)
    assert torch.equal(ops.grouped_backward(dy, x, gw, plan)[0], want)
    assert torch.equal(ops.adapter_forward(x, w, a, b, s, plan), R.adapter_forward(x, w, a, b, s, c)[0].to(dt))
    want = R.adapter_backward(dy, x, w, a, b, s, c)[0][0].to(dt)
    assert torch.equal(ops.adapter_backward(dy, x, w, a, b, s, plan, need_dab=False)[0], want)
    assert torch.equal(ops.adapter_backward(dy, x, w, a, b, s, plan)[0], want)


def test_same_bits_again(ops):
    """Cut tiles are joined in a fixed order: the same call gives the same bits."""
    T, G, K, N, r = 700, 5, 1024, 1040, 16
    c = choices(T, G, "skew")
    x, w, a, b, s = adapter_inputs(T, G, K, N, r, BF)
    dy, gw = make(T, N, seed=4), make(G, N, K, std=0.03, seed=5)
    plan = ops.dispatch(c, G)

    def all_of():
        return [ops.grouped_forward(x, gw, plan), *ops.grouped_backward(dy, x, gw, plan),
                ops.adapter_forward(x, w, a, b, s, plan), *ops.adapter_backward(dy, x, w, a, b, s, plan)]
    first = all_of()
    for _ in range(5):
        assert all(torch.equal(p, q) for p, q in zip(first, all_of()))


def test_other_streams(ops):
    """A call under another current stream is ordered between that stream's work."""
    T, G, K, N = 2000, 4, 512, 512
    c = choices(T, G, "any")
    w = ints(G, N, K)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for k in range(4):
            x = torch.zeros(T, K, device="cuda", dtype=BF)
            torch.cuda._sleep(2_000_000)
            x.copy_(ints(T, K, seed=k))
            y = ops.grouped_forward(x, w, ops.dispatch(c, G))
            got = y.clone()
            y.zero_()
            assert torch.equal(got, R.grouped_forward(x, w, c)[0].to(BF))
    side_ops = None
    with torch.cuda.stream(side):
        side_ops = H.Operators()
    x = ints(T, K, seed=11)
    y = side_ops.grouped_forward(x, w, side_ops.dispatch(c, G))     # the default stream is current
    assert torch.equal(y, R.grouped_forward(x, w, c)[0].to(BF))
    side_ops.synchronize()
    side_ops.close()


def test_graph_capture(ops):
    """After a call of the same sizes nothing is allocated: a step can be captured and
    replayed on new values, by a context on the capturing stream or another one.  (The
    legacy default stream takes no part in a capture: its context says so, and stays usable.)"""
    T, G, K, N, r = 48, 6, 256, 384, 16
    c, x = choices(T, G, "any"), ints(T, K)
    w, b = ints(G, N, K), ints(G, K, r, lo=-1, hi=1)
    a, sh, s = ints(G, r, N, lo=-1, hi=1), ints(K, N, lo=-1, hi=1), torch.ones(G, device="cuda")
    torch.cuda.synchronize()

    def step(o):
        plan = o.dispatch(c, G)
        y = o.grouped_forward(x, w, plan)
        g = y.clone()
        return y, o.adapter_forward(y, sh, a, b, s, plan), o.clip_gradients([g], 1e9), g
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    for on in (side, other):
        with torch.cuda.stream(on):
            own = H.Operators()
        with torch.cuda.stream(side):
            step(own)
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                held = step(own)
            for k in range(3):
                x.copy_(ints(T, K, seed=k))
                c.copy_(choices(T, G, "holes", seed=k))
                graph.replay()
                now = step(own)
                for p, q in zip(held, now):
                    assert torch.equal(p, q)
                assert torch.equal(held[0], R.grouped_forward(x, w, c)[0].to(BF))
        torch.cuda.synchronize()
        own.close()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        with pytest.raises(H.HwrError) as e:
            ops.dispatch(c, G)
        assert e.value.status == 7
    assert ops.dispatch(c, G).offsets.shape == (G + 1,)


def test_no_rows(ops):
    c = torch.empty(0, device="cuda", dtype=torch.int32)
    plan = ops.dispatch(c, 3)
    assert plan.offsets.tolist() == [0, 0, 0, 0]
    x, w = torch.empty(0, 16, device="cuda", dtype=BF), ints(3, 24, 16)
    assert ops.grouped_forward(x, w, plan).shape == (0, 24)
    dx, dw = ops.grouped_backward(torch.empty(0, 24, device="cuda", dtype=BF), x, w, plan)
    assert dx.shape == (0, 16) and (dw == 0).all()
    a, b, s = ints(3, 4, 16), ints(3, 24, 4), torch.ones(3, device="cuda")
    assert ops.adapter_forward(x, w[0], a, b, s, plan).shape == (0, 24)
    dx, da, db = ops.adapter_backward(torch.empty(0, 24, device="cuda", dtype=BF), x, w[0], a, b, s, plan)
    assert dx.shape == (0, 16) and (da == 0).all() and (db == 0).all()


def test_foreign_plan_stays_inside(ops):
    """Offsets and orders that no dispatch made: wrong results, no access outside."""
    T, G, K, N = 300, 4, 64, 64
    x, w = ints(T, K), ints(G, N, K)
    for offsets in ([0, 5000, -7, 20, 1 << 30], [-5, -5, -5, -5, -5], [300, 200, 100, 50, 0], [0, 300, 0, 300, 0]):
        plan = H.Plan(torch.tensor(offsets, device="cuda", dtype=torch.int32),
                      torch.randint(-(1 << 31), (1 << 31) - 1, (T,), device="cuda").to(torch.int32))
        a, b, s = ints(G, 8, K), ints(G, N, 8), torch.ones(G, device="cuda")
        ops.grouped_forward(x, w, plan)
        ops.grouped_backward(ints(T, N), x, w, plan)
        ops.adapter_forward(x, w[0], a, b, s, plan)
        ops.adapter_backward(ints(T, N), x, w[0], a, b, s, plan)
    ops.synchronize()


# ---- clipping -------------------------------------------------------------------

@pytest.mark.parametrize("dt", [torch.float32, BF, HF])
@pytest.mark.parametrize("sizes", [[1], [7, 0, 33], [16384, 8192, 5], [100_003, 65_536, 1, 262_144],
                                   [3_000_001] * 3, [300] * 700])
@pytest.mark.parametrize("factor", [0.5, 2.0])
def test_clip(ops, dt, sizes, factor):
    grads = [make(n, std=0.1 * (1 + i % 3), dt=dt, seed=i) for i, n in enumerate(sizes)]
    norm = math.sqrt(sum(float(g.double().square().sum()) for g in grads))
    limit = norm * factor
    keep = [g.clone() for g in grads]
    out = [torch.full_like(g, float("nan")) for g in grads]
    got = ops.clip_gradients(grads, limit, out=out)
    # fp32 sums of at most 512 squares a thread, a rounding each; then 64 bits
    assert abs(float(got) - norm) <= norm * 512 * 2.0 ** -24
    assert all(torch.equal(a, b) for a, b in zip(grads, keep))
    k = min(1.0, limit / (norm + 1e-6))
    unit = 2.0 ** -24 if dt is torch.float32 else R.UNIT[dt]
    floor = 2.0 ** -150 if dt is not HF else R.FLOOR[HF]
    for g, o in zip(keep, out):
        want = g.double() * k
        assert ((o.double() - want).abs() <= want.abs() * (unit + 516 * 2.0 ** -24) + floor).all()
    once = ops.gradient_list(grads, [o.zero_() for o in out])
    for _ in range(2):
        assert float(ops.clip_gradients(once, limit)) == float(got)
    for g, o in zip(keep, out):
        want = g.double() * k
        assert ((o.double() - want).abs() <= want.abs() * (unit + 516 * 2.0 ** -24) + floor).all()
    once.close()
    again = ops.clip_gradients(grads, limit)                 # in place
    assert float(again) == float(got)
    assert all(torch.equal(a, b) for a, b in zip(grads, out))


def test_clip_unaligned(ops):
    buf = make(100_000, dt=BF)
    grads = [buf[1:40_000], buf[40_001:99_999]]
    edge = buf[[0, 40_000, 99_999]].clone()
    norm = math.sqrt(sum(float(g.double().square().sum()) for g in grads))
    want = [g.double() * (0.25 * norm / (norm + 1e-6)) for g in grads]
    ops.clip_gradients(grads, 0.25 * norm)
    for g, v in zip(grads, want):
        assert ((g.double() - v).abs() <= v.abs() * (R.UNIT[BF] + 516 * 2.0 ** -24)).all()
    assert torch.equal(buf[[0, 40_000, 99_999]], edge)


@pytest.mark.parametrize("value", [1e25, 3e38, 1e-25, 1e-38])
def test_clip_range(ops, value):
    """Squares outside fp32's range."""
    g = torch.full((20_000,), value, device="cuda")
    got = float(ops.clip_gradients([g, torch.zeros(50_000, device="cuda")], float("inf")))
    want = float(torch.tensor(value)) * math.sqrt(20_000)
    if want > 3.4028234e38:
        assert got == float("inf")
    else:
        assert abs(got - want) <= 1e-6 * want
    assert (g == torch.tensor(value)).all()


def test_clip_not_finite(ops):
    g = make(5000, dt=torch.float32)
    g[17] = float("inf")
    norm = ops.clip_gradients([g], 1.0)
    assert float(norm) == float("inf") and g[17].isnan() and (g[:17] == 0).all()
    g = make(5000, dt=BF)
    g[4999] = float("nan")
    norm = ops.clip_gradients([g, make(3, dt=torch.float32)], 1.0)
    assert norm.isnan() and g.isnan().all()


def test_clip_nothing(ops):
    assert float(ops.clip_gradients([], 1.0)) == 0.0
    z = torch.zeros(100, device="cuda")
    assert float(ops.clip_gradients([z], 1.0)) == 0.0 and (z == 0).all()


# ---- refusals -------------------------------------------------------------------

def test_refusals(ops):
    c = choices(10, 3, "any")
    plan = ops.dispatch(c, 3)
    x, w, dy = ints(10, 16), ints(3, 24, 16), ints(10, 24)
    a, b, s = ints(3, 4, 16), ints(3, 24, 4), torch.ones(3, device="cuda")
    with pytest.raises(TypeError):
        ops.dispatch(c.long(), 3)
    with pytest.raises(ValueError):
        ops.dispatch(c, 0)
    with pytest.raises(ValueError):
        ops.dispatch(c.cpu(), 3)
    with pytest.raises(H.HwrError):
        ops.dispatch(c, H.HWR_OPS_MAX_GROUPS + 1)
    with pytest.raises(TypeError):
        ops.grouped_forward(x.float(), w.float(), plan)
    with pytest.raises(TypeError):
        ops.grouped_forward(x, w.half(), plan)
    with pytest.raises(ValueError):
        ops.grouped_forward(x[:9], w, plan)
    with pytest.raises(ValueError):
        ops.grouped_forward(x, w[:2], plan)
    with pytest.raises(ValueError):
        ops.grouped_forward(x.cpu(), w, plan)
    with pytest.raises(ValueError):
        ops.grouped_forward(ints(16, 10).T, w, plan)
    with pytest.raises(ValueError):
        ops.grouped_backward(dy[:, :23], x, w, plan)
    with pytest.raises(ValueError):
        ops.grouped_forward(x[:1].expand(10, 16), w, plan)
    with pytest.raises(ValueError):
        ops.adapter_forward(x, w[0], a, b[:, :, :3], s, plan)
    with pytest.raises(ValueError):
        ops.adapter_forward(x, w[0], a, b, s.double(), plan)
    with pytest.raises(ValueError):
        ops.adapter_forward(x, w[0], a.transpose(0, 1).contiguous().transpose(0, 1), b, s, plan)
    big = ints(3, H.HWR_OPS_MAX_RANK + 1, 16)
    with pytest.raises(H.HwrError):
        ops.adapter_forward(x, w[0], big, ints(3, 24, H.HWR_OPS_MAX_RANK + 1), s, plan)
    with pytest.raises(H.HwrError):
        ops.clip_gradients([torch.ones(3, device="cuda")], 0.0)
    with pytest.raises(H.HwrError):
        ops.clip_gradients([torch.ones(3, device="cuda")], float("nan"))
    with pytest.raises(TypeError):
        ops.clip_gradients([torch.ones(3, device="cuda", dtype=torch.float64)], 1.0)
    with pytest.raises(ValueError):
        ops.clip_gradients([torch.ones(4, 4, device="cuda").T[:2]], 1.0)
    # the context is as it was
    assert torch.equal(ops.grouped_forward(x, w, plan), R.grouped_forward(x, w, c)[0].to(BF))


@pytest.mark.parametrize("T", [40, 600])
def test_timeout(monkeypatch, T):
    """A producer that never loads (the test hook): the kernel's waits run out, the
    call's failure is reported, the context is broken, and a new one works."""
    monkeypatch.setenv("HWR_TEST_STALL", "1")
    bad = H.Operators()
    monkeypatch.delenv("HWR_TEST_STALL")
    c = choices(T, 3, "any")
    x, w = ints(T, 256), ints(3, 512, 256)
    bad.grouped_forward(x, w, bad.dispatch(c, 3))
    with pytest.raises(H.HwrError) as e:
        bad.synchronize()
    assert e.value.status == 5
    with pytest.raises(H.HwrError) as e:
        bad.dispatch(c, 3)
    assert e.value.status == 6
    bad.close()
    good = H.Operators()
    assert torch.equal(good.grouped_forward(x, w, good.dispatch(c, 3)), R.grouped_forward(x, w, c)[0].to(BF))
    good.close()


def test_allocation_failure(monkeypatch):
    monkeypatch.setenv("HWR_TEST_FAIL_ALLOC", "2")
    with pytest.raises(H.HwrError) as e:
        H.Operators()
    assert e.value.status == 3


def test_example_learns():
    """The example runs the operators together after a routing call."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "routed_layer.py")
    spec = importlib.util.spec_from_file_location("routed_layer", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    for losses in example.main(Q=1024, width=256, steps=6, say=lambda *a: None):
        assert all(b < a for a, b in zip(losses, losses[1:])), losses
