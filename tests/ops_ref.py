"""Plain 64-bit restatements of the operators after a routing decision, and the
error each output may have, for the tests."""
import torch

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}       # half an ulp, relative
FLOOR = {torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -25}    # half the smallest step
# A product of two 16-bit values is exact in fp32.  Every addition of a sum of n
# of them, in whatever order, is off by at most 2^-22 of the sum of their
# magnitudes (twice fp32's rounding: the tensor cores may truncate), to first
# order n 2^-22 of it in all; adding pieces of a cut sum is n further terms at most.
ADD = 2.0 ** -22


def rows_of(choice, G):
    c = choice.cpu()
    return [torch.nonzero(c == g).flatten().to(choice.device) for g in range(G)]


def dispatch(choice, G):
    rows = rows_of(choice, G)
    none = torch.nonzero((choice < 0) | (choice >= G)).flatten()
    offsets = torch.tensor([0] + [r.numel() for r in rows]).cumsum(0)
    return offsets.to(torch.int32), torch.cat(rows + [none]).to(torch.int32)


def bound(exact, mags, terms, dt):
    """Error of a sum of `terms` products with magnitudes summing to `mags`, rounded once."""
    e = (terms + 64) * ADD * mags
    return UNIT[dt] * (exact.abs() + e) + e + FLOOR[dt]


def grouped_forward(x, w, choice):
    """(y, error bound)"""
    G, N, K = w.shape
    y = torch.zeros(x.shape[0], N, dtype=torch.float64, device=x.device)
    m = torch.zeros_like(y)
    for g, r in enumerate(rows_of(choice, G)):
        y[r] = x[r].double() @ w[g].double().T
        m[r] = x[r].double().abs() @ w[g].double().abs().T
    return y, bound(y, m, K, x.dtype)


def grouped_backward(dy, x, w, choice):
    """((dx, bound), (dw, bound))"""
    G, N, K = w.shape
    dx = torch.zeros(x.shape[0], K, dtype=torch.float64, device=x.device)
    dw = torch.zeros(G, N, K, dtype=torch.float64, device=x.device)
    mx, mw = torch.zeros_like(dx), torch.zeros_like(dw)
    d, xx = dy.double(), x.double()
    for g, r in enumerate(rows_of(choice, G)):
        dx[r], mx[r] = d[r] @ w[g].double(), d[r].abs() @ w[g].double().abs()
        dw[g], mw[g] = d[r].T @ xx[r], d[r].abs().T @ xx[r].abs()
    return (dx, bound(dx, mx, N, x.dtype)), (dw, bound(dw, mw, x.shape[0], x.dtype))


def _low(v, mags, terms, dt):
    """Error of a low-rank inner product: its sum's, its product with the scale
    (one fp32 rounding) and its two 16-bit terms'."""
    e = (terms + 64) * ADD * mags
    return e + (v.abs() + e) * (2.0 ** -23 + UNIT[dt] ** 2) + FLOOR[dt]


def adapter_forward(x, w, a, b, scale, choice):
    xx, ww = x.double(), w.double()
    K, R = w.shape[1], a.shape[1]
    y, m = xx @ ww.T, xx.abs() @ ww.abs().T
    extra = torch.zeros_like(y)
    for g, r in enumerate(rows_of(choice, a.shape[0])):
        A, B, s = a[g].double(), b[g].double(), scale[g].double()
        u = s * (xx[r] @ A.T)
        mu = s.abs() * (xx[r].abs() @ A.abs().T)
        y[r] += u @ B.T
        m[r] += (u.abs() + _low(u, mu, K, x.dtype)) @ B.abs().T
        extra[r] = _low(u, mu, K, x.dtype) @ B.abs().T
    e = bound(y, m, K + 2 * R, x.dtype)
    return y, e + extra * (1 + UNIT[x.dtype])


def adapter_backward(dy, x, w, a, b, scale, choice):
    d, xx, ww = dy.double(), x.double(), w.double()
    (N, K), R, T, dt = w.shape, a.shape[1], x.shape[0], x.dtype
    dx, mx = d @ ww, d.abs() @ ww.abs()
    ex = torch.zeros_like(dx)
    da, db = torch.zeros(a.shape, dtype=torch.float64, device=x.device), torch.zeros(b.shape, dtype=torch.float64, device=x.device)
    ea, eb = torch.zeros_like(da), torch.zeros_like(db)
    for g, r in enumerate(rows_of(choice, a.shape[0])):
        A, B, s = a[g].double(), b[g].double(), scale[g].double()
        u, mu = s * (xx[r] @ A.T), s.abs() * (xx[r].abs() @ A.abs().T)
        v, mv = s * (d[r] @ B), s.abs() * (d[r].abs() @ B.abs())
        lu, lv = _low(u, mu, K, dt), _low(v, mv, N, dt)
        dx[r] += v @ A
        mx[r] += (v.abs() + lv) @ A.abs()
        ex[r] = lv @ A.abs()
        da[g] = v.T @ xx[r]
        ea[g] = bound(da[g], 2 * (v.abs() + lv).T @ xx[r].abs(), T, dt) + lv.T @ xx[r].abs() * (1 + UNIT[dt])
        db[g] = d[r].T @ u
        eb[g] = bound(db[g], 2 * d[r].abs().T @ (u.abs() + lu), T, dt) + d[r].abs().T @ lu * (1 + UNIT[dt])
    return (dx, bound(dx, mx, N + 2 * R, dt) + ex * (1 + UNIT[dt])), (da, ea), (db, eb)


def inside(got, want, name=""):
    exact, err = want
    off = (got.double() - exact).abs()
    bad = ~(off <= err)
    assert not bad.any(), (name, int(bad.sum()), bad.numel(), float((off / err).max()),
                           torch.nonzero(bad)[:4].tolist())
