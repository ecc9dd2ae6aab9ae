"""What a context does around its calls: order, refusals, lifetimes."""
import pytest

torch = pytest.importorskip("torch")

import paper_2608_14575_gb300 as H
import ops_ref as R
from test_ops_gpu import BF, choices, ints

pytestmark = pytest.mark.gpu


@pytest.fixture
def ops():
    """A context on a stream of its own, while the default stream is current."""
    H.build()
    ops = H.Operators(torch.cuda.Stream())
    yield ops
    ops.close()


def test_a_failed_call_is_ordered_too(ops):
    """What the caller frees after a failed call goes to its own stream's next work,
    which has to wait for whatever the context's stream still runs."""
    c = choices(10, 3, "any")
    plan = ops.dispatch(c, 3)
    R1 = H.HWR_OPS_MAX_RANK + 1
    args = ints(10, 16), ints(24, 16), ints(3, R1, 16), ints(3, 24, R1), torch.ones(3, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(ops.stream):
        torch.cuda._sleep(400_000_000)          # some 0.2 s
    with pytest.raises(H.HwrError) as e:
        ops.adapter_forward(*args, plan)
    assert e.value.status == 7 and "rank" in str(e.value)
    done = torch.cuda.Event()
    done.record()
    early, busy = done.query(), not ops.stream.query()
    torch.cuda.synchronize()
    assert busy and not early


def test_another_current_device(monkeypatch):
    """Refused before anything is launched, and nothing breaks.  (The test hook makes the
    current device seem another one.)"""
    monkeypatch.setenv("HWR_TEST_DEVICE", "1")
    off = H.Operators()
    monkeypatch.delenv("HWR_TEST_DEVICE")
    for _ in range(2):
        with pytest.raises(H.HwrError) as e:
            off.dispatch(choices(10, 3, "any"), 3)
        assert e.value.status == 1 and "device 1 is current" in str(e.value)
    off.close()


def test_lists_go_with_their_context():
    """A gradient list that outlives its closed context leaves no device memory behind."""
    H.build()
    grads = [torch.zeros(1 << 28, device="cuda", dtype=BF)]     # (a table of 1 MB)
    norms = []

    def cycle():
        ops = H.Operators()
        one, two = ops.gradient_list(grads), ops.gradient_list(grads)
        norms.append(float(ops.clip_gradients(one, 1.0)) + float(ops.clip_gradients(two, 1.0)))
        one.close()
        ops.close()
        two.close()
    for _ in range(3):
        cycle()
    torch.cuda.synchronize()
    before = torch.cuda.mem_get_info()[0]
    for _ in range(40):
        cycle()
    torch.cuda.synchronize()
    assert before - torch.cuda.mem_get_info()[0] < 8 << 20      # (40 MB if they stayed)
    assert norms == [0.0] * 43


def test_written_tensors_count_as_modified(ops):
    """Autograd sees what a call writes into a tensor of the caller's."""
    for lists in (False, True):
        for place in (False, True):
            grads = [torch.ones(n, device="cuda") for n in (5, 70_000)]
            out = grads if place else [torch.empty_like(g) for g in grads]
            it = ops.gradient_list(grads, None if place else out) if lists else grads
            before = [g._version for g in grads], [o._version for o in out]
            ops.clip_gradients(it, 1.0, **({} if lists or place else {"out": out}))
            assert all(o._version > v for o, v in zip(out, before[1]))
            assert place or [g._version for g in grads] == before[0]
    t = torch.ones(100, device="cuda", requires_grad=True)
    z = t.exp()                                             # saved for the backward pass
    ops.clip_gradients([z.detach()], 1.0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        z.sum().backward()
    c, x, w = choices(10, 3, "any"), ints(10, 16), ints(3, 24, 16)
    a, b, s = ints(3, 4, 16), ints(3, 24, 4), torch.ones(3, device="cuda")
    plan = ops.dispatch(c, 3)
    for call in (lambda y: ops.grouped_forward(x, w, plan, out=y),
                 lambda y: ops.adapter_forward(x, w[0], a, b, s, plan, out=y)):
        y = torch.empty(10, 24, device="cuda", dtype=BF)
        v = y._version
        assert call(y) is y and y._version > v
    with torch.inference_mode():                            # (no version to count)
        g = torch.ones(10, device="cuda")
        ops.clip_gradients([g], 1.0)


@pytest.mark.parametrize("T", [4097, 32_768, 32_769, 65_536, 65_537, 300_001])
@pytest.mark.parametrize("G", [1, 64, 1024])
def test_dispatch_where_clusters_of_16_do_not_fit(monkeypatch, T, G):
    """With clusters of the portable size (the test hook): the same plan."""
    monkeypatch.setenv("HWR_TEST_SMALL_CLUSTERS", "1")
    small = H.Operators()
    monkeypatch.delenv("HWR_TEST_SMALL_CLUSTERS")
    c = choices(T, G, "holes")
    offsets, order = R.dispatch(c, G)
    plan = small.dispatch(c, G)
    assert torch.equal(plan.order.cpu(), order.cpu()) and torch.equal(plan.offsets.cpu(), offsets)
    small.close()


def test_two_contexts_at_work_at_once():
    """Each has its own workspace, partial sums and counters."""
    H.build()
    T, G, K, N, r = 700, 5, 1024, 1040, 16
    c = choices(T, G, "holes")
    x, w, a, b, dy, gw = (ints(*s, lo=-1, hi=1, seed=i) for i, s in
                          enumerate(((T, K), (N, K), (G, r, K), (G, N, r), (T, N), (G, N, K))))
    s = torch.ones(G, device="cuda")
    want = [R.grouped_forward(x, gw, c)[0].to(BF), *(e.to(BF) for e, _ in R.grouped_backward(dy, x, gw, c)),
            R.adapter_forward(x, w, a, b, s, c)[0].to(BF), *(e.to(BF) for e, _ in R.adapter_backward(dy, x, w, a, b, s, c))]
    norm = float(torch.cat([e.double().flatten() for e in want]).square().sum().sqrt())
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    both, got = [], []
    for stream in streams:
        with torch.cuda.stream(stream):
            both.append(H.Operators())
    for _ in range(8):
        for stream, ops in zip(streams, both):
            with torch.cuda.stream(stream):
                plan = ops.dispatch(c, G)
                out = [ops.grouped_forward(x, gw, plan), *ops.grouped_backward(dy, x, gw, plan),
                       ops.adapter_forward(x, w, a, b, s, plan), *ops.adapter_backward(dy, x, w, a, b, s, plan)]
                got.append((out, ops.clip_gradients([t.clone() for t in out], 1.0)))
    torch.cuda.synchronize()
    for out, n in got:
        assert all(torch.equal(p, q) for p, q in zip(out, want))
        assert abs(float(n) - norm) <= 1e-6 * norm
    for ops in both:
        ops.close()


def test_element_offsets_beyond_32_bits(ops):
    """Rows, weights and results 2^25 elements apart: offsets up to 2.3e9."""
    T, G, K, N, r, far = 70, 70, 64, 72, 8, 1 << 25

    def apart(n, *shape, seed=0):
        buf = torch.empty((n - 1) * far + shape[0] * (shape[1] if len(shape) > 1 else 1) + 8, device="cuda", dtype=BF)
        v = buf.as_strided((n, *shape), (far, *((shape[1], 1) if len(shape) > 1 else (1,))))
        v.copy_(ints(n, *shape, lo=-1, hi=1, seed=seed))
        return v
    c = choices(T, G, "holes")
    x, dy, y, gw = apart(T, K), apart(T, N, seed=1), apart(T, N, seed=2), apart(G, N, K, seed=3)
    w, a, b, s = ints(N, K), ints(G, r, K), ints(G, N, r), torch.ones(G, device="cuda")
    plan = ops.dispatch(c, G)
    assert torch.equal(ops.grouped_forward(x, gw, plan, out=y), R.grouped_forward(x, gw, c)[0].to(BF))
    for got, (want, _) in zip(ops.grouped_backward(dy, x, gw, plan), R.grouped_backward(dy, x, gw, c)):
        assert torch.equal(got, want.to(BF))
    del gw
    assert torch.equal(ops.adapter_forward(x, w, a, b, s, plan, out=y), R.adapter_forward(x, w, a, b, s, c)[0].to(BF))
    few = ops.dispatch(c[:9], G)
    assert torch.equal(ops.adapter_forward(x[-9:], w, a, b, s, few, out=y[-9:]),
                       R.adapter_forward(x[-9:], w, a, b, s, c[:9])[0].to(BF))
    for got, (want, _) in zip(ops.adapter_backward(dy, x, w, a, b, s, plan), R.adapter_backward(dy, x, w, a, b, s, c)):
        assert torch.equal(got, want.to(BF))


@pytest.mark.parametrize("dt", [BF, torch.float16])
def test_foreign_plans_write_nothing_beside_the_results(dt):
    """Offsets and orders that no dispatch made: the results are wrong, but what lies beside
    them and the inputs stay as they are (the C interface, with results in guarded buffers)."""
    import ctypes as ct
    from paper_2608_14575_gb300 import _hwr, _ops
    lib = _ops.load_ops()
    T, G, K, N, r, edge = 300, 4, 64, 72, 40, 4096
    x, w, dy, a, b = (ints(*s, dt=dt, seed=i) for i, s in enumerate(((T, K), (G, N, K), (T, N), (G, r, K), (G, N, r))))
    s = torch.ones(G, device="cuda")
    inputs = x, w, dy, a, b, s
    kept = [t.clone() for t in inputs]
    ctx = ct.c_void_p()
    assert lib.hwr_ops_create(None, ct.byref(ctx)) == _hwr.HWR_OK
    guards = []

    def guarded(n):
        buf = torch.full((n + 2 * edge,), 7.0, device="cuda", dtype=dt)
        guards.append((buf, n))
        return ct.c_void_p(buf.data_ptr() + 2 * edge)
    order = torch.randint(-(1 << 31), (1 << 31) - 1, (T,), device="cuda").to(torch.int32)
    near = torch.randint(-2, T + 2, (T,), device="cuda", dtype=torch.int32)
    for offsets in ([0, 5000, -7, 20, 1 << 30], [-5, -5, -5, -5, -5], [300, 200, 100, 50, 0], [0, 300, 0, 300, 0]):
        o = torch.tensor(offsets, device="cuda", dtype=torch.int32)
        for p in (order, near):
            torch.cuda.synchronize()
            rows = _ops.hwr_rows(T, G, K, N, H.HWR_F16 if dt is torch.float16 else _hwr.HWR_BF16, o.data_ptr(), p.data_ptr(),
                                 x.data_ptr(), K, w.data_ptr(), K, N * K)
            ad = _ops.hwr_adapters(r, a.data_ptr(), b.data_ptr(), s.data_ptr())
            R_, A_, d = ct.byref(rows), ct.byref(ad), ct.c_void_p(dy.data_ptr())
            assert lib.hwr_grouped_forward(ctx, R_, guarded(T * N), N) == 0
            assert lib.hwr_grouped_backward(ctx, R_, d, N, guarded(T * K), K, guarded(G * N * K)) == 0
            assert lib.hwr_grouped_backward(ctx, R_, d, N, guarded(T * K), K, None) == 0
            assert lib.hwr_adapter_forward(ctx, R_, A_, guarded(T * N), N) == 0
            assert lib.hwr_adapter_backward(ctx, R_, A_, d, N, guarded(T * K), K, guarded(G * r * K), guarded(G * N * r)) == 0
            assert lib.hwr_ops_synchronize(ctx) == 0
    for buf, n in guards:
        assert (buf[:edge] == 7).all() and (buf[edge + n:] == 7).all()
    for t, k in zip(inputs, kept):
        assert torch.equal(t, k)
    assert lib.hwr_ops_destroy(ctx) == 0


@pytest.mark.parametrize("dt", [BF, torch.float16])
def test_each_result_of_the_adapters_backward_alone(dt):
    """The C interface takes any of dx, dA and dB: the same bits as all three together."""
    import ctypes as ct
    from paper_2608_14575_gb300 import _hwr, _ops
    lib = _ops.load_ops()
    T, G, K, N, r = 333, 5, 136, 72, 40
    c = choices(T, G, "holes")
    x, w, dy, a, b = (ints(*s, lo=-1, hi=1, dt=dt, seed=i) for i, s in
                      enumerate(((T, K), (N, K), (T, N), (G, r, K), (G, N, r))))
    s = torch.ones(G, device="cuda")
    torch.cuda.synchronize()
    ctx = ct.c_void_p()
    assert lib.hwr_ops_create(None, ct.byref(ctx)) == 0
    offsets, order = (torch.empty(n, device="cuda", dtype=torch.int32) for n in (G + 1, T))
    P = lambda t: ct.c_void_p(t.data_ptr())  # noqa: E731
    assert lib.hwr_dispatch(ctx, T, G, P(c), P(offsets), P(order)) == 0
    rows = _ops.hwr_rows(T, G, K, N, H.HWR_F16 if dt is torch.float16 else _hwr.HWR_BF16, offsets.data_ptr(), order.data_ptr(),
                         x.data_ptr(), K, w.data_ptr(), K, 0)
    ad = _ops.hwr_adapters(r, a.data_ptr(), b.data_ptr(), s.data_ptr())
    want = [e.to(dt) for e, _ in R.adapter_backward(dy, x, w, a, b, s, c)]
    for which in range(1, 8):
        out = [torch.full_like(e, 7) if which >> i & 1 else None for i, e in enumerate(want)]
        torch.cuda.synchronize()
        p = [None if o is None else P(o) for o in out]
        assert lib.hwr_adapter_backward(ctx, ct.byref(rows), ct.byref(ad), P(dy), N, p[0], K, p[1], p[2]) == 0
        assert lib.hwr_ops_synchronize(ctx) == 0
        for o, e in zip(out, want):
            assert o is None or torch.equal(o, e)
    assert lib.hwr_ops_destroy(ctx) == 0
