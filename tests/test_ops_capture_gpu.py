"""The operators in captured graphs, beside eager calls of the same context."""
import pytest

torch = pytest.importorskip("torch")

import paper_2608_14575_gb300 as H
import ops_ref as R
from test_ops_gpu import BF, choices, ints

pytestmark = pytest.mark.gpu
UNSUPPORTED = 7


@pytest.fixture
def side():
    """A context on a stream of its own."""
    H.build()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ops = H.Operators()
        yield ops, stream
    torch.cuda.synchronize()
    ops.close()


def layer(T, G=5, K=264, N=200, r=24, seed=0):
    c = choices(T, G, "holes", seed=seed)
    t = [ints(*s, lo=-1, hi=1, seed=seed + i) for i, s in enumerate(((T, K), (N, K), (G, r, K), (G, N, r), (T, N)))]
    return [c, *t, torch.ones(G, device="cuda")]


def step(ops, c, x, w, a, b, dy, s):
    """Everything that takes workspace: sorted rows, padded weights, inner products, a gradient table."""
    plan = ops.dispatch(c, a.shape[0])
    y = ops.adapter_forward(x, w, a, b, s, plan)
    grads = ops.adapter_backward(dy, x, w, a, b, s, plan)
    clipped = [g.clone() for g in grads]
    return [y, *grads, ops.clip_gradients(clipped, 1.0), *clipped]


def want(c, x, w, a, b, dy, s):
    return [R.adapter_forward(x, w, a, b, s, c)[0].to(BF),
            *(e.to(BF) for e, _ in R.adapter_backward(dy, x, w, a, b, s, c))]


def test_graphs_outlive_a_larger_call(side):
    """Graphs of growing sizes captured on one context: each keeps the workspace it was
    captured with, also when that has given way to a larger one and other memory is taken."""
    ops, stream = side
    graphs = []
    for T in (20, 300, 1500):
        args = layer(T)
        step(ops, *args)                        # grows the workspace: the graphs before hold theirs
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            held = step(ops, *args)
        graphs.append((graph, held, args))
    step(ops, *layer(6000))
    # memory that was given back would be handed out here
    guard = [torch.full((1 << 20,), 7, device="cuda", dtype=torch.int8) for _ in range(200)]
    for k in range(2):
        for graph, held, (c, x, w, a, b, dy, s) in graphs:
            T, G = c.numel(), a.shape[0]
            c.copy_(choices(T, G, "any", seed=50 + k))
            x.copy_(ints(*x.shape, lo=-1, hi=1, seed=70 + k))
            dy.copy_(ints(*dy.shape, lo=-1, hi=1, seed=90 + k))
            graph.replay()
            for got, exact in zip(held, want(c, x, w, a, b, dy, s)):
                assert torch.equal(got, exact)
            again = step(ops, c, x, w, a, b, dy, s)
            for p, q in zip(held, again):
                assert torch.equal(p, q)
    assert all(bool((g == 7).all()) for g in guard)


@pytest.mark.parametrize("mine", [True, False])
def test_growing_in_a_capture_is_refused(side, mine):
    """The call says so, queues nothing, and leaves the context and the capture as they
    were; on the context's own stream and on another."""
    ops, stream = side
    on = stream if mine else torch.cuda.Stream()
    small, large = layer(30), layer(3000)
    with torch.cuda.stream(on):
        step(ops, *small)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=on):
            plan = ops.dispatch(large[0], 5)
            with pytest.raises(H.HwrError) as e:
                ops.adapter_backward(large[5], *large[1:5], large[6], plan)
            assert e.value.status == UNSUPPORTED
            with pytest.raises(H.HwrError) as e:
                ops.reserve(1 << 32)
            assert e.value.status == UNSUPPORTED
            held = step(ops, *small)
        graph.replay()
        c, x, w, a, b, dy, s = small
        for got, exact in zip(held, want(c, x, w, a, b, dy, s)):
            assert torch.equal(got, exact)
        for got, exact in zip(step(ops, *large), want(*large)):
            assert torch.equal(got, exact)


def test_a_list_stays_under_its_graph(side):
    """A gradient list that is closed after a capture leaves its table to the graph."""
    ops, stream = side
    grads = [ints(n, dt=torch.float32, seed=n) for n in (4000, 70_001, 33)]
    out = [torch.zeros_like(g) for g in grads]
    once = ops.gradient_list(grads, out)
    ops.clip_gradients(once, 1.0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        norm = ops.clip_gradients(once, 1.0)
    once.close()
    guard = [torch.full((1 << 16,), 7, device="cuda", dtype=torch.int8) for _ in range(64)]
    others = [ops.gradient_list([torch.ones(50_000, device="cuda")]) for _ in range(8)]   # tables of their own
    for k in range(3):
        for i, g in enumerate(grads):
            g.copy_(ints(g.numel(), dt=torch.float32, seed=10 * k + i))
        graph.replay()
        exact = sum(float(g.double().square().sum()) for g in grads) ** 0.5
        assert abs(float(norm) - exact) <= exact * 2.0 ** -16
        for g, o in zip(grads, out):
            assert ((o.double() - g.double() / (exact + 1e-6)).abs() <= 2.0 ** -16 * g.double().abs() / exact).all()
    assert all(bool((g == 7).all()) for g in guard)
    for o in others:
        o.close()


def test_calls_that_wait_are_refused_in_a_capture(side):
    """Making or closing a list and waiting for the stream; the capture and the context go on."""
    ops, stream = side
    g = torch.ones(5000, device="cuda")
    once = ops.gradient_list([g.clone()])
    small = layer(30)
    step(ops, *small)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        plan = ops.dispatch(small[0], 5)
        for refused in (lambda: ops.gradient_list([g]), ops.synchronize):
            with pytest.raises(H.HwrError) as e:
                refused()
            assert e.value.status == UNSUPPORTED
        once.close()
        y = ops.adapter_forward(*small[1:5], small[6], plan)
    graph.replay()
    assert torch.equal(y, want(*small)[0])
    ops.synchronize()
    again = ops.gradient_list([g])
    assert abs(float(ops.clip_gradients(again, 1.0)) - 5000 ** 0.5) < 1e-3
    again.close()


def bounds(T, G, K, N, r, grads):
    """The header's bounds of the workspace."""
    P, S = T + 15 * min(T, G), K + N
    grouped = 16384 + 4 * G + 2 * P * (S + 18) + 2 * G * N * (K + 8)
    adapter = 16384 + 12 * G + 2 * P * (S + 18) + 12 * P * (r + 63) + 2 * N * (K + 8) + 6 * G * (r + 63) * (S + 16)
    clip = sum(-(-g.numel() * g.element_size() // 1024) * 8 + 32 for g in grads)
    return max(5 * (T // 4096 + 16) * (G + 1), grouped, adapter, clip)


PROGRAM = """
import sys
sys.path[:0] = [{tests!r}, {root!r}]
import torch
import paper_2608_14575_gb300 as H
from test_ops_capture_gpu import bounds
T, G, K, N, r, dt = {shape!r}
dt = getattr(torch, dt)
stream = torch.cuda.Stream()
with torch.cuda.stream(stream):
    c = (torch.arange(T, device="cuda", dtype=torch.int32) * 7) % (G + 1) - 1
    x, w, a, b, dy, gw = (torch.ones(s, device="cuda", dtype=dt) for s in
                          ((T, K), (N, K), (G, r, K), (G, N, r), (T, N), (G, N, K)))
    s = torch.ones(G, device="cuda")
    grads = [torch.ones(n, device="cuda") for n in (1, 5000, 3_000_001)]
    ops = H.Operators()
    ops.reserve(bounds(T, G, K, N, r, grads))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        plan = ops.dispatch(c, G)
        out = [ops.grouped_forward(x, gw, plan), *ops.grouped_backward(dy, x, gw, plan),
               ops.adapter_forward(x, w, a, b, s, plan), *ops.adapter_backward(dy, x, w, a, b, s, plan),
               ops.adapter_backward(dy, x, w, a, b, s, plan, need_dab=False)[0]]
        norm = ops.clip_gradients(grads, float("inf"))
    graph.replay()
    plan = ops.dispatch(c, G)
    now = [ops.grouped_forward(x, gw, plan), *ops.grouped_backward(dy, x, gw, plan),
           ops.adapter_forward(x, w, a, b, s, plan), *ops.adapter_backward(dy, x, w, a, b, s, plan),
           ops.adapter_backward(dy, x, w, a, b, s, plan, need_dab=False)[0]]
    assert all(torch.equal(p, q) for p, q in zip(out, now))
    assert abs(float(norm) - 3_005_002 ** 0.5) < 1e-2
print("captured")
"""


@pytest.mark.parametrize("shape", [(300, 7, 130, 65, 24, "bfloat16"), (40_000, 1000, 64, 72, 8, "float16"),
                                   (5, 64, 1000, 999, 100, "float16"), (2000, 3, 1, 1, 1, "bfloat16"),
                                   (70_000, 2, 33, 17, 256, "float16")])
def test_a_process_that_reserves_captures_at_once(shape):
    """A new process: with the header's bound reserved, its first calls are captured."""
    import os
    import subprocess
    import sys
    H.build()
    here = os.path.dirname(os.path.abspath(__file__))
    program = PROGRAM.format(tests=here, root=os.path.dirname(here), shape=shape)
    run = subprocess.run([sys.executable, "-c", program], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and run.stdout.strip().endswith("captured"), run.stderr[-2000:]


def test_other_contexts_come_and_go_beside_a_capture(side):
    """What a context that takes no part in a capture allocates and frees leaves it alone."""
    ops, stream = side
    small = layer(30)
    step(ops, *small)
    other = [H.Operators(torch.cuda.Stream()) for _ in range(2)]
    g = torch.ones(5000, device="cuda")
    lists = [o.gradient_list([g]) for o in other]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        held = step(ops, *small)
        lists[0].close()
        other[1].close()
        lists[1].close()
        new = H.Operators(torch.cuda.Stream())
    graph.replay()
    for got, exact in zip(held, want(*small)):
        assert torch.equal(got, exact)
    for o in (other[0], new):
        assert torch.equal(o.adapter_forward(*small[1:5], small[6], o.dispatch(small[0], 5)), want(*small)[0])
        o.close()
