"""The AdamW step against a plain 64-bit form, and its 8-bit moments bit for bit."""
import math

import pytest

torch = pytest.importorskip("torch")

import model_ref as M
import paper_2608_14575_gb300 as H
from ops_ref import inside
from test_ops_gpu import BF, HF

pytestmark = pytest.mark.gpu
F32 = torch.float32
ARGS = dict(lr=1e-2, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.1)


@pytest.fixture(scope="module")
def ops():
    H.build()
    return H.Operators()


def normal(n, std=1.0, dt=F32, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + 31 * n)
    return torch.empty(n, device="cuda", dtype=dt).normal_(0, std, generator=g)


SIZES = [[1], [8], [2048], [2049], [0, 5, 0], [255, 256, 257], [70_001, 3, 4096, 2047], list(range(1, 300)), [1_000_003]]


@pytest.mark.parametrize("sizes", SIZES)
@pytest.mark.parametrize("gt", [F32, BF, HF])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("copy", [None, BF, HF])
def test_steps(ops, sizes, gt, bits, copy):
    """Three steps from zero moments, each against the formula from the state before it;
    8-bit moments bit for bit."""
    params = [normal(n, seed=1) for n in sizes]
    copies = None if copy is None else [torch.zeros(n, device="cuda", dtype=copy) for n in sizes]
    state = ops.adamw_state(params, bits=bits, copies=copies)
    for t in (1, 2, 3):
        grads = [normal(n, 0.3, gt, seed=10 * t) for n in sizes]
        norm = torch.tensor(7.5, device="cuda")
        max_norm = (float("inf"), 2.5, 100.0)[t - 1]
        k = min(1.0, max_norm / (7.5 + 1e-6))
        before = [p.clone() for p in params]
        old = [[u.clone() for u in state.moments(i)] for i in range(len(sizes))]
        ops.adamw_step(state, grads, norm=norm, max_norm=max_norm, seed=9, **ARGS)
        assert int(state.step) == t
        for i, n in enumerate(sizes):
            if n == 0 or (len(sizes) > 50 and i % 23):
                continue
            want = M.adamw(before[i], grads[i], old[i][0].double(), old[i][1].double(), t, ARGS["lr"], ARGS["betas"],
                           ARGS["eps"], ARGS["weight_decay"], k)
            inside(params[i], want["params"], (i, "params"))
            if copy is not None:
                assert torch.equal(copies[i], params[i].to(copy))
            if bits == 32:
                inside(state.m[i], want["m"], (i, "m"))
                inside(state.v[i], want["v"], (i, "v"))
                continue
            # the same single fp32 operations
            b1, b2 = ARGS["betas"]
            one = torch.tensor(1.0, device="cuda")
            f = grads[i].float() * (torch.full_like(one, max_norm) / (norm + 1e-6)).clamp(max=1.0)
            m = old[i][0] * b1 + f * (1 - b1)
            r = torch.sqrt(old[i][1] * b2 + (f * f) * (1 - b2))
            bits_of = M.random_bits(n, i, t, 9, "cuda")
            for got, scale, x, rnd, least in ((state.m[i], state.m_scale[i], m, bits_of & 0xffff, False),
                                              (state.v[i], state.v_scale[i], r, bits_of >> 16, True)):
                values, scales = M.to_blocks(x, rnd, least)
                assert torch.equal(scale, scales)
                assert torch.equal(got.view(torch.uint8).view(-1), values.view(torch.uint8))
    state.close()


def test_a_late_step_and_small_betas(ops):
    for betas, done in (((0.9, 0.999), 123_456), ((0.0, 0.0), 0), ((0.95, 0.98), 7)):
        p, g = normal(5000), normal(5000, 0.1, seed=2)
        m, v = normal(5000, 0.01, seed=3), normal(5000, 0.1, seed=4).square()
        before = [u.clone() for u in (p, m, v)]
        step = torch.full((1,), done, device="cuda", dtype=torch.int32)
        state = ops.adamw_state([p], m=[m], v=[v], step=step)
        lr = torch.tensor(3e-4, device="cuda")
        ops.adamw_step(state, [g], lr=lr, betas=betas, weight_decay=0.0)
        want = M.adamw(before[0], g, before[1].double(), before[2].double(), done + 1, 3e-4, betas, 1e-8, 0.0)
        inside(p, want["params"])
        inside(m, want["m"])
        inside(v, want["v"])
        assert int(step) == done + 1 and state.step is step


def test_missing_gradients(ops):
    """A parameter without a gradient, its moments and its copy stay as they are."""
    sizes = [3000, 5000, 17]
    for bits in (32, 8):
        params = [normal(n) for n in sizes]
        copies = [p.to(BF) for p in params]
        state = ops.adamw_state(params, bits=bits, copies=[copies[0], None, copies[2]])
        grads = [normal(n, seed=4) for n in sizes]
        ops.adamw_step(state, grads, lr=0.1)
        held = [t.clone() for t in (params[1], state.m[1].view(torch.uint8), state.v[1].view(torch.uint8))]
        other = params[0].clone()
        ops.adamw_step(state, [grads[0], None, grads[2]], lr=0.1)
        for a, b in zip(held, (params[1], state.m[1].view(torch.uint8), state.v[1].view(torch.uint8))):
            assert torch.equal(a, b)
        assert not torch.equal(other, params[0]) and int(state.step) == 2
        ops.adamw_step(state, [None] * 3, lr=0.1)
        assert int(state.step) == 3


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_steps_without_a_finite_norm_are_left_out(ops, bits, bad):
    p, g = normal(4000), normal(4000, dt=BF, seed=1)
    state = ops.adamw_state([p], bits=bits)
    ops.adamw_step(state, [g], lr=0.1, seed=3)
    g[77] = bad
    norm = ops.clip_gradients([g], float("inf"))
    held = [t.clone() for t in (p, state.m[0].view(torch.uint8), state.v[0].view(torch.uint8))]
    ops.adamw_step(state, [g], lr=0.1, norm=norm, max_norm=1.0, seed=3)
    for a, b in zip(held, (p, state.m[0].view(torch.uint8), state.v[0].view(torch.uint8))):
        assert torch.equal(a, b)
    assert int(state.step) == 1
    # without the norm a NaN stays with its element, or with its block of 8-bit moments
    ops.adamw_step(state, [g], lr=0.1, seed=3)
    m = state.moments(0)[0]
    assert m[77].isnan() or m[77].isinf() or bits == 8 and m[77].isnan()
    lo, hi = (77, 78) if bits == 32 else (0, 256)
    rest = torch.cat([m[:lo], m[hi:]])
    assert rest.isfinite().all() and torch.cat([p[:77], p[78:]]).isfinite().all()


def test_rounding_keeps_the_expectation(ops):
    """A constant gradient over 1,500 steps: v goes to g^2 (nearest rounding would hold it
    near a sixtieth of that), sqrt(v) of each of 65,536 elements by steps of up to 1/8 of
    it at random.  Mean of sqrt(v)^2: the steps' variance per step is at most the drift
    0.001 / 2 times 1/8 of the value, relative, over 1,000 steps of memory: 0.2^2 at most; v's
    mean exceeds the mean of its root squared by as much, 4 %, and the mean over the elements
    varies by 0.4 / 256."""
    n, g0 = 65_536, 0.01
    p = torch.zeros(n, device="cuda")
    state = ops.adamw_state([p], bits=8)
    g = torch.full((n,), g0, device="cuda")
    for _ in range(1500):
        ops.adamw_step(state, [g], lr=0.0, seed=1)
    m, v = state.moments(0)
    want = g0 * g0 * (1 - 0.999 ** 1500)
    assert abs(float(m.double().mean()) / g0 - 1) <= 0.01
    assert 0.9 * want <= float(v.double().mean()) <= 1.1 * want
    assert abs(float(v.sqrt().double().mean()) / math.sqrt(want) - 1) <= 0.06


def test_quiet_elements(ops):
    """Beside an element 10^9 times larger a moment's root rounds up, never to 0, so that no
    update is larger than a few learning rates."""
    p = torch.zeros(256, device="cuda")
    g = torch.full((256,), 1e-9, device="cuda")
    g[0] = 1.0
    state = ops.adamw_state([p], bits=8)
    for _ in range(20):
        ops.adamw_step(state, [g], lr=1.0, weight_decay=0.0, eps=0.0)
        assert (state.v[0].float() > 0).all()
    assert p.isfinite().all() and p.abs().max() <= 20 * 2.0


@pytest.mark.parametrize("bits", [32, 8])
def test_alignment_does_not_matter(ops, bits):
    """Tensors that begin anywhere give the bits of aligned ones."""
    n = 10_007
    kind = torch.float8_e4m3fn if bits == 8 else F32
    out = []
    for off in (0, 1, 3):
        def at(dt):
            return torch.zeros(n + 8, device="cuda", dtype=dt)[off:off + n]
        p, c, g, m, v = at(F32), at(BF), at(HF), at(kind), at(kind)
        p.copy_(normal(n))
        g.copy_(normal(n, seed=2))
        state = ops.adamw_state([p], bits=bits, copies=[c], m=[m], v=[v])
        for _ in range(3):
            ops.adamw_step(state, [g], lr=0.1, seed=5)
        out.append([t.clone().view(torch.uint8) for t in (p, c, m, v)])
    for other in out[1:]:
        for a, b in zip(out[0], other):
            assert torch.equal(a, b)


def test_neighbours_are_left_alone(ops):
    """Nothing beside the tensors is written."""
    for bits in (32, 8):
        kind = torch.float8_e4m3fn if bits == 8 else F32
        for n in (1, 7, 300, 2047, 4100):
            big = [torch.ones(n + 32, device="cuda", dtype=dt) for dt in (F32, BF, kind, kind)]
            p, c, m, v = (t[16:16 + n] for t in big)
            blocks = -(-n // 256)
            scales = [torch.ones(blocks + 2, device="cuda") for _ in range(2)]
            state = ops.adamw_state([p], bits=bits, copies=[c], m=[m], v=[v], m_scale=[scales[0][1:-1]] if bits == 8 else None,
                                    v_scale=[scales[1][1:-1]] if bits == 8 else None)
            ops.adamw_step(state, [normal(n)], lr=0.1)
            for t in big:
                assert (t[:16].float() == 1).all() and (t[16 + n:].float() == 1).all()
            for t in scales:
                assert t[0] == 1 and t[-1] == 1


def test_more_than_2_31_elements(ops):
    n = (1 << 31) + 4099
    p = torch.zeros(n, device="cuda")
    g = torch.zeros(n, device="cuda", dtype=BF)
    at = torch.tensor([0, 4095, (1 << 31) - 1, 1 << 31, n - 1], device="cuda")
    g[at] = 3.0
    state = ops.adamw_state([p], bits=8)
    ops.adamw_step(state, [g], lr=0.5, weight_decay=0.0)
    # the first step moves by the learning rate: 3 c1 / c1 / (3 + eps), a few roundings
    assert ((p[at] + 0.5).abs() <= 0.5 * 2.0 ** -18).all()
    assert int((p != 0).sum()) == 5 and int((state.v[0].view(torch.uint8) != 0).sum()) == 5


def test_captured_steps_count(ops):
    """Replays go on counting, on a gradient whose values change in place."""
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        own = H.Operators()
        p, g = normal(5000), normal(5000, dt=BF, seed=1)
        eager = p.clone()
        state, twin = own.adamw_state([p], bits=8), own.adamw_state([eager], bits=8)
        norm = torch.tensor(3.0, device="cuda")
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            own.adamw_step(state, [g], norm=norm, max_norm=2.0, seed=4, **ARGS)
            with pytest.raises(H.HwrError) as e:
                own.adamw_state([p.clone()], m=[p], v=[p], step=state.step)
            assert e.value.status == 7
        for k in range(4):
            g.copy_(normal(5000, seed=20 + k))
            graph.replay()
            own.adamw_step(twin, [g], norm=norm, max_norm=2.0, seed=4, **ARGS)
            assert torch.equal(p, eager) and int(state.step) == k + 1
        state.close()                      # the graph keeps its table
        g.copy_(normal(5000, seed=40))
        graph.replay()
        own.adamw_step(twin, [g], norm=norm, max_norm=2.0, seed=4, **ARGS)
        assert torch.equal(p, eager)
        torch.cuda.synchronize()
        own.close()


def test_lifetimes(ops):
    """A state outlives its closed context without harm, and is refused by others."""
    other = H.Operators()
    p = normal(100)
    state = other.adamw_state([p])
    with pytest.raises(ValueError):
        ops.adamw_step(state, [p], lr=0.1)
    other.close()
    with pytest.raises(RuntimeError):
        other.adamw_step(state, [p], lr=0.1)
    state.close()
    state.close()
    mine = ops.adamw_state([p])
    mine.close()
    with pytest.raises(ValueError):
        ops.adamw_step(mine, [p], lr=0.1)


def test_written_tensors_count_as_modified(ops):
    p, c = normal(100), torch.zeros(100, device="cuda", dtype=BF)
    state = ops.adamw_state([p], copies=[c])
    was = [t._version for t in (p, c, state.m[0], state.v[0], state.step)]
    ops.adamw_step(state, [normal(100)], lr=0.1)
    assert all(t._version > w for t, w in zip((p, c, state.m[0], state.v[0], state.step), was))


def test_refusals(ops):
    p, g = normal(300), normal(300)
    for args, kw in ((([p.half()],), {}), (([p.cpu()],), {}), (([p[::2]],), {}), (([p],), dict(bits=16)),
                     (([p],), dict(copies=[p])), (([p],), dict(copies=[p[:9].half()])), (([p],), dict(copies=[])),
                     (([p],), dict(m=[g.half()])), (([p],), dict(bits=8, m=[g])), (([p],), dict(step=torch.zeros(1, device="cuda"))),
                     (([p],), dict(bits=8, m_scale=[torch.ones(3, device="cuda")]))):
        with pytest.raises((TypeError, ValueError)):
            ops.adamw_state(*args, **kw)
    state = ops.adamw_state([p])
    held = p.clone()
    for grads, kw in (([], {}), ([g, g], {}), ([g.double()], {}), ([g[:200]], {}), ([g.cpu()], {}), ([normal(600)[::2]], {}),
                      ([g], dict(lr=torch.zeros(2, device="cuda"))), ([g], dict(lr=torch.zeros(1, device="cuda").double())),
                      ([g], dict(norm=torch.ones(1)))):
        with pytest.raises((TypeError, ValueError)):
            ops.adamw_step(state, grads, **dict(dict(lr=0.1), **kw))
    nan = float("nan")
    for kw in (dict(lr=-1.0), dict(lr=nan), dict(betas=(1.0, 0.9)), dict(betas=(0.9, -0.1)), dict(eps=-1.0), dict(weight_decay=nan),
               dict(norm=torch.ones(1, device="cuda"), max_norm=0.0), dict(norm=torch.ones(1, device="cuda"), max_norm=nan)):
        with pytest.raises(H.HwrError) as e:
            ops.adamw_step(state, [g], **dict(dict(lr=0.1), **kw))
        assert e.value.status == 1
    assert torch.equal(p, held) and int(state.step) == 0
    ops.adamw_step(state, [g], lr=0.1)
    assert int(state.step) == 1


@pytest.mark.parametrize("bits", [32, 8])
def test_every_thread_reads_the_same_step_number(ops, bits):
    """Early steps, whose corrections differ most from one to the next, over a few blocks that
    end at different times (some have little to do, some no gradient): the same start gives
    the same bits, again and again, and the number goes up by one."""
    sizes = [2048, 1, 2047, 300, 2048 * 3 + 5]
    start = [normal(n, seed=1) for n in sizes]
    grads = [normal(n, seed=2) for n in sizes]
    grads[3] = None
    params = [p.clone() for p in start]
    state = ops.adamw_state(params, bits=bits)
    written = params + [t.view(torch.uint8) for t in state.m + state.v]
    held = [t.clone() for t in written]
    first = None
    for _ in range(300):
        for t, h in zip(written, held):
            t.copy_(h)
        state.step.zero_()
        for n in (1, 2):
            ops.adamw_step(state, grads, lr=0.1, seed=4)
        got = [t.clone() for t in written] + [state.step.clone()]
        first = first or got
        assert all(torch.equal(a, b) for a, b in zip(got, first))
    assert int(state.step) == 2


def test_gradients_of_another_shape(ops):
    """A gradient has its parameter's shape: one with as many elements (a transposed one that
    was made contiguous) is refused, and nothing changes."""
    p = normal(600).view(20, 30)
    state = ops.adamw_state([p])
    before = p.clone()
    g = normal(600, seed=1).view(20, 30)
    for bad in (g.t().contiguous(), g.view(-1), g.view(1, 20, 30)):
        with pytest.raises(ValueError):
            ops.adamw_step(state, [bad], lr=0.1)
    assert torch.equal(p, before) and int(state.step) == 0
    ops.adamw_step(state, [g], lr=0.1)
    assert int(state.step) == 1 and not torch.equal(p, before)


def test_an_optimizer_of_another_context_is_refused(ops):
    """By the C entry too, whose contexts have streams and counters of their own."""
    other = H.Operators()
    p = normal(3000)
    state = ops.adamw_state([p])
    before = p.clone()
    with pytest.raises(H.HwrError) as e:
        other.native.adamw_step(other.ctx, other._current(), state.handle, [normal(3000, seed=1)], 0.1, 0.9, 0.999, 1e-8,
                                0.0, None, math.inf, 0)
    assert e.value.status == 1
    assert torch.equal(p, before) and int(state.step) == 0
    other.adamw_step(other.adamw_state([p]), [normal(3000, seed=1)], lr=0.1)      # (it stays usable)
    assert not torch.equal(p, before)
    other.close()


def test_a_launch_that_fails(ops, monkeypatch):
    """Of a step's several launches (over 256 tensors each): the first one's failure leaves
    everything as it is and the context usable; a later one's, when some tensors have made the
    step, breaks the context whatever the error, and other contexts do not notice."""
    params = [normal(40, seed=i) for i in range(300)]
    grads = [normal(40, seed=i + 1000) for i in range(300)]
    for failing in (1, 2):
        monkeypatch.setenv("HWR_TEST_FAIL_LAUNCH", str(failing))
        own = H.Operators()
        monkeypatch.delenv("HWR_TEST_FAIL_LAUNCH")
        before = [p.clone() for p in params]
        state = own.adamw_state(params)
        with pytest.raises(H.HwrError) as e:
            own.adamw_step(state, grads, lr=0.1)
        assert e.value.status == (3 if failing == 1 else 4)          # out of memory, or CUDA
        assert int(state.step) == 0
        if failing == 1:
            assert all(torch.equal(a, b) for a, b in zip(params, before))
            own.adamw_step(state, grads, lr=0.1)
            assert int(state.step) == 1 and not torch.equal(params[-1], before[-1])
        else:
            with pytest.raises(H.HwrError) as e:
                own.adamw_step(state, grads, lr=0.1)
            assert e.value.status == 6                               # unusable
            own.close()
    state = ops.adamw_state(params)
    ops.adamw_step(state, grads, lr=0.1)
    assert int(state.step) == 1


@pytest.mark.parametrize("bits", [32, 8])
def test_tensors_that_overlap_are_refused(ops, bits):
    """What a step writes lies nowhere twice: the same parameter two times, parts of one, a
    moment in another's place (two blocks would write it, in any order)."""
    p, q = normal(3000), normal(3000, seed=1)
    for params in ([p, q, p], [p, p[2999:]], [p[:2000], p[1999:]]):
        with pytest.raises(H.HwrError) as e:
            ops.adamw_state(params, bits=bits)
        assert e.value.status == 1
    m = [torch.zeros(3000, device="cuda", dtype=torch.float8_e4m3fn if bits == 8 else F32) for _ in range(2)]
    for args in (dict(m=[m[0], m[0]]), dict(m=m, v=[m[1], m[0]]), dict(copies=[q.to(BF)] * 2)):
        with pytest.raises(H.HwrError):
            ops.adamw_state([p, q], bits=bits, **args)
    # side by side, and empty ones anywhere, are fine
    state = ops.adamw_state([p[:1500], p[1500:], q, p[700:700]], bits=bits)
    ops.adamw_step(state, [normal(n, seed=2) for n in (1500, 1500, 3000, 0)], lr=0.1)
    assert int(state.step) == 1
