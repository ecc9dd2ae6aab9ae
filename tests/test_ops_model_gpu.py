"""The layer of experts, token log probabilities and AdamW as they are used: together, in
captured graphs, on other streams, at the edges of a context."""
import math

import pytest

torch = pytest.importorskip("torch")

import model_ref as M
import ops_ref as R
import paper_2608_14575_gb300 as H
from ops_ref import inside
from test_ops_gpu import BF, HF, choices, make

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


def training_set(T=300, G=5, K=136, V=1000, r=8):
    x, w = make(T, K), make(V, K, std=K ** -0.5, seed=1)
    a, b = make(G, r, K, std=K ** -0.5, seed=2), make(G, V, r, std=0.1, seed=3)
    c = choices(T, G, "holes")
    token = torch.randint(0, V, (T,), device="cuda", dtype=torch.int32, generator=torch.Generator(device="cuda").manual_seed(5))
    return x, w, a, b, torch.ones(G, device="cuda"), c, token


def train_step(ops, plan, x, w, a, b, s, token, state, scale):
    """Logits of adapters, their tokens' log probabilities, gradients, norm, optimizer."""
    z = ops.adapter_forward(x, w, a, b, s, plan)
    got = ops.token_logprobs(z, token)
    dz = ops.token_logprobs_backward(scale, z, token, got, out=z)
    _, da, db = ops.adapter_backward(dz, x, w, a, b, s, plan, need_dx=False)
    norm = ops.clip_gradients([da, db], float("inf"))
    ops.adamw_step(state, [da, db], lr=1e-2, norm=norm, max_norm=0.5, seed=2)
    return got, dz, da, db, norm


@pytest.mark.parametrize("bits", [32, 8])
def test_a_training_step(side, bits):
    """Each operator of the chain against the plain form of what it was given."""
    ops, _ = side
    x, w, a, b, s, c, token = training_set()
    plan = ops.dispatch(c, a.shape[0])
    master = [a.float(), b.float()]
    state = ops.adamw_state(master, bits=bits, copies=[a, b])
    scale = torch.full((x.shape[0],), -1.0 / x.shape[0], device="cuda")
    for t in (1, 2, 3):
        z = ops.adapter_forward(x, w, a, b, s, plan)
        old_a, old_b = a.clone(), b.clone()
        was = [m.clone() for m in master]
        moments = [[u.double() for u in state.moments(i)] for i in range(2)]
        got, dz, da, db, norm = train_step(ops, plan, x, w, a, b, s, token, state, scale)
        inside(got.logprob, M.tokens(z, token)["logprob"])
        inside(dz, M.tokens_backward(z, token, scale, scale * 0))
        _, wa, wb = R.adapter_backward(dz, x, w, old_a, old_b, s, c)
        inside(da, wa)
        inside(db, wb)
        exact = math.sqrt(float(da.double().square().sum() + db.double().square().sum()))
        assert abs(float(norm) - exact) <= 1e-6 * exact
        k = min(1.0, 0.5 / (float(norm) + 1e-6))
        for i, g in enumerate((da, db)):
            want = M.adamw(was[i], g, *moments[i], t, 1e-2, (0.9, 0.999), 1e-8, 0.01, k)
            inside(master[i], want["params"])
            assert torch.equal((a, b)[i], master[i].to(BF))
    state.close()


def decode(ops, x, w_in, w_out, scores, head):
    y = ops.expert_layer(x, w_in, w_out, scores=scores, top=2)
    plan = ops.dispatch(torch.zeros(x.shape[0], device="cuda", dtype=torch.int32), 1)
    z = ops.grouped_forward(y, head[None], plan)
    return y, z, ops.token_logprobs(z, top=4)


def decode_set(T=9, E=6, D=192, F=320, V=3000, dt=BF):
    g = torch.Generator(device="cuda").manual_seed(T)
    return (make(T, D, dt=dt), make(E, 2 * F, D, std=D ** -0.5, dt=dt, seed=1), make(E, D, F, std=F ** -0.5, dt=dt, seed=2),
            torch.empty(T, E, device="cuda").normal_(0, 1, generator=g), make(V, D, std=0.3, dt=dt, seed=3))


@pytest.mark.parametrize("dt", [BF, HF])
def test_a_decode_step(side, dt):
    ops, _ = side
    args = decode_set(dt=dt)
    y, z, got = decode(ops, *args)
    choice, p = M.choices(args[3], 2, False)
    inside(y, M.expert_layer(*args[:3], choice, p, "silu"))
    inside(got.entropy, M.tokens(z, torch.zeros(9, device="cuda", dtype=torch.int32))["entropy"])
    assert torch.equal(got.top_token.long(), torch.sort(z.double(), dim=1, descending=True, stable=True).indices[:, :4])


def test_captured(side):
    """Graphs of a decode and a training step, replayed on new inputs beside eager calls; a
    call of larger sizes in between takes a workspace of its own."""
    ops, stream = side
    args = decode_set()
    x, w, a, b, s, c, token = training_set()
    plan = ops.dispatch(c, a.shape[0])
    master = [a.float(), b.float()]
    state = ops.adamw_state(master, bits=8, copies=[a, b])
    twin_copies = [a.clone(), b.clone()]
    twin = ops.adamw_state([m.clone() for m in master], bits=8, copies=twin_copies)
    scale = torch.full((x.shape[0],), -1.0 / x.shape[0], device="cuda")
    # (calls of the same sizes first, on tensors of their own)
    decode(ops, *args)
    spare = [a.clone(), b.clone()]
    train_step(ops, plan, x, w, *spare, s, token, ops.adamw_state([u.float() for u in spare], bits=8, copies=spare), scale)
    torch.cuda.synchronize()
    serve, train = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(serve, stream=stream):
        y, z, got = decode(ops, *args)
    with torch.cuda.graph(train, stream=stream):
        held = train_step(ops, plan, x, w, a, b, s, token, state, scale)
    guard = [torch.full((1 << 20,), 7, device="cuda", dtype=torch.int8) for _ in range(60)]
    ops.expert_layer(*decode_set(T=100, E=9, D=512, F=2048)[:3], scores=torch.randn(100, 9, device="cuda"), top=5)
    for k in range(3):
        args[0].copy_(make(*args[0].shape, seed=10 + k))
        args[3].copy_(torch.empty_like(args[3]).normal_(0, 1, generator=torch.Generator(device="cuda").manual_seed(k)))
        x.copy_(make(*x.shape, seed=20 + k))
        serve.replay()
        train.replay()
        y2, z2, got2 = decode(ops, *args)
        assert torch.equal(y, y2) and torch.equal(z, z2)
        for name in ("entropy", "stats", "top_token", "top_logprob"):
            assert torch.equal(getattr(got, name), getattr(got2, name))
        again = train_step(ops, plan, x, w, *twin_copies, s, token, twin, scale)
        for p, q in zip(held[1:], again[1:]):
            assert torch.equal(p, q)
        assert torch.equal(held[0].logprob, again[0].logprob)
        for p, q in zip(state.params + state.copies, twin.params + twin.copies):
            assert torch.equal(p, q)
        assert int(state.step) == k + 1 == int(twin.step)
    assert all(bool((g == 7).all()) for g in guard)


def test_growing_in_a_capture_is_refused(side):
    """Nothing is queued, and the context and the capture go on."""
    ops, stream = side
    small, large = decode_set(), decode_set(T=100, D=512, F=4096)
    decode(ops, *small)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        with pytest.raises(H.HwrError) as e:
            ops.expert_layer(*large[:3], scores=large[3], top=6)
        assert e.value.status == UNSUPPORTED
        y, _, _ = decode(ops, *small)
    graph.replay()
    assert torch.equal(y, decode(ops, *small)[0])


@pytest.mark.parametrize("T,top,D,F,N", [(1, 1, 64, 64, 64), (128, 16, 72, 1000, 520), (7, 3, 300, 8192, 64), (128, 1, 64, 8192, 64), (128, 16, 64, 8193, 8)])
@pytest.mark.parametrize("dt", [BF, HF])
def test_workspace_bounds(T, top, D, F, N, dt):
    """With the header's bound reserved, a new context captures its first calls."""
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ops = H.Operators()
        x, w_in, w_out = make(T, D, dt=dt), make(20, F, D, dt=dt), make(20, N, F, dt=dt)
        scores = torch.randn(T, 20, device="cuda")
        z = make(T, 70_000, dt=dt)
        ops.reserve(max(4096 + 8 * T * top * (F + 9 + 8 * N), 2176 * torch.cuda.get_device_properties(0).multi_processor_count))
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            y = ops.expert_layer(x, w_in, w_out, scores=scores, top=top)
            got = ops.token_logprobs(z, top=5)
        graph.replay()
        assert torch.equal(y, ops.expert_layer(x, w_in, w_out, scores=scores, top=top))
        assert torch.equal(got.top_token, ops.token_logprobs(z, top=5).top_token)
        torch.cuda.synchronize()
        ops.close()


def test_another_current_stream():
    """Calls under another stream are ordered after its work, and it after them."""
    ops = H.Operators(torch.cuda.Stream())
    other = torch.cuda.Stream()
    args = decode_set()
    master = torch.zeros(5000, device="cuda")
    state = ops.adamw_state([master])
    want = ops.expert_layer(*args[:3], scores=args[3], top=2)
    torch.cuda.synchronize()
    with torch.cuda.stream(other):
        late = torch.zeros_like(args[0])
        grad = torch.zeros(5000, device="cuda")
        torch.cuda._sleep(100_000_000)
        late.copy_(args[0])
        grad.fill_(1.0)
        y = ops.expert_layer(late, *args[1:3], scores=args[3], top=2)
        ops.adamw_step(state, [grad], lr=1.0, weight_decay=0.0)
        y, moved = y.clone(), master.clone()
    other.synchronize()
    assert torch.equal(y, want) and bool((moved + 1).abs().max() <= 2.0 ** -18)
    ops.close()


def test_two_contexts_at_once():
    """Two contexts on streams of their own do not disturb each other."""
    pair = [H.Operators(torch.cuda.Stream()) for _ in range(2)]
    sets = [decode_set(T=16, E=8, D=512, F=1024), decode_set(T=64, E=8, D=256, F=704, dt=HF)]
    z = [make(4, 100_000, seed=k) for k in range(2)]
    want = [(ops.expert_layer(*s[:3], scores=s[3], top=3), ops.token_logprobs(v, top=8)) for ops, s, v in zip(pair, sets, z)]
    torch.cuda.synchronize()
    got = []
    for _ in range(30):
        for ops, s, v in zip(pair, sets, z):
            with torch.cuda.stream(ops.stream):
                got.append((ops.expert_layer(*s[:3], scores=s[3], top=3), ops.token_logprobs(v, top=8)))
    torch.cuda.synchronize()
    for i, (y, t) in enumerate(got):
        assert torch.equal(y, want[i % 2][0])
        assert torch.equal(t.top_logprob, want[i % 2][1].top_logprob) and torch.equal(t.entropy, want[i % 2][1].entropy)
    for ops in pair:
        ops.close()


def test_another_current_device(monkeypatch):
    """Refused before anything is launched.  (The test hook makes the current device seem
    another one.)"""
    monkeypatch.setenv("HWR_TEST_DEVICE", "1")
    off = H.Operators()
    monkeypatch.delenv("HWR_TEST_DEVICE")
    args = decode_set()
    for call in (lambda: off.expert_layer(*args[:3], scores=args[3], top=2), lambda: off.token_logprobs(args[4]),
                 lambda: off.adamw_state([torch.zeros(9, device="cuda")])):
        with pytest.raises(H.HwrError) as e:
            call()
        assert e.value.status == 1 and "device 1 is current" in str(e.value)
    off.close()


def test_timeout(monkeypatch):
    """Copies that never come (the test hook): the waits run out, the failure is reported, the
    context is broken, and a new one works."""
    args = decode_set()
    monkeypatch.setenv("HWR_TEST_STALL", "1")
    bad = H.Operators()
    monkeypatch.delenv("HWR_TEST_STALL")
    bad.expert_layer(*args[:3], scores=args[3], top=2)
    with pytest.raises(H.HwrError) as e:
        bad.synchronize()
    assert e.value.status == 5
    with pytest.raises(H.HwrError) as e:
        bad.token_logprobs(args[4])
    assert e.value.status == 6
    bad.close()
    good = H.Operators()
    choice, p = M.choices(args[3], 2, False)
    inside(good.expert_layer(*args[:3], scores=args[3], top=2), M.expert_layer(*args[:3], choice, p, "silu"))
    good.close()


def test_optimizers_go_with_their_context():
    """A state that outlives its closed context leaves no device memory behind."""
    p = [torch.zeros(1 << 28, device="cuda")]                  # (a table of 1 MB)
    m, v = [torch.zeros_like(p[0])], [torch.zeros_like(p[0])]

    def cycle():
        ops = H.Operators()
        one, two = (ops.adamw_state(p, m=m, v=v) for _ in range(2))
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
    assert before - torch.cuda.mem_get_info()[0] < 8 << 20


@pytest.mark.parametrize("bits", [32, 8])
def test_example_runs(bits):
    """The example trains adapters on answer tokens and decodes through experts."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "token_training.py")
    spec = importlib.util.spec_from_file_location("token_training", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    means, adapters, tokens = example.main(rows=200, width=64, vocab=300, groups=3, rank=4, steps=2, bits=bits, say=lambda *_: None)
    assert len(means) == 2 and all(math.isfinite(m) and m < 0 for m in means)
    assert all(a.isfinite().all() for a in adapters) and bool((adapters[1] != 0).any())
    assert tokens.shape == (4,) and bool((tokens >= 0).all()) and bool((tokens < 300).all())
