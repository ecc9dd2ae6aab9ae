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
