"""A layer of experts for a few rows against a plain 64-bit form."""
import pytest

torch = pytest.importorskip("torch")

import model_ref as M
import paper_2608_14575_gb300 as H
from ops_ref import inside
from test_ops_gpu import BF, HF, ints, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    H.build()
    return H.Operators()


def scores_of(T, E, kind="any", seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + 17 * T + E)
    s = torch.empty(T, E, device="cuda").normal_(0, 1, generator=g)
    if kind == "ties":
        s = (s * 2).round()
        s = torch.where(s == 0, -s, s)              # (zeros of either sign are equal)
    elif kind == "masked":
        s = torch.where(s < 0.3, torch.full_like(s, float("-inf")), s)
        s[0] = float("-inf")
    elif kind == "one":
        s[:, E // 2] += 100
    return s


def layer(T, E, D, F, N, gated, dt, seed=0):
    return (make(T, D, dt=dt, seed=seed), make(E, 2 * F if gated else F, D, std=D ** -0.5, dt=dt, seed=seed + 1),
            make(E, N, F, std=F ** -0.5, dt=dt, seed=seed + 2))


SHAPES = [   # T, E, top, D, F, N
    (1, 1, 1, 8, 8, 8), (1, 12, 2, 256, 512, 256), (2, 5, 3, 64, 72, 40), (3, 4, 4, 33, 35, 17), (1, 3, 1, 1, 1, 1),
    (8, 64, 6, 128, 176, 128), (9, 7, 2, 1000, 520, 136), (16, 16, 2, 512, 1024, 512), (17, 1024, 16, 64, 32, 24),
    (33, 2, 2, 264, 136, 264), (64, 64, 2, 256, 264, 200), (128, 40, 16, 72, 48, 72), (128, 1, 1, 128, 256, 128),
    (100, 3, 1, 101, 257, 99), (4, 8, 2, 4104, 40, 1000), (5, 8, 2, 40, 4104, 33), (7, 12, 1, 1001, 1365, 1001),    # experts of more than 8 rows on average, one to several steps of both products
    (24, 2, 2, 2056, 1544, 1100), (20, 1, 1, 1030, 2054, 513), (40, 3, 2, 1088, 4104, 72), (17, 1, 1, 520, 640, 24),
    (50, 5, 2, 192, 1088, 264),
]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("gated", [True, False])
def test_layer(ops, shape, dt, gated):
    T, E, top, D, F, N = shape
    x, w_in, w_out = layer(T, E, D, F, N, gated, dt)
    for kind, over_all, name in (("any", False, "silu"), ("masked", True, "gelu"), ("one", True, "relu"), ("ties", False, "silu")):
        s = scores_of(T, E, kind)
        y = ops.expert_layer(x, w_in, w_out, scores=s, top=top, over_all=over_all, activation=name)
        choice, p = M.choices(s, top, over_all)
        inside(y, M.expert_layer(x, w_in, w_out, choice, p, name), (kind, name))


@pytest.mark.parametrize("shape", [(1, 4, 1, 64, 64, 64), (6, 3, 2, 200, 100, 72), (70, 5, 3, 65, 33, 31), (128, 2, 16, 64, 64, 64)])
@pytest.mark.parametrize("dt", [BF, HF])
def test_given_choices(ops, shape, dt):
    """Choices of the caller's: none, outside the groups, the same one twice; any gates."""
    T, E, top, D, F, N = shape
    x, w_in, w_out = layer(T, E, D, F, N, True, dt)
    g = torch.Generator(device="cuda").manual_seed(T)
    choice = torch.randint(-1, E + 1, (T, top), device="cuda", dtype=torch.int32, generator=g)
    choice[-1] = E - 1                                   # all the same
    if T > 1:
        choice[0] = -5                                   # none
    gates = torch.empty(T, top, device="cuda").normal_(0, 1, generator=g)
    y = ops.expert_layer(x, w_in, w_out, choice=choice, gates=gates)
    inside(y, M.expert_layer(x, w_in, w_out, choice, gates, "silu"))
    if T > 1:
        assert (y[0] == 0).all()


def test_exact_on_whole_numbers(ops):
    """ReLU layers on small whole numbers: one rounding is all that may differ."""
    for dt in (BF, HF):
        for T, E, top, D, F, N in ((3, 4, 2, 64, 64, 48), (50, 6, 1, 130, 70, 33)):
            x, w_in, w_out = ints(T, D, dt=dt, lo=-1, hi=1), ints(E, F, D, dt=dt, lo=-1, hi=1), ints(E, N, F, dt=dt, lo=-1, hi=1)
            choice = torch.arange(T * top, device="cuda", dtype=torch.int32).view(T, top) % E
            gates = torch.full((T, top), 0.5, device="cuda")
            y = ops.expert_layer(x, w_in, w_out, choice=choice, gates=gates, activation="relu")
            want, _ = M.expert_layer(x, w_in, w_out, choice, gates, "relu")
            assert torch.equal(y, want.to(dt))


def test_no_choice_at_all(ops):
    x, w_in, w_out = layer(5, 3, 64, 40, 56, True, BF)
    out = torch.full((5, 56), 7.0, device="cuda", dtype=BF)
    y = ops.expert_layer(x, w_in, w_out, scores=torch.full((5, 3), float("-inf"), device="cuda"), top=2, out=out)
    assert y is out and (out == 0).all()
    y = ops.expert_layer(x, w_in, w_out, choice=torch.full((5, 1), -1, device="cuda", dtype=torch.int32),
                         gates=torch.ones(5, 1, device="cuda"))
    assert (y == 0).all()
    assert ops.expert_layer(x[:0], w_in, w_out, scores=torch.zeros(0, 3, device="cuda"), top=1).shape == (0, 56)


@pytest.mark.parametrize("dt", [BF, HF])
def test_rows_and_experts_keep_apart(ops, dt):
    """NaN and infinities of a row reach that row alone, those of an expert its rows alone."""
    T, E, D, F, N = 20, 5, 72, 56, 40
    x, w_in, w_out = layer(T, E, D, F, N, True, dt)
    choice = (torch.arange(T, device="cuda", dtype=torch.int32) % E)[:, None]
    gates = torch.ones(T, 1, device="cuda")
    want = ops.expert_layer(x, w_in, w_out, choice=choice, gates=gates)
    x[7], x[11, 3] = float("nan"), float("inf")
    w_in[1, 5], w_out[2, :, 4] = float("nan"), float("inf")
    y = ops.expert_layer(x, w_in, w_out, choice=choice, gates=gates)
    keep = torch.tensor([t for t in range(T) if t not in (7, 11) and t % E not in (1, 2)], device="cuda")
    assert torch.equal(y[keep], want[keep])
    assert y[7].isnan().all() and y[1].isnan().all()
    two = torch.tensor([t for t in range(T) if t % E == 2 and t not in (7, 11)], device="cuda")
    assert y[two].isinf().all()               # an infinite weight, not NaN


@pytest.mark.parametrize("dt", [BF, HF])
@pytest.mark.parametrize("size", [2.0 ** -12, 2.0 ** 7])
def test_hidden_values_of_any_size(ops, dt, size):
    """Hidden values far below and above fp16's range keep their bits."""
    T, E, D, F, N = 6, 2, 64, 64, 64
    x, w_in, w_out = layer(T, E, D, F, N, True, dt)
    x, w_out = x * size, (w_out / size / size).clamp(-60000, 60000) if size > 1 else w_out
    w_in = w_in * (8 if size > 1 else 1)
    s = scores_of(T, E)
    y = ops.expert_layer(x, w_in, w_out, scores=s, top=2)
    choice, p = M.choices(s, 2, False)
    inside(y, M.expert_layer(x, w_in, w_out, choice, p, "silu"))


@pytest.mark.parametrize("off", [0, 1, 3])
def test_strides(ops, off):
    """Rows, weights and results inside larger tensors, aligned and not."""
    T, E, D, F, N = 11, 4, 120, 88, 104
    base = [make(T, D + 24, seed=1), make(E, 2 * F + 3, D + 16, std=0.1, seed=2), make(E, N + 2, F + 8, std=0.1, seed=3)]
    x = base[0][:, off:off + D]
    w_in, w_out = base[1][:, 1:2 * F + 1, off:off + D], base[2][:, 2:, off:off + F]
    s = scores_of(T, E + 3)[:, 1:E + 1]
    big = torch.full((T + 2, N + 9), 3.0, device="cuda", dtype=BF)
    out = big[1:T + 1, off:off + N]
    ops.expert_layer(x, w_in, w_out, scores=s, top=2, out=out)
    choice, p = M.choices(s, 2, False)
    inside(out, M.expert_layer(x, w_in, w_out, choice, p, "silu"))
    out.fill_(3.0)
    assert (big == 3.0).all()                 # nothing beside the result was written


@pytest.mark.parametrize("shape", [(3, 4, 2, 1000, 1100, 72), (3, 4, 2, 1001, 1098, 40), (20, 2, 2, 1096, 523, 24),
                                   (5, 3, 1, 40, 61, 8), (9, 3, 2, 576, 1089, 1000)])
@pytest.mark.parametrize("dt", [BF, HF])
def test_rows_that_end_before_their_stride(ops, shape, dt):
    """Widths of any remainder on aligned rows: what lies behind them (NaN) is not part of them."""
    T, E, top, D, F, N = shape
    whole = lambda n: (n + 7) // 8 * 8 + 8
    padded = []
    for t in layer(T, E, D, F, N, True, dt):
        big = torch.full((*t.shape[:-1], whole(t.shape[-1])), float("nan"), device="cuda", dtype=dt)
        big[..., :t.shape[-1]] = t
        padded.append(big[..., :t.shape[-1]])
    x, w_in, w_out = padded
    s = scores_of(T, E)
    y = ops.expert_layer(x, w_in, w_out, scores=s, top=top)
    choice, p = M.choices(s, top, False)
    inside(y, M.expert_layer(x, w_in, w_out, choice, p, "silu"))


def test_offsets_beyond_32_bits(ops):
    """Weights of more than 2^31 elements: the last expert's."""
    D, F, E = 4096, 4096, 140
    w_in = torch.zeros(E, F, D, device="cuda", dtype=BF)
    w_out = torch.zeros(E, 64, F, device="cuda", dtype=BF)
    w_in[-1], w_out[-1] = ints(F, D, lo=-1, hi=1), ints(64, F, lo=-1, hi=1)
    x = ints(2, D, lo=-1, hi=1)
    choice = torch.tensor([[E - 1], [0]], device="cuda", dtype=torch.int32)
    gates = torch.ones(2, 1, device="cuda")
    y = ops.expert_layer(x, w_in, w_out, choice=choice, gates=gates, activation="relu")
    inside(y[:1], M.expert_layer(x[:1], w_in[-1:], w_out[-1:], choice[:1] * 0, gates[:1], "relu"))
    assert (y[1] == 0).all()


def test_same_bits(ops):
    x, w_in, w_out = layer(64, 16, 512, 264, 200, True, BF)
    s = scores_of(64, 16)
    first = ops.expert_layer(x, w_in, w_out, scores=s, top=4)
    for _ in range(20):
        assert torch.equal(ops.expert_layer(x, w_in, w_out, scores=s, top=4), first)


def test_refusals(ops):
    x, w_in, w_out = layer(5, 3, 64, 40, 56, True, BF)
    s = scores_of(5, 3)
    c, g = torch.zeros(5, 2, device="cuda", dtype=torch.int32), torch.ones(5, 2, device="cuda")
    good = dict(scores=s, top=2)
    for error, args in (
            (ValueError, dict(good, activation="tanh")), (ValueError, dict(good, top=0)), (ValueError, dict(good, top=4)),
            (ValueError, dict(good, choice=c, gates=g)), (TypeError, dict(choice=c)), (TypeError, dict(gates=g)), (TypeError, {}),
            (TypeError, dict(choice=c.long(), gates=g)), (TypeError, dict(choice=c, gates=g.double())),
            (ValueError, dict(choice=c, gates=g[:, :1])), (TypeError, dict(good, scores=s.double())),
            (ValueError, dict(good, scores=s[:, :2])), (ValueError, dict(good, scores=s.cpu())),
            (ValueError, dict(good, out=torch.empty(5, 55, device="cuda", dtype=BF))),
            (TypeError, dict(good, out=torch.empty(5, 56, device="cuda")))):
        with pytest.raises(error):
            ops.expert_layer(x, w_in, w_out, **args)
    for bad in ((x.float(), w_in, w_out), (x, w_in.half(), w_out), (x, w_in[:, :70], w_out), (x[:, :60], w_in, w_out),
                (x, w_in[0], w_out), (x, w_in, w_out[:2]), (x, w_in.transpose(1, 2), w_out), (x.cpu(), w_in, w_out)):
        with pytest.raises((TypeError, ValueError)):
            ops.expert_layer(*bad, **good)
    for T, E, top in ((129, 3, 1), (5, 1025, 1), (5, 20, 17)):
        w = torch.zeros(E, 16, 8, device="cuda", dtype=BF), torch.zeros(E, 8, 8, device="cuda", dtype=BF)
        with pytest.raises(H.HwrError) as e:
            ops.expert_layer(torch.zeros(T, 8, device="cuda", dtype=BF), *w, scores=scores_of(T, E), top=top)
        assert e.value.status == 7
    choice, p = M.choices(s, 2, False)
    inside(ops.expert_layer(x, w_in, w_out, **good), M.expert_layer(x, w_in, w_out, choice, p, "silu"))


@pytest.mark.parametrize("dt", [BF, HF])
def test_gelu_of_negative_values(ops, dt):
    """u Phi(u) keeps its relative accuracy far below 0: one whole or half number u a row (its
    product with 1 is exact), gates (powers of two) that bring the results near 1.  The
    argument's two roundings (2^-24 each) move erfc(-u / sqrt 2) by u^2 2^-23 of it at most
    (its logarithm's slope is below u^2 + 1 in u's relative change); erfcf is within 4 units
    of the last place, two products round once each; and the hidden value's terms."""
    u = -torch.arange(1, 25, device="cuda", dtype=torch.float64) / 2
    T = u.numel()
    x = torch.zeros(T, 8, device="cuda", dtype=dt)
    x[:, 0] = u
    w_in, w_out = torch.zeros(1, 16, 8, device="cuda", dtype=dt), torch.zeros(1, 8, 16, device="cuda", dtype=dt)
    w_in[0, 3, 0] = w_out[0, :, 3] = 1
    want = u * torch.special.erfc(-u * 2 ** -0.5) / 2
    gates = torch.exp2(-torch.floor(torch.log2(want.abs())))[:, None].float()
    y = ops.expert_layer(x, w_in, w_out, choice=torch.zeros(T, 1, device="cuda", dtype=torch.int32), gates=gates,
                         activation="gelu").double()
    want = (want * gates[:, 0].double())[:, None]
    term, unit = (2.0 ** -15, 2.0 ** -8) if dt == BF else (2.0 ** -20, 2.0 ** -11)
    rel = (u * u + 1) * 2.0 ** -23 + 16 * 2.0 ** -23 + term
    assert ((y - want).abs() <= want.abs() * (rel[:, None] + unit * (1 + rel[:, None]))).all()


@pytest.mark.parametrize("E", [5, 40, 300])
def test_nan_scores(ops, E):
    """A NaN is never chosen.  Among the chosen scores there is none; a softmax over all of a
    row's scores (over_all) has one in its sum, and the row is NaN."""
    T, D, F, N, top = 6, 64, 48, 40, 2
    x, w_in, w_out = layer(T, E, D, F, N, True, BF)
    s = scores_of(T, E)
    bad = s.clone()
    bad[1, E - 1], bad[3, 0], bad[4] = float("nan"), float("nan"), float("nan")
    bad[3, 1] = float("-inf")
    masked = torch.where(bad.isnan(), torch.full_like(bad, float("-inf")), bad)
    y = ops.expert_layer(x, w_in, w_out, scores=bad, top=top)
    assert torch.equal(y, ops.expert_layer(x, w_in, w_out, scores=masked, top=top)) and (y[4] == 0).all()
    y = ops.expert_layer(x, w_in, w_out, scores=bad, top=top, over_all=True)
    assert y[1].isnan().all() and y[3].isnan().all() and (y[4] == 0).all()      # (4: no choice)
    keep = torch.tensor([0, 2, 5], device="cuda")
    assert torch.equal(y[keep], ops.expert_layer(x, w_in, w_out, scores=masked, top=top, over_all=True)[keep])


@pytest.mark.parametrize("T,F", [(3, 16), (8, 33), (64, 16), (64, 33)])
def test_hidden_values_keep_24_bits(ops, T, F):
    """Two hidden values of a bf16 layer that agree in 16 bits, taken apart: h = x1 + x2 + x3 and
    x1 + x2, with x1 in [1/2, 1), x2 below 2^-8 and x3 below 2^-16, eight bits each.  Their
    difference is x3, off by 2^-22 of at most 1 for each of 11 additions (model: ops_ref.ADD);
    values of 16 bits would lose up to 2^-17."""
    def bits(lowest):
        g = torch.Generator(device="cuda").manual_seed(T + lowest)
        return torch.randint(128, 256, (T,), device="cuda", generator=g).double() * 2.0 ** lowest
    parts = [bits(-8), bits(-16), bits(-24)]
    x = torch.zeros(T, 8, device="cuda", dtype=BF)
    w_in, w_out = torch.zeros(1, F, 8, device="cuda", dtype=BF), torch.zeros(1, 24, F, device="cuda", dtype=BF)
    for i, part in enumerate(parts):
        x[:, i] = part
        assert torch.equal(x[:, i].double(), part)
    w_in[0, 0, :3] = w_in[0, F - 1, :2] = 1
    w_out[0, :, 0], w_out[0, :, F - 1] = 1, -1
    y = ops.expert_layer(x, w_in, w_out, choice=torch.zeros(T, 1, device="cuda", dtype=torch.int32),
                         gates=torch.ones(T, 1, device="cuda"), activation="relu").double()
    assert ((y - parts[2][:, None]).abs() <= 11 * 2.0 ** -22 + 2.0 ** -8 * parts[2][:, None]).all()
