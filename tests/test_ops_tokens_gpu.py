"""Log probabilities of tokens, entropies, alternatives and gradients against plain forms."""
import math

import pytest

torch = pytest.importorskip("torch")

import model_ref as M
import paper_2608_14575_gb300 as H
from ops_ref import inside
from test_ops_gpu import BF, HF

pytestmark = pytest.mark.gpu
F32 = torch.float32
INF = float("inf")


@pytest.fixture(scope="module")
def ops():
    H.build()
    return H.Operators()


def logits_of(T, V, dt, kind="any", seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + 13 * T + V)
    z = torch.empty(T, V, device="cuda").normal_(0, 3, generator=g)
    if kind == "masked":                 # most ruled out, in one row nearly all
        z = torch.where(torch.rand(T, V, device="cuda", generator=g) < 0.9, torch.full_like(z, -INF), z)
        z[0] = -INF
        z[0, V // 2] = 1.5
        z[-1, V - 1] = 0.0
    elif kind == "lowest":               # masked by the type's lowest value
        z = torch.where(torch.rand(T, V, device="cuda", generator=g) < 0.5,
                        torch.full_like(z, torch.finfo(dt).min), z)
        z[0] = torch.finfo(dt).min
    elif kind == "flat":
        z.fill_(0.25)
    elif kind == "ties":
        z = (z / 2).round()
        z = torch.where(z == 0, -z, z)
    elif kind == "rising":               # each step's maximum is a new one
        z = torch.linspace(-30, 30, V, device="cuda").expand(T, V).clone()
    elif kind == "large":
        z = z * 300 + 5000
    return z.to(dt)


def tokens_of(z, seed=0):
    T, V = z.shape
    g = torch.Generator(device="cuda").manual_seed(seed + T + V)
    token = torch.randint(0, V, (T,), device="cuda", dtype=torch.int32, generator=g)
    token = torch.where(torch.isinf(z.gather(1, token[:, None].long()))[:, 0], z.argmax(1).to(torch.int32), token)
    if T > 2:
        token[1], token[2] = -1, V
    return token


def best_of(z, top):
    """Stable: equal values in the order of their indices."""
    return torch.sort(z.double() + 0.0, dim=1, descending=True, stable=True).indices[:, :top]


SHAPES = [(1, 1), (1, 5), (3, 7), (2, 31), (5, 32), (4, 33), (7, 255), (3, 1000), (6, 1023), (1, 4099), (2, 8192), (400, 257),
          (1, 32_768), (9, 50_001), (1, 200_003), (700, 3001), (65, 20_000), (461, 20_001), (458, 30_001)]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dt", [F32, BF, HF])
@pytest.mark.parametrize("kind", ["any", "masked", "lowest", "flat", "ties", "rising", "large"])
def test_rows(ops, shape, dt, kind):
    T, V = shape
    z = logits_of(T, V, dt, kind)
    token = tokens_of(z)
    want = M.tokens(z, token)
    top = min(V, (1, 5, 20, 32)[(T + V) % 4])
    for n in (0, top):
        got = ops.token_logprobs(z, token, top=n)
        M.near(got.logprob, want["logprob"], "logprob")
        inside(got.entropy, want["entropy"], "entropy")
        assert torch.equal(got.stats[:, 0], z.float().amax(1))
        if n == 0:
            assert got.top_token is None and got.top_logprob is None
            continue
        best = best_of(z, n)
        assert torch.equal(got.top_token.long(), best)
        lq = want["logq"].gather(1, best)
        live = torch.isfinite(lq)
        assert torch.equal(got.top_logprob == -INF, lq == -INF)
        err = want["e_log"][:, None] + 2.0 ** -22 * (want["dist"].gather(1, best) + lq.abs().where(live, torch.zeros_like(lq)))
        assert ((got.top_logprob.double() - lq).abs() <= err)[live].all()


@pytest.mark.parametrize("shape", [(1, 1), (3, 7), (2, 33), (5, 1000), (1, 50_001), (300, 4097), (33, 8192)])
@pytest.mark.parametrize("dt", [F32, BF, HF])
@pytest.mark.parametrize("kind", ["any", "masked", "flat", "large"])
def test_gradient(ops, shape, dt, kind):
    T, V = shape
    z = logits_of(T, V, dt, kind)
    token = tokens_of(z)
    g = torch.Generator(device="cuda").manual_seed(V)
    a, b = (torch.empty(T, device="cuda").normal_(0, 1, generator=g) for _ in range(2))
    got = ops.token_logprobs(z, token)
    dz = ops.token_logprobs_backward(a, z, token, got, dentropy=b)
    assert dz.dtype == dt
    inside(dz, M.tokens_backward(z, token, a, b), "both")
    inside(ops.token_logprobs_backward(a, z, token, got), M.tokens_backward(z, token, a, b * 0), "logprob")
    inside(ops.token_logprobs_backward(None, z, token, got, dentropy=b), M.tokens_backward(z, token, a * 0, b), "entropy")
    # in the logits' place
    same = ops.token_logprobs_backward(a, z, token, got, dentropy=b, out=z)
    assert same is z and torch.equal(z, dz)


def test_gradient_against_differences(ops):
    """Central differences of the forward results: with h = 2^-3 the formula's third
    derivative (at most |a| + 8 |b|, q's moments below 1 and log q above -9 here) leaves
    h^2 / 6 of it, and fp32 sums near 10 leave 2^-20 / h."""
    V, h = 40, 2.0 ** -3
    g = torch.Generator(device="cuda").manual_seed(3)
    z = torch.empty(1, V, device="cuda").normal_(0, 1, generator=g)
    token = torch.tensor([7], device="cuda", dtype=torch.int32)
    a, b = torch.tensor([0.7], device="cuda"), torch.tensor([-0.4], device="cuda")
    dz = ops.token_logprobs_backward(a, z, token, ops.token_logprobs(z, token), dentropy=b)[0]
    rows = z.repeat(2 * V, 1)
    at = torch.arange(V, device="cuda")
    rows[at, at] += h
    rows[V + at, at] -= h
    got = ops.token_logprobs(rows, token.repeat(2 * V))
    f = a * got.logprob + b * got.entropy
    diff = (f[:V] - f[V:]) / (2 * h)
    assert (diff - dz).abs().max() <= h * h / 6 * (0.7 + 8 * 0.4) + 2.0 ** -20 / h


def test_rows_that_leave_nothing(ops):
    """All of a row masked: probabilities 0, entropy 0, no gradient; its neighbours as ever."""
    for dt in (F32, BF, HF):
        for V in (3, 100, 9000):
            z = logits_of(4, V, dt)
            z[1] = -INF
            token = torch.tensor([0, 1, 2, 0], device="cuda", dtype=torch.int32)
            got = ops.token_logprobs(z, token, top=3)
            assert got.logprob[1] == -INF and got.entropy[1] == 0
            assert got.top_token[1].tolist() == [0, 1, 2] and (got.top_logprob[1] == -INF).all()
            want = M.tokens(z[[0, 2, 3]], token[[0, 2, 3]])
            inside(got.logprob[[0, 2, 3]], want["logprob"])
            one = torch.ones(4, device="cuda")
            dz = ops.token_logprobs_backward(one, z, token, got, dentropy=one)
            assert (dz[1] == 0).all()
            inside(dz[[0, 2, 3]], M.tokens_backward(z[[0, 2, 3]], token[[0, 2, 3]], one[:3], one[:3]))


def test_masked_tokens(ops):
    """A token that is ruled out: log probability -inf; the gradient is the formula's."""
    z = logits_of(2, 300, F32)
    z[:, 5] = -INF
    token = torch.full((2,), 5, device="cuda", dtype=torch.int32)
    got = ops.token_logprobs(z, token)
    assert (got.logprob == -INF).all()
    one = torch.ones(2, device="cuda")
    inside(ops.token_logprobs_backward(one, z, token, got), M.tokens_backward(z, token, one, one * 0))


def test_nan_and_infinity(ops):
    """They make their own row's results NaN, and rank last (NaN) or first (+inf)."""
    for V in (40, 5000, 40_000):
        z = logits_of(5, V, BF)
        clean = ops.token_logprobs(z, None, top=4)
        z[1, V // 3], z[3, V - 1] = float("nan"), INF
        got = ops.token_logprobs(z, torch.zeros(5, device="cuda", dtype=torch.int32), top=4)
        for t in (1, 3):
            assert got.logprob[t].isnan() and got.entropy[t].isnan()
        assert got.top_token[3, 0] == V - 1
        assert V // 3 not in got.top_token[1].tolist()
        for t in (0, 2, 4):
            assert got.entropy[t] == clean.entropy[t] and torch.equal(got.top_token[t], clean.top_token[t])
    # nothing but NaN and a few numbers: the numbers first, then by index
    z = torch.full((1, 3000), float("nan"), device="cuda")
    z[0, 2000], z[0, 70] = 1.0, -2.0
    assert ops.token_logprobs(z, None, top=5).top_token[0].tolist() == [2000, 70, 0, 1, 2]


@pytest.mark.parametrize("dt", [F32, BF])
def test_strides(ops, dt):
    base = logits_of(9, 1500, dt)
    token = torch.arange(9, device="cuda", dtype=torch.int32) * 100
    a = torch.ones(9, device="cuda")
    for lo, hi in ((0, 1500), (1, 1499), (3, 1203), (8, 1000), (5, 12)):
        z = base[:, lo:hi]
        got = ops.token_logprobs(z, token, top=7)
        want = M.tokens(z, token)
        inside(got.logprob, want["logprob"])
        inside(got.entropy, want["entropy"])
        assert torch.equal(got.top_token.long(), best_of(z, 7))
        for shift in (lo, lo + 1):
            big = torch.full((9, 1600), 7.0, device="cuda", dtype=dt)
            out = big[:, shift:shift + hi - lo]
            ops.token_logprobs_backward(a, z, token, got, out=out)
            inside(out, M.tokens_backward(z, token, a, a * 0))
            out.fill_(7.0)
            assert (big == 7.0).all()


def test_no_rows_and_no_tokens(ops):
    z = logits_of(4, 100, BF)
    got = ops.token_logprobs(z)
    assert (got.logprob == 0).all()
    inside(got.entropy, M.tokens(z, torch.zeros(4, device="cuda", dtype=torch.int32))["entropy"])
    dz = ops.token_logprobs_backward(torch.ones(4, device="cuda"), z, None, got)
    assert (dz == 0).all()
    none = ops.token_logprobs(z[:0], top=3)
    assert none.logprob.shape == (0,) and none.top_token.shape == (0, 3)
    assert ops.token_logprobs_backward(None, z[:0], None, none).shape == (0, 100)


def test_offsets_beyond_32_bits(ops):
    """More than 2^31 logits: the last row's."""
    T, V = 16_500, 131_072
    z = torch.zeros(T, V, device="cuda", dtype=BF)
    z[-1, -1] = 20.0
    token = torch.full((T,), V - 1, device="cuda", dtype=torch.int32)
    got = ops.token_logprobs(z, token, top=2)
    total = math.exp(20.0) + V - 1
    # (512 additions of a thread, and joins: model_ref.serial)
    assert abs(float(got.logprob[-1]) - (20 - math.log(total))) <= M.serial(V) * M.U32 + 2.0 ** -20
    assert abs(float(got.logprob[0]) + math.log(V)) <= M.serial(V) * M.U32 + 2.0 ** -20 + 2.0 ** -21 * 12
    assert got.top_token[-1].tolist() == [V - 1, 0] and got.top_token[0].tolist() == [0, 1]
    dz = ops.token_logprobs_backward(torch.ones(T, device="cuda"), z, token, got, out=z)
    assert abs(float(dz[-1, -1]) - (V - 1) / total) <= 2.0 ** -7 * V / total + 2.0 ** -20
    assert float(dz[0, 0]) == pytest.approx(-1 / V, rel=2.0 ** -7)


def test_same_bits(ops):
    z = logits_of(3, 100_000, BF)
    token = tokens_of(z)
    first = ops.token_logprobs(z, token, top=9)
    for _ in range(20):
        again = ops.token_logprobs(z, token, top=9)
        for k in ("logprob", "entropy", "stats", "top_token", "top_logprob"):
            assert torch.equal(getattr(again, k), getattr(first, k))


def test_refusals(ops):
    z = logits_of(3, 50, BF)
    token = torch.zeros(3, device="cuda", dtype=torch.int32)
    got = ops.token_logprobs(z, token)
    one = torch.ones(3, device="cuda")
    for args in ((z.double(), token), (z.int(), token), (z, token.long()), (z, token[:2]), (z[0], token), (z.t(), token),
                 (z.cpu(), token), (z, token.cpu()), (z, token, -1), (z, token, 51)):
        with pytest.raises((TypeError, ValueError)):
            ops.token_logprobs(*args)
    with pytest.raises(H.HwrError) as e:
        ops.token_logprobs(z, token, 33)
    assert e.value.status == 7
    for args in ((one[:2], z, token, got), (one.double(), z, token, got), (one, z.float()[:2], token, got),
                 (one, z, token.long(), got)):
        with pytest.raises((TypeError, ValueError)):
            ops.token_logprobs_backward(*args)
    with pytest.raises((TypeError, ValueError)):
        ops.token_logprobs_backward(one, z, token, got, out=torch.empty(3, 50, device="cuda"))
    assert torch.equal(ops.token_logprobs(z, token).logprob, got.logprob)


@pytest.mark.parametrize("V", [1, 37, 3000, 200_003])
@pytest.mark.parametrize("dt", [F32, BF, HF])
def test_rows_of_nan_and_nothing_else(ops, V, dt):
    """Nothing but NaN, or NaN beside masked values (in one place of the row, whose pieces
    may have none): NaN as in any row, not the results of a row of -inf."""
    nan = float("nan")
    z = logits_of(6, V, dt)
    top = min(V, 5)
    clean = {n: ops.token_logprobs(z, None, top=n) for n in (0, top)}
    z[1] = nan
    z[2], z[3], z[4] = -INF, -INF, -INF
    z[2, 0], z[3, V // 2], z[4, V - 1] = nan, nan, nan
    token = torch.full((6,), V - 1, device="cuda", dtype=torch.int32)
    one = torch.ones(6, device="cuda")
    for n in (0, top):
        got = ops.token_logprobs(z, token, top=n)
        assert got.logprob[1:5].isnan().all() and got.entropy[1:5].isnan().all()
        for k in ("entropy", "stats"):
            assert torch.equal(getattr(got, k)[[0, 5]], getattr(clean[n], k)[[0, 5]])
        if n:
            assert got.top_logprob[1:5].isnan().all()
            assert got.top_token[1].tolist() == list(range(n))       # (by index, and the masked ones first)
            if V > 5:
                assert got.top_token[2].tolist() == list(range(1, n + 1))
                assert got.top_token[4].tolist() == list(range(n))
        for a, b in ((one, one), (one, None), (None, one)):
            dz = ops.token_logprobs_backward(a, z, token, got, dentropy=b)
            assert dz[1:5].isnan().all() and dz[[0, 5]].isfinite().all()


def test_the_longest_rows(ops):
    """2^31 - 1 logits, the most that a row can have: seven of them behind its last vector.
    All alike but for the last and one in the middle, q = e^{z - m} / S in closed form."""
    V = 2 ** 31 - 1
    z = torch.zeros(1, V, device="cuda", dtype=BF)
    z[0, V - 1], z[0, 1 << 30] = 24.0, 23.0
    token = torch.tensor([V - 1], device="cuda", dtype=torch.int32)
    log_s = math.log(1 + math.exp(-1) + (V - 2) * math.exp(-24))
    for top in (0, 4):
        got = ops.token_logprobs(z, token, top=top)
        # A thread's two sums count their ones exactly (fewer than 2^24).  Beside the 23 (a sum
        # of 1 for it) each e^-23 more may be lost whole: 2^31 / (32 * 128) / 2 of them.
        assert abs(float(got.logprob[0]) + log_s) <= 2.0 ** 18 * math.exp(-24) + 2.0 ** -19
        if top:
            assert got.top_token[0].tolist() == [V - 1, 1 << 30, 0, 1]
    dz = ops.token_logprobs_backward(torch.ones(1, device="cuda"), z, token, got, out=z)
    q = math.exp(float(got.logprob[0]))
    assert float(dz[0, V - 1]) == pytest.approx(1 - q, rel=2.0 ** -7)
    assert float(dz[0, 0]) == pytest.approx(-q * math.exp(-24), rel=2.0 ** -7)
    assert float(dz[0, V - 2]) == float(dz[0, 0])


@pytest.mark.parametrize("dt", [F32, BF, HF])
def test_large_gradients_at_masked_logits(ops, dt):
    """However large dentropy is, a logit of probability 0 has the gradient 0."""
    z = torch.full((2, 5000), -INF, device="cuda", dtype=dt)
    z[0, 7] = 1.0                                        # q = 1: log q + entropy = 0
    z[1, [3, 4000]] = 2.0
    got = ops.token_logprobs(z, None)
    for b in (1e9, -1e30, 3e38):
        dz = ops.token_logprobs_backward(None, z, None, got, dentropy=torch.full((2,), b, device="cuda"))
        assert (dz[z == -INF] == 0).all() and dz[0, 7] == 0


@pytest.mark.parametrize("dt", [F32, BF, HF])
def test_small_log_probabilities(ops, dt):
    """Nearly all of the probability on one logit, beside terms that are just too small to
    count next to it one by one (0.89 2^-24).  A row's sum near 1 is rounded (by 2^-24 at most)
    once a step of a block (4,096 logits, in 32 bits 2,048), four times within one, five between
    lanes, four between halves and warps and, here, never between pieces; exp within 2^-20."""
    T, V = 1300, 40_960
    z = torch.full((T, V), -16.75, device="cuda", dtype=dt)
    token = torch.arange(T, device="cuda", dtype=torch.int32) * 31 + 7
    z[torch.arange(T, device="cuda"), token.long()] = 0.0
    got = ops.token_logprobs(z, token)
    want = -math.log1p((V - 1) * math.exp(-16.75))
    steps = V // (2048 if dt == F32 else 4096)
    assert float((got.logprob.double() - want).abs().max()) <= (steps + 14) * 2.0 ** -24 + 2.0 ** -20 * abs(want)
    # With alternatives: blocks of twice the threads and warps, a rounding for every four logits of
    # a thread (two pairs), once for a pair.
    top = ops.token_logprobs(z, token, top=2)
    assert float((top.logprob.double() - want).abs().max()) <= (V // 1024 + 14) * 2.0 ** -24 + 2.0 ** -20 * abs(want)
