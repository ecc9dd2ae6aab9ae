"""Plain 64-bit restatements of the layer of experts, the token log probabilities and
the AdamW step, and the error each output may have, for the tests."""
import math

import torch

from ops_ref import ADD, FLOOR, UNIT, inside

# fp32's rounding, relative; expf, erff, logf, expm1f and the divisions are within 4 units
# of the last place (2^-21), the fast ones within 2^-20.
U32 = 2.0 ** -24
FUNC = 2.0 ** -20


# ---- a layer of experts --------------------------------------------------------

def choices(scores, top, over_all):
    """(choice, p): the largest scores, ties to the lowest index; -1 where none is left."""
    T, E = scores.shape
    choice = torch.full((T, top), -1, dtype=torch.int32)
    p = torch.zeros(T, top, dtype=torch.float64)
    s = scores.double().cpu()
    for t in range(T):
        row = s[t].tolist()
        able = [e for e in range(E) if row[e] > -math.inf]
        best = sorted(able, key=lambda e: (-row[e], e))[:top]
        if not best:
            continue
        m = row[best[0]]
        total = math.fsum(math.exp(row[e] - m) for e in (able if over_all else best))
        for j, e in enumerate(best):
            choice[t, j] = e
            p[t, j] = math.exp(row[e] - m) / total
    return choice.to(scores.device), p.to(scores.device)


def act(u, name):
    if name == "relu":
        return torch.relu(u)
    if name == "silu":
        return u * torch.sigmoid(u)
    return u * torch.special.ndtr(u)


def expert_layer(x, w_in, w_out, choice, p, name):
    """(y, error bound)"""
    T, (E, N, F), dt = x.shape[0], w_out.shape, x.dtype
    gated = w_in.shape[1] == 2 * F
    term = 2.0 ** -15 if dt == torch.bfloat16 else 2.0 ** -20
    y = torch.zeros(T, N, dtype=torch.float64, device=x.device)
    err = torch.zeros_like(y)
    xx = x.double()
    for e in range(E):
        t, j = torch.nonzero(choice == e, as_tuple=True)
        if not t.numel():
            continue
        W, V = w_in[e].double(), w_out[e].double()
        u, mags = xx[t] @ W.T, xx[t].abs() @ W.abs().T
        eu = (x.shape[1] + 64) * ADD * mags
        g = act(u[:, :F], name)
        # (the activations' slopes are at most 1.13)
        eg = 1.13 * eu[:, :F] + FUNC * (g.abs() + eu[:, :F])
        h, eh = g, eg
        if gated:
            h = g * u[:, F:]
            eh = eg * (u[:, F:].abs() + eu[:, F:]) + g.abs() * eu[:, F:] + U32 * h.abs()
        eh = eh + term * (h.abs() + eh) + FLOOR[torch.bfloat16]
        w = p[t, j].double()[:, None]
        out = h @ V.T
        eo = eh @ V.abs().T + (F + 64) * ADD * ((h.abs() + eh) @ V.abs().T)
        y.index_put_((t,), w * out, accumulate=True)
        err.index_put_((t,), w.abs() * (eo + (2.0 ** -18) * out.abs()), accumulate=True)
    return y, UNIT[dt] * (y.abs() + err) + err + FLOOR[dt]


# ---- log probabilities ---------------------------------------------------------

def serial(V):
    """Additions of a thread, and the joins above them."""
    return V / 256 + 64 + 32 + 64


def tokens(logits, token):
    """{name: (value, error)} for logprob, entropy; and logq [rows][vocab]"""
    z = logits.double()
    # (a row of -inf alone: probabilities 0, log probabilities -inf)
    empty = (z == -math.inf).all(1, keepdim=True)
    logq = torch.where(empty, z, torch.log_softmax(torch.where(empty, torch.zeros_like(z), z), 1))
    q = torch.exp(logq)
    m = torch.where(empty, torch.zeros_like(z[:, :1]), z.amax(1, keepdim=True))
    d = torch.where(q > 0, m - z, torch.zeros_like(z))              # distance from the largest
    H = torch.special.entr(q).sum(1)
    mean, square = (q * d).sum(1), (q * d * d).sum(1)
    # of each exp: the function, and the distance's and its product's rounding
    ulps = serial(z.shape[1]) * U32 + FUNC
    e_sum = ulps + 2.0 ** -22 * mean
    log_s = torch.where(empty[:, 0], torch.zeros_like(H), torch.logsumexp(z - m, 1))
    e_log = e_sum + 2.0 ** -21 * log_s.abs() + 2.0 ** -23
    eH = e_log + mean * (ulps + e_sum + 2.0 ** -21) + 2.0 ** -22 * square + U32 * H
    has = (token >= 0) & (token < z.shape[1])
    at = torch.where(has, token, torch.zeros_like(token)).long()[:, None]
    lp = logq.gather(1, at)[:, 0]
    dist = d.gather(1, at)[:, 0]
    e_lp = e_log + 2.0 ** -22 * (dist + lp.abs())
    zero = torch.zeros_like(lp)
    return {"logprob": (torch.where(has, lp, zero), torch.where(has, e_lp, zero)), "entropy": (H, eH),
            "logq": logq, "e_log": e_log, "dist": d}


def near(got, want, name=""):
    """As ops_ref.inside, infinities equal."""
    exact, err = want
    live = torch.isfinite(exact)
    assert torch.equal(got.double()[~live], exact[~live]), name
    inside(got[live], (exact[live], err[live]), name)


def tokens_backward(logits, token, a, b):
    """(dlogits, error bound)"""
    r = tokens(logits, token)
    logq, (H, eH) = r["logq"], r["entropy"]
    q = torch.exp(logq)
    has = (token >= 0) & (token < q.shape[1]) & (q.sum(1) > 0)
    a = (a.double() * has)[:, None]
    b = b.double()[:, None]
    inner = torch.where(q > 0, logq + H[:, None], torch.zeros_like(q))
    g = -q * (a + b * inner)
    at = torch.where(has, token, torch.zeros_like(token)).long()[:, None]
    g.scatter_add_(1, at, a)
    e_lq = r["e_log"][:, None] + 2.0 ** -22 * (r["dist"] + torch.where(q > 0, logq.abs(), torch.zeros_like(q)))
    # (an exp below fp32's smallest normal number, 2^-126, counts as 0: off by less than that)
    e_q = 2.0 ** -126 + q * (e_lq + FUNC + 2.0 ** -23 * torch.where(q > 0, logq.abs(), torch.zeros_like(q)))
    err = (e_q + q * 2.0 ** -22) * (a.abs() + b.abs() * inner.abs()) + q * b.abs() * (e_lq + eH[:, None])
    err = err + 2.0 ** -22 * a.abs() * torch.zeros_like(q).scatter_(1, at, 1.0)
    unit, floor = (U32, 2.0 ** -126) if logits.dtype == torch.float32 else (UNIT[logits.dtype], FLOOR[logits.dtype])
    return g, unit * (g.abs() + err) + err + floor


# ---- AdamW ---------------------------------------------------------------------

def adamw(p, g, m, v, t, lr, betas, eps, decay, k=1.0):
    """{name: (value, error)} of params, m, v after step t, from 64-bit m, v; k: the clip factor"""
    b1, b2 = betas
    g = g.double() * k
    m1, v1 = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    em = 8 * U32 * (b1 * m.abs() + (1 - b1) * g.abs()) + 2.0 ** -126
    ev = 12 * U32 * (b2 * v + (1 - b2) * g * g) + 2.0 ** -126
    c1, c2 = 1 - b1 ** t, 1 - b2 ** t
    den = (v1 / c2).sqrt() + eps
    step = m1 / c1 / den
    w = p.double()
    new = w - lr * (decay * w + step)
    # (a root of v with a small error: half of the relative one, or all of it near 0)
    e_den = (((v1 + ev) / c2).sqrt() - (v1 / c2).sqrt()) + 8 * U32 * den
    e_step = em / c1 / (den - e_den) + step.abs() * (e_den / (den - e_den) + 8 * FUNC)
    e_new = lr * (e_step + 4 * U32 * decay * w.abs() + 4 * U32 * step.abs()) + 2 * U32 * (new.abs() + lr * step.abs()) + 2.0 ** -126
    return {"params": (new, e_new), "m": (m1, em), "v": (v1, ev)}


MASK = 0xffffffff


def mixed(x):
    x = ((x ^ (x >> 16)) * 0x7feb352d) & MASK
    x = ((x ^ (x >> 15)) * 0x68e31da5) & MASK
    return x ^ (x >> 16)


def random_bits(n, number, t, seed, device, first=0):
    """The 32 random bits of n elements of tensor `number` at step t."""
    key = mixed((mixed((t + seed * 0x9e3779b1) & MASK) + (number + 1) * 0x85157af5) & MASK)
    return mixed(((torch.arange(first, first + n, device=device) & MASK) * 0x9e3779b1 + key) & MASK)


def to_blocks(x, bits, least):
    """fp32 x as e4m3 values and powers of two of its blocks of 256, rounded by 16 random bits."""
    n = x.numel()
    pad = -n % 256
    b = torch.nn.functional.pad(x.reshape(-1), (0, pad)).view(-1, 256)
    r = torch.nn.functional.pad(bits, (0, pad)).view(-1, 256)
    field = (b.abs().amax(1).view(torch.int32) >> 23)
    scale = (field - 7).clamp(min=1) << 23
    inverse = ((254 << 23) - scale).view(torch.float32)
    tiny = b.abs() * inverse[:, None] * 2.0 ** -120
    code = (tiny.view(torch.int32).long() + ((r << 4) | 8)) >> 20
    if least:
        code = torch.where((b > 0) & (code == 0), torch.ones_like(code), code)
    code = code | ((b.view(torch.int32) >> 24) & 0x80)
    return code.to(torch.uint8).view(torch.float8_e4m3fn).view(-1)[:n], scale.view(torch.float32)


def from_blocks(values, scale):
    x = values.float().reshape(-1)
    return x * scale.repeat_interleave(256)[:x.numel()]
