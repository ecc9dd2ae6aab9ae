"""A served and a trained model's other operators, as measurable cases.

What surrounds the products of routed rows: the layer of experts that a decode
step runs for its few tokens, the probabilities that its answer is given with
and trained on, and the optimizer's step on what the backward passes leave.

  experts    y[t] = sum over j of p[t, j] W_out[e] h[t, j], e the j-th choice of
             row t, h = act(W_gate[e] x[t]) * (W_up[e] x[t]) or act(W_in[e] x[t]).
             The choices are the ``top`` largest of scores [T][E] (ties to the
             lowest index) with p the softmax over those or over all scores, or
             are given: one choice per row (-1 where it has none) and its p;
  tokens     of logits z [T][V] and a token per row (-1 where it has none):
             logprob = z[token] - lse (0 without a token), entropy of softmax(z),
             and the ``top`` most probable tokens with their log probabilities;
             train: the gradient of sum a[t] logprob[t] + b[t] entropy[t] too,
             dz[v] = a (1[v = token] - q[v]) - b q[v] (log q[v] + entropy);
  adamw      one step over many tensors, g the gradients times
             min(1, max_norm / (norm + 1e-6)):
             m' = b1 m + (1 - b1) g,  v' = b2 v + (1 - b2) g^2,
             w' = w - lr (decay w + (m' / (1 - b1^t)) / (sqrt(v' / (1 - b2^t)) + eps)).
             Moments in 32 bits, or m and sqrt(v) in 8: e4m3 values with a power
             of two for each 256 elements, rounded up or down by a hash of seed,
             step, tensor and element (the expectation is the value, so that
             small changes are not lost); sqrt(v) > 0 stays above 0.

Weights are w_in [E][2 F or F][D] (gate rows first) and w_out [E][N][F].
"""
from __future__ import annotations

import math

import torch

own = False

DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "f32": torch.float32}
EPS = 1e-6
BLOCK = 256             # elements that share a power of two

# The most that a drawn case costs (that of the listed ones or less).
MOST_WEIGHTS = 800_000_000
MOST_LOGITS = 1 << 28
MOST_PARAMS = 113_000_000

# A late step of a long run: moments that gradients of the same size have left.
HYPER = dict(lr=1e-3, b1=0.9, b2=0.999, eps=1e-8, decay=0.1)


def listed():
    return [
        # One token of one request: two of 12 experts, all of it latency and weights.
        dict(name="experts_token", op="experts", rows=1, groups=12, top=2, n_in=1024, hidden=4096,
             n_out=1024, gated=True, act="silu", over_all=False, given=False, dtype="bf16"),
        # The router's own decisions carried out for a few queries: one expert each,
        # none for some, plain layers of odd widths.
        dict(name="experts_chosen", op="experts", rows=7, groups=12, top=1, n_in=1001, hidden=2731,
             n_out=1001, gated=False, act="gelu", over_all=False, given=True, dtype="bf16"),
        # A decode step of 16 requests with many small experts.
        dict(name="experts_step", op="experts", rows=16, groups=64, top=6, n_in=2048, hidden=1408,
             n_out=2048, gated=True, act="silu", over_all=True, given=False, dtype="bf16"),
        # A decode step of a micro-batch in half precision: nearly every expert is read.
        dict(name="experts_batch", op="experts", rows=64, groups=64, top=2, n_in=1024, hidden=4096,
             n_out=1024, gated=True, act="silu", over_all=False, given=False, dtype="fp16"),
        # One sampled token with its five best alternatives.
        dict(name="tokens_one", op="tokens", train=False, rows=1, vocab=32_768, top=5, dtype="f32"),
        # A decode step of a micro-batch: the answer's tokens with 20 alternatives each.
        dict(name="tokens_step", op="tokens", train=False, rows=64, vocab=131_072, top=20, dtype="bf16"),
        # Scoring given answers: log probabilities and entropies of a few thousand tokens.
        dict(name="tokens_score", op="tokens", train=False, rows=4099, vocab=50_001, top=0, dtype="bf16"),
        # The loss of a training step and its gradient.
        dict(name="tokens_train", op="tokens", train=True, rows=4096, vocab=32_768, top=0, dtype="bf16"),
        # A set of adapters: many small tensors, 16-bit gradients and copies.
        dict(name="adamw_adapters", op="adamw", tensors=48, largest=65_536, bits=32, grads="bf16", copies="bf16"),
        # The same with moments in 8 bits, and half precision.
        dict(name="adamw_adapters8", op="adamw", tensors=48, largest=65_536, bits=8, grads="fp16", copies="fp16"),
        # Whole layers, everything in 32 bits.
        dict(name="adamw_layers", op="adamw", tensors=16, largest=16_777_216, bits=32, grads="f32", copies="none"),
        # Whole layers, moments in 8 bits.
        dict(name="adamw_layers8", op="adamw", tensors=16, largest=16_777_216, bits=8, grads="bf16", copies="bf16"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    w = _log(rng, lo, hi)
    return w if rng.random() < 0.25 else max(8, w // 8 * 8)   # mostly whole 16-byte rows


def draw(rng):
    op = rng.choice(("experts", "tokens", "adamw"))
    if op == "experts":
        case = dict(op=op, rows=_log(rng, 1, 64), groups=_log(rng, 1, 128), n_in=_width(rng, 64, 4096),
                    hidden=_width(rng, 64, 8192), gated=rng.random() < 0.7, act=rng.choice(("silu", "gelu", "relu")),
                    over_all=rng.random() < 0.5, given=rng.random() < 0.25, dtype=rng.choice(("bf16", "fp16")))
        case["n_out"] = case["n_in"]
        case["groups"] = max(1, min(case["groups"], MOST_WEIGHTS // (3 * case["n_in"] * case["hidden"])))
        case["top"] = 1 if case["given"] else min(case["groups"], rng.randint(1, 8))
        return case
    if op == "tokens":
        case = dict(op=op, train=rng.random() < 0.4, rows=_log(rng, 1, 8192), vocab=_width(rng, 100, 200_000),
                    dtype=rng.choice(("bf16", "fp16", "f32")))
        case["rows"] = max(1, min(case["rows"], MOST_LOGITS // (2 * case["vocab"] if case["train"] else case["vocab"])))
        case["top"] = 0 if case["train"] else rng.choice((0, 1, 5, 20, 32))
        return case
    n, most = _log(rng, 1, 60), _log(rng, 1000, 1 << 24)
    return dict(op=op, tensors=n, largest=min(most, MOST_PARAMS // n), bits=rng.choice((8, 32)),
                grads=rng.choice(("bf16", "fp16", "f32")), copies=rng.choice(("bf16", "fp16", "none")))


# ---- inputs -------------------------------------------------------------------

def sizes_of(case):
    """Elements of each tensor: matrices, halves and quarters of them, biases, odd ones."""
    big = case["largest"]
    return [max(1, (big, big // 2, big // 4 + 1, big // 64)[i % 4] - (i % 3)) for i in range(case["tensors"])]


def starts_of(sizes):
    """Where each tensor begins in the flat buffers, and their length."""
    at = [0]
    for n in sizes:
        at.append(at[-1] + -(-n // BLOCK) * BLOCK)
    return at


def in_blocks(x):
    """(e4m3 values, the blocks' powers of two) nearest to x, whose length is whole blocks."""
    b = x.view(-1, BLOCK)
    _, e = torch.frexp(b.abs().amax(1))
    scale = torch.ldexp(torch.ones_like(b[:, 0]), (e - 8).clamp(min=-126))     # the largest in [2^7, 2^8)
    return (b / scale[:, None]).to(torch.float8_e4m3fn).view(-1), scale


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)

    def normal(*shape, std=1.0, dtype=torch.float32):
        return torch.empty(shape, device=dev, dtype=dtype).normal_(0.0, std, generator=gen)

    s = dict(case=case, op=case["op"])
    if case["op"] == "experts":
        T, E, D, F, N = (case[k] for k in ("rows", "groups", "n_in", "hidden", "n_out"))
        dt = DT[case["dtype"]]
        s["x"] = normal(T, D, dtype=dt)
        s["w_in"] = normal(E, 2 * F if case["gated"] else F, D, std=D ** -0.5, dtype=dt)
        s["w_out"] = normal(E, N, F, std=F ** -0.5, dtype=dt)
        if case["given"]:
            choice = torch.randint(0, E, (T, 1), device=dev, dtype=torch.int32, generator=gen)
            none = torch.rand(T, 1, device=dev, generator=gen) < 0.05
            none[0] = False
            s["choice"] = torch.where(none, torch.full_like(choice, -1), choice)
            s["gates"] = 0.5 + 0.5 * torch.rand(T, 1, device=dev, generator=gen)
        else:
            s["scores"] = normal(T, E) + normal(E, std=0.5)
        return s
    if case["op"] == "tokens":
        T, V = case["rows"], case["vocab"]
        # a model's logits: most of the mass on a few tokens; some of them ruled out
        s["logits"] = normal(T, V, std=2.0, dtype=DT[case["dtype"]])
        best = torch.randint(0, V, (T, 8), device=dev, generator=gen)
        s["logits"].scatter_add_(1, best, normal(T, 8, std=3.0).abs().add_(6.0).to(s["logits"].dtype))
        s["logits"][:, torch.randint(0, V, (max(1, V // 100),), device=dev, generator=gen)] = -math.inf
        token = best[:, 0].to(torch.int32)
        token = torch.where(torch.rand(T, device=dev, generator=gen) < 0.8, token,
                            torch.randint(0, V, (T,), device=dev, dtype=torch.int32, generator=gen))
        # (none that is ruled out, and some rows without one)
        ruled = torch.isinf(s["logits"].gather(1, token[:, None].long()))[:, 0]
        if T > 1:
            ruled |= torch.rand(T, device=dev, generator=gen) < 0.02
        s["token"] = torch.where(ruled, torch.full_like(token, -1), token)
        if case["train"]:
            s["a"] = normal(T) / T
            s["b"] = normal(T).abs() * 0.01 / T
        return s

    sizes = sizes_of(case)
    at = starts_of(sizes)
    flat = {k: torch.zeros(at[-1], device=dev) for k in ("params", "grads", "m", "r")}
    for i, n in enumerate(sizes):
        p, g, m, r = (flat[k][at[i]:at[i] + n] for k in ("params", "grads", "m", "r"))
        std = 0.01 * (1 + i % 5)
        p.normal_(0.0, 0.02, generator=gen)
        g.normal_(0.0, std, generator=gen)
        m.normal_(0.0, 0.23 * std, generator=gen)
        r.normal_(std, 0.05 * std, generator=gen).abs_()
    s["params"] = flat["params"]
    s["grads"] = flat["grads"].to(DT[case["grads"]])
    if case["copies"] != "none":
        s["copies"] = flat["params"].to(DT[case["copies"]])
    if case["bits"] == 8:
        (s["m"], s["m_scale"]), (s["v"], s["v_scale"]) = in_blocks(flat["m"]), in_blocks(flat["r"])
    else:
        s["m"], s["v"] = flat["m"], flat["r"].square_()
    s["step"] = torch.full((1,), 1000, device=dev, dtype=torch.int32)
    total = math.sqrt(sum(n * (0.01 * (1 + i % 5)) ** 2 for i, n in enumerate(sizes)))
    s["norm"] = torch.tensor(total, device=dev)
    s["max_norm"] = 0.5 * total
    s["seed"] = seed & 0xffff
    s["at"], s["sizes"] = at, sizes
    return s


# ---- the framework's operators ----------------------------------------------------

_context = None


def operators():
    """One context for all passes, as a serving process or a training loop keeps it."""
    global _context
    if _context is None:
        import paper_2608_14575_gb300 as hwr
        _context = hwr.Operators()
    return _context


def pieces(s, key, per=1):
    """The tensors in a flat buffer (of a value for each `per` elements)."""
    if key not in s:
        return None
    return [s[key][a // per:a // per + -(-n // per)] for a, n in zip(s["at"], s["sizes"])]


def run_own(s):
    ops, case = operators(), s["case"]
    if s["op"] == "experts":
        if case["given"]:
            return {"y": ops.expert_layer(s["x"], s["w_in"], s["w_out"], choice=s["choice"], gates=s["gates"],
                                          activation=case["act"])}
        return {"y": ops.expert_layer(s["x"], s["w_in"], s["w_out"], scores=s["scores"], top=case["top"],
                                      over_all=case["over_all"], activation=case["act"])}
    if s["op"] == "tokens":
        got = ops.token_logprobs(s["logits"], s["token"], top=case["top"])
        out = {"logprob": got.logprob, "entropy": got.entropy}
        if case["top"]:
            out |= {"top_token": got.top_token, "top_logprob": got.top_logprob}
        if case["train"]:
            out["dlogits"] = ops.token_logprobs_backward(s["a"], s["logits"], s["token"], got, dentropy=s["b"])
        return out
    if "state" not in s:     # parameters and moments of a training loop stay where they are
        s["state"] = ops.adamw_state(pieces(s, "params"), bits=case["bits"], copies=pieces(s, "copies"),
                                     m=pieces(s, "m"), v=pieces(s, "v"), m_scale=pieces(s, "m_scale", BLOCK),
                                     v_scale=pieces(s, "v_scale", BLOCK), step=s["step"])
        s["grad_list"] = pieces(s, "grads")
    h = HYPER
    ops.adamw_step(s["state"], s["grad_list"], lr=h["lr"], betas=(h["b1"], h["b2"]), eps=h["eps"],
                   weight_decay=h["decay"], norm=s["norm"], max_norm=s["max_norm"], seed=s["seed"])
    return updated(s)


def updated(s):
    """What a step leaves (8-bit moments as e4m3 values beside their powers of two)."""
    return {k: s[k] for k in ("params", "copies", "m", "v", "m_scale", "v_scale", "step") if k in s}


# ---- the plain form ---------------------------------------------------------------

def activated(u, act):
    if act == "relu":
        return u.clamp(min=0)
    if act == "silu":
        return u / (1 + torch.exp(-u))
    return 0.5 * u * (1 + torch.erf(u * math.sqrt(0.5)))


def keys_of(z):
    """Whole numbers that order a row's values: larger values first, then lower indices."""
    b = z.float().add(0.0).view(torch.int32).long()         # (-0 counts as 0)
    b = torch.where(b >= 0, b, -(b & 0x7fffffff))
    return b * (1 << 31) - torch.arange(z.shape[1], device=z.device)


def plain_choice(scores, top, over_all):
    choice = torch.topk(keys_of(scores), top, dim=1).indices
    p = torch.softmax(scores, 1).gather(1, choice) if over_all else torch.softmax(scores.gather(1, choice), 1)
    return choice, p


def plain_experts(s):
    """Every row through every expert, and what each row's choices make of it."""
    case, x = s["case"], s["x"].float()
    if case["given"]:
        choice, p = s["choice"].long(), s["gates"]
        p = torch.where(choice < 0, torch.zeros_like(p), p)
        choice = choice.clamp(min=0)
    else:
        choice, p = plain_choice(s["scores"], case["top"], case["over_all"])
    h = x @ s["w_in"].float().transpose(1, 2)                       # [E][T][F or 2 F]
    F = case["hidden"]
    h = activated(h[..., :F], case["act"]) * h[..., F:] if case["gated"] else activated(h, case["act"])
    y = h @ s["w_out"].float().transpose(1, 2)                      # [E][T][N]
    weight = torch.zeros(x.shape[0], case["groups"], device=x.device).scatter_add_(1, choice, p)
    return {"y": (y * weight.T[:, :, None]).sum(0).to(s["x"].dtype)}


def plain_tokens(s):
    case, token = s["case"], s["token"]
    z = s["logits"].float()
    z = z - z.amax(1, keepdim=True)
    e = torch.exp(z)
    total = e.sum(1, keepdim=True)
    logq = z - torch.log(total)
    q = e / total
    entropy = -torch.where(q > 0, q * logq, torch.zeros_like(q)).sum(1)
    has = token >= 0
    at = token.clamp(min=0).long()[:, None]
    logprob = torch.where(has, logq.gather(1, at)[:, 0], torch.zeros_like(entropy))
    out = {"logprob": logprob, "entropy": entropy}
    if case["top"]:
        best = torch.topk(keys_of(s["logits"]), case["top"], dim=1).indices
        out |= {"top_token": best.to(torch.int32), "top_logprob": logq.gather(1, best)}
    if case["train"]:
        a = torch.where(has, s["a"], torch.zeros_like(s["a"]))[:, None]
        b = s["b"][:, None]
        d = -q * (a + torch.where(q > 0, b * (logq + entropy[:, None]), torch.zeros_like(q)))
        out["dlogits"] = d.scatter_add_(1, at, a).to(s["logits"].dtype)
    return out


MASK = 0xffffffff


def mixed(x):
    """A hash of 32-bit whole numbers (in 64 bits)."""
    x = ((x ^ (x >> 16)) * 0x7feb352d) & MASK
    x = ((x ^ (x >> 15)) * 0x68e31da5) & MASK
    return x ^ (x >> 16)


def randoms(s, t):
    """32 random bits for each element of the flat buffers, at step t."""
    dev = t.device
    lengths = torch.tensor(s["at"], device=dev).diff()
    number = torch.repeat_interleave(torch.arange(len(s["sizes"]), device=dev), lengths, output_size=s["at"][-1])
    index = torch.arange(s["at"][-1], device=dev) - torch.tensor(s["at"], device=dev)[number]
    key = mixed((mixed((t.long() + s["seed"] * 0x9e3779b1) & MASK) + (number + 1) * 0x85157af5) & MASK)
    return mixed((index * 0x9e3779b1 + key) & MASK)


def to_blocks(x, bits, least):
    """x as e4m3 values (rounded by 16 random bits; not below the least positive one
    where `least` and x is positive) and powers of two."""
    b = x.view(-1, BLOCK)
    field = b.abs().amax(1).view(torch.int32) >> 23
    scale = ((field - 7).clamp(min=1) << 23)
    inverse = ((254 << 23) - scale).view(torch.float32)
    tiny = (b.abs() * inverse[:, None]) * 2.0 ** -120               # e4m3's exponents on fp32's last ones
    code = (tiny.view(torch.int32) + ((bits.view(-1, BLOCK) << 4) | 8).to(torch.int32)) >> 20
    if least:
        code = torch.where((b > 0) & (code == 0), torch.ones_like(code), code)
    code = code | ((b.view(torch.int32) >> 24) & 0x80)
    return code.to(torch.uint8).view(torch.float8_e4m3fn).view(-1), scale.view(torch.float32)


def plain_adamw(s):
    h = HYPER
    g = s["grads"].float() * (torch.full_like(s["norm"], s["max_norm"]) / (s["norm"] + EPS)).clamp(max=1.0)
    t = s["step"] + 1
    if s["case"]["bits"] == 8:
        m = (s["m"].float().view(-1, BLOCK) * s["m_scale"][:, None]).view(-1)
        v = (s["v"].float().view(-1, BLOCK) * s["v_scale"][:, None]).view(-1).square()
    else:
        m, v = s["m"], s["v"]
    m = m * h["b1"] + g * (1 - h["b1"])
    v = v * h["b2"] + (g * g) * (1 - h["b2"])
    c1, c2 = (1 - b ** t.double() for b in (h["b1"], h["b2"]))
    step = m * (1 / c1).float() / (torch.sqrt(v) * c2.rsqrt().float() + h["eps"])
    s["params"].sub_((s["params"] * h["decay"] + step) * h["lr"])
    if "copies" in s:
        s["copies"].copy_(s["params"])
    if s["case"]["bits"] == 8:
        bits = randoms(s, t)
        for key, (x, y) in (("m", to_blocks(m, bits & 0xffff, False)),
                            ("v", to_blocks(torch.sqrt(v), bits >> 16, True))):
            s[key].copy_(x)
            s[key + "_scale"].copy_(y)
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
    s["step"].add_(1)
    return updated(s)


def run_plain(s):
    return {"experts": plain_experts, "tokens": plain_tokens, "adamw": plain_adamw}[s["op"]](s)


def run(state):
    return run_own(state) if own else run_plain(state)


# ---- what a pass cannot do without --------------------------------------------------

def work(case):
    if case["op"] == "experts":
        T, E, D, F, N, k = (case[n] for n in ("rows", "groups", "n_in", "hidden", "n_out", "top"))
        wide = 2 * F if case["gated"] else F
        # (the experts that so many even choices reach, on average)
        used = E * (1 - (1 - k / E) ** T)
        return {"bytes": 2 * used * (wide * D + N * F) + 2 * T * (D + N) + (8 * T if case["given"] else 4 * T * E),
                "flops": 2 * T * k * (wide * D + N * F)}
    if case["op"] == "tokens":
        n, b = case["rows"] * case["vocab"], 4 if case["dtype"] == "f32" else 2
        rows = case["rows"] * (12 + 8 * case["top"] + (8 if case["train"] else 0))
        # (the gradient's pass cannot begin before the whole row is known: it reads again)
        return {"bytes": (3 if case["train"] else 1) * n * b + rows, "flops": (10 if case["train"] else 5) * n}
    n, state = sum(sizes_of(case)), 4 if case["bits"] == 32 else 1 + 4 / BLOCK
    b = 8 + (4 if case["grads"] == "f32" else 2) + (0 if case["copies"] == "none" else 2) + 4 * state
    return {"bytes": b * n, "flops": 16 * n}


# ---- the definition in 64 bits --------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "experts":
        x, F = s["x"].double(), case["hidden"]
        y = torch.zeros(x.shape[0], case["n_out"], dtype=torch.float64, device=x.device)
        for t in range(x.shape[0]):
            if case["given"]:
                picks = [(int(s["choice"][t, 0]), float(s["gates"][t, 0]))]
            else:
                row = [float(v) for v in s["scores"][t].tolist()]
                best = sorted(range(len(row)), key=lambda e: (-row[e], e))[:case["top"]]
                among = row if case["over_all"] else [row[e] for e in best]
                top = max(among)
                total = math.fsum(math.exp(v - top) for v in among)
                picks = [(e, math.exp(row[e] - top) / total) for e in best]
            for e, p in picks:
                if e < 0:
                    continue
                u = s["w_in"][e].double() @ x[t]
                g = u[:F]
                if case["act"] == "silu":
                    h = g * torch.sigmoid(g)
                elif case["act"] == "gelu":
                    h = g * torch.special.ndtr(g)
                else:
                    h = torch.relu(g)
                if case["gated"]:
                    h = h * u[F:]
                y[t] += p * (s["w_out"][e].double() @ h)
        return {"y": y}
    if case["op"] == "tokens":
        got = {"logprob": [], "entropy": [], "top_logprob": [], "dlogits": []}
        for at in range(0, case["rows"], 512):
            z = s["logits"][at:at + 512].double()
            token = s["token"][at:at + 512].long()
            logq = torch.log_softmax(z, 1)
            q = torch.exp(logq)
            entropy = torch.special.entr(q).sum(1)
            mine = torch.gather(logq, 1, token.clamp(min=0)[:, None])[:, 0]
            got["logprob"].append(torch.where(token < 0, torch.zeros_like(mine), mine))
            got["entropy"].append(entropy)
            if case["top"]:
                got["top_logprob"].append(torch.sort(logq, 1, descending=True).values[:, :case["top"]])
            if case["train"]:
                a = s["a"][at:at + 512].double() * (token >= 0)
                b = s["b"][at:at + 512].double()
                spread = torch.special.entr(q) - q * entropy[:, None]       # -q (log q + H)
                d = b[:, None] * spread - a[:, None] * q
                d[torch.arange(d.shape[0], device=d.device), token.clamp(min=0)] += a
                got["dlogits"].append(d)
        out = {k: torch.cat(v) for k, v in got.items() if v}
        if case["top"]:
            out["top_token"] = None
        return out
    h = HYPER
    k = min(1.0, s["max_norm"] / (float(s["norm"]) + EPS))
    g = s["grads"].double() * k
    t = int(s["step"]) + 1
    m, v = s["m"].double(), s["v"].double()
    if case["bits"] == 8:
        m = m * s["m_scale"].double().repeat_interleave(BLOCK)
        v = (v * s["v_scale"].double().repeat_interleave(BLOCK)) ** 2
    m, v = torch.lerp(g, m, h["b1"]), torch.lerp(g ** 2, v, h["b2"])
    w = s["params"].double()
    w = w - h["lr"] * (h["decay"] * w + m / (1 - h["b1"] ** t) / ((v / (1 - h["b2"] ** t)) ** 0.5 + h["eps"]))
    out = dict.fromkeys(updated(s))
    out["params"] = w
    if "copies" in s:
        out["copies"] = w
    if case["bits"] == 32:
        out["m"], out["v"] = m, v
    return out
