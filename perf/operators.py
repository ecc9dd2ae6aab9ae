"""What follows a routing decision, as measurable cases.

A router answers with one deployment per query (``chosen``, -1 where a query
has none).  Where the deployments share a GPU -- experts with weights of their
own, or low-rank adapters of one base model -- that answer is what the next
operators read:

  dispatch   the rows of each choice together, in their own order: offsets
             [G + 1] and order [T] (rows without a choice come last);
  grouped    y[t] = W[choice[t]] x[t]: one product with ragged groups of rows,
             forward, or backward (dx[t] = W[choice[t]]^T dy[t] and
             dW[g] = sum of dy[t] x[t]^T over the rows of g);
  adapter    y[t] = W x[t] + s[c] B[c] (A[c] x[t]), c = choice[t]: a projection
             shared by all rows and each row's own low-rank adapter, forward,
             or backward (dx, dA, dB; the shared projection stays as it is);
  clip       the norm over all gradients together, and the gradients scaled
             by min(1, max_norm / (norm + 1e-6)).

A row without a choice has y = 0 and dx = 0 in the grouped product, and the
shared projection alone with adapters.  Weights are [out][in].

What the fields of a case mean: ``op`` the operator, ``train`` its backward
pass, ``rows`` T, ``groups`` G, ``n_in`` / ``n_out`` the widths, ``rank`` the
adapters' rank, ``skew`` how unevenly the choices fall (standard deviation of
the log popularity), ``dtype`` the type of inputs, weights and outputs; for
clip ``tensors`` and ``largest`` (elements of the largest) give the sizes.
"""
from __future__ import annotations

import math

import torch

own = False

DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "f32": torch.float32}
NO_CHOICE = 0.01        # share of rows without a choice
EPS = 1e-6

# The most that a drawn case costs (that of the listed ones or less).
MOST_FLOPS = 2.6e11
MOST_WEIGHTS = 1 << 27
MOST_GRADS = 1 << 27


def listed():
    return [
        # The requests of one micro-batch on a cluster of 12 deployments, sorted
        # by their deployment: latency is all that counts.
        dict(name="dispatch_micro_batch", op="dispatch", rows=64, groups=12, skew=0.7),
        # The largest batch of the router's sweep, on 64 deployments.
        dict(name="dispatch_sweep", op="dispatch", rows=1_048_576, groups=64, skew=0.7),
        # One decode step of a micro-batch through 12 experts: every weight is
        # read for a handful of rows.
        dict(name="grouped_step", op="grouped", train=False, rows=64, groups=12, n_in=1024,
             n_out=4096, skew=0.7, dtype="bf16"),
        # A prefill of a few thousand tokens over 32 experts, unevenly taken.
        dict(name="grouped_prefill", op="grouped", train=False, rows=4001, groups=32, n_in=1024,
             n_out=4096, skew=1.0, dtype="bf16"),
        # A full batch over 64 experts, in half precision.
        dict(name="grouped_batch", op="grouped", train=False, rows=65_536, groups=64, n_in=1024,
             n_out=2048, skew=0.5, dtype="fp16"),
        # The backward pass of a training step's expert layer.
        dict(name="grouped_train", op="grouped", train=True, rows=8191, groups=16, n_in=1024,
             n_out=4096, skew=0.7, dtype="bf16"),
        # One token of one request through a projection with 32 adapters loaded.
        dict(name="adapter_token", op="adapter", train=False, rows=1, groups=32, n_in=4096,
             n_out=4096, rank=16, skew=0.7, dtype="bf16"),
        # One decode step of 64 requests, each with the adapter of its choice.
        dict(name="adapter_step", op="adapter", train=False, rows=64, groups=64, n_in=4096,
             n_out=4096, rank=16, skew=0.5, dtype="bf16"),
        # A prefill of mixed requests in half precision.
        dict(name="adapter_prefill", op="adapter", train=False, rows=8191, groups=12, n_in=4096,
             n_out=4096, rank=64, skew=0.7, dtype="fp16"),
        # A training step of 8 adapters side by side.
        dict(name="adapter_train", op="adapter", train=True, rows=4096, groups=8, n_in=4096,
             n_out=2048, rank=32, skew=0.7, dtype="bf16"),
        # The gradients of a set of adapters: many small tensors.
        dict(name="clip_adapters", op="clip", tensors=48, largest=65_536, dtype="bf16"),
        # The gradients of whole layers, kept in 32 bits.
        dict(name="clip_layers", op="clip", tensors=16, largest=16_777_216, dtype="f32"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    w = _log(rng, lo, hi)
    return w if rng.random() < 0.25 else max(8, w // 8 * 8)   # mostly whole 16-byte rows


def draw(rng):
    op = rng.choice(("dispatch", "grouped", "grouped", "adapter", "adapter", "clip"))
    if op == "dispatch":
        return dict(op=op, rows=_log(rng, 1, 1_048_576), groups=_log(rng, 1, 512),
                    skew=round(rng.uniform(0, 1.5), 2))
    if op == "clip":
        n, most = _log(rng, 1, 60), _log(rng, 1000, 1 << 24)
        return dict(op=op, tensors=n, largest=min(most, MOST_GRADS // n),
                    dtype=rng.choice(("bf16", "fp16", "f32")))
    case = dict(op=op, train=rng.random() < 0.4, rows=_log(rng, 1, 65_536),
                groups=_log(rng, 1, 64 if op == "grouped" else 128),
                n_in=_width(rng, 64, 4096), n_out=_width(rng, 64, 4096),
                skew=round(rng.uniform(0, 1.2), 2), dtype=rng.choice(("bf16", "fp16")))
    if op == "adapter":
        case["rank"] = rng.choice((4, 8, 12, 16, 24, 32, 64, 100, 128))
        case["rows"] = min(case["rows"], 16_384)
    else:
        case["groups"] = max(1, min(case["groups"], MOST_WEIGHTS // (case["n_in"] * case["n_out"])))
    most = MOST_FLOPS / (2.0 * case["n_in"] * case["n_out"] * (2 if case["train"] else 1))
    case["rows"] = max(1, min(case["rows"], int(most)))
    return case


# ---- inputs -------------------------------------------------------------------

def clip_sizes(case):
    """Elements of each tensor: matrices, halves and quarters of them, biases, odd ones."""
    big = case["largest"]
    return [max(1, (big, big // 2, big // 4 + 1, big // 64)[i % 4] - (i % 3)) for i in range(case["tensors"])]


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)

    def normal(*shape, std=1.0, dtype=torch.float32):
        return torch.empty(shape, device=dev, dtype=dtype).normal_(0.0, std, generator=gen)

    s = dict(case=case, op=case["op"])
    if case["op"] == "clip":
        sizes, dt = clip_sizes(case), DT[case["dtype"]]
        # a step whose gradients are too large by a factor of 2 or so
        s["grads"] = [normal(n, std=0.01 * (1 + i % 5), dtype=dt) for i, n in enumerate(sizes)]
        s["out"] = [torch.empty_like(g) for g in s["grads"]]
        s["max_norm"] = 0.5 * math.sqrt(sum(n * (0.01 * (1 + i % 5)) ** 2 for i, n in enumerate(sizes)))
        return s

    T, G = case["rows"], case["groups"]
    share = torch.softmax(normal(G, std=case["skew"] or 1e-3), 0)
    choice = torch.multinomial(share, T, replacement=True, generator=gen).to(torch.int32)
    none = torch.rand(T, device=dev, generator=gen) < NO_CHOICE
    s["choice"] = torch.where(none, torch.full_like(choice, -1), choice)
    s["groups"] = G
    if case["op"] == "dispatch":
        return s
    K, N, dt = case["n_in"], case["n_out"], DT[case["dtype"]]
    s["x"] = normal(T, K, dtype=dt)
    if case["train"]:
        s["dy"] = normal(T, N, std=0.1, dtype=dt)
    if case["op"] == "grouped":
        s["w"] = normal(G, N, K, std=K ** -0.5, dtype=dt)
    else:
        R = case["rank"]
        s["w"] = normal(N, K, std=K ** -0.5, dtype=dt)
        s["a"] = normal(G, R, K, std=K ** -0.5, dtype=dt)
        s["b"] = normal(G, N, R, std=0.3 * R ** -0.5, dtype=dt)
        s["scale"] = 0.5 + 1.5 * torch.rand(G, device=dev, generator=gen)
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


def run_own(s):
    ops = operators()
    if s["op"] == "clip":
        if "list" not in s:     # the gradient buffers of a training loop stay the same
            s["list"] = ops.gradient_list(s["grads"], s["out"])
        norm = ops.clip_gradients(s["list"], s["max_norm"])
        return {"norm": norm, "grads": s["out"]}
    plan = ops.dispatch(s["choice"], s["groups"])
    if s["op"] == "dispatch":
        return {"offsets": plan.offsets, "order": plan.order}
    if s["op"] == "grouped":
        if "dy" not in s:
            return {"y": ops.grouped_forward(s["x"], s["w"], plan)}
        dx, dw = ops.grouped_backward(s["dy"], s["x"], s["w"], plan)
        return {"dx": dx, "dw": dw}
    if "dy" not in s:
        return {"y": ops.adapter_forward(s["x"], s["w"], s["a"], s["b"], s["scale"], plan)}
    dx, da, db = ops.adapter_backward(s["dy"], s["x"], s["w"], s["a"], s["b"], s["scale"], plan)
    return {"dx": dx, "da": da, "db": db}


# ---- the plain form ---------------------------------------------------------------

def plain_dispatch(choice, G):
    key = torch.where((choice >= 0) & (choice < G), choice, torch.full_like(choice, G)).long()
    sorted_key, order = torch.sort(key, stable=True)
    offsets = torch.searchsorted(sorted_key, torch.arange(G + 1, device=key.device))
    return offsets.to(torch.int32), order.to(torch.int32)


class Padded:
    """The rows of each group side by side, padded to the longest group."""

    def __init__(self, choice, G):
        offsets, order = plain_dispatch(choice, G)
        offsets, order = offsets.long(), order.long()
        self.G, self.T = G, choice.numel()
        self.row = order[:int(offsets[-1])]
        self.group = choice[self.row].long()
        self.at = torch.arange(self.row.numel(), device=choice.device) - offsets[self.group]
        self.most = max(1, int((offsets[1:] - offsets[:-1]).max()))

    def spread(self, x):
        p = torch.zeros(self.G, self.most, x.shape[1], device=x.device)
        p[self.group, self.at] = x[self.row].float()
        return p

    def gather(self, p):
        y = torch.zeros(self.T, p.shape[2], device=p.device)
        y[self.row] = p[self.group, self.at]
        return y


def plain_rows(x, w, choice):
    """x[t] times w[choice[t]] [out][in], for a few rows: each row's own matrix is taken."""
    y = (w[choice.clamp(min=0).long()].float() @ x.float()[:, :, None])[:, :, 0]
    return y * (choice >= 0)[:, None]


def plain_grouped(s):
    x, w, choice, dt = s["x"], s["w"], s["choice"], s["x"].dtype
    if "dy" not in s:
        if x.shape[0] < w.shape[0]:
            return {"y": plain_rows(x, w, choice).to(dt)}
        p = Padded(choice, w.shape[0])
        return {"y": p.gather(p.spread(x) @ w.float().transpose(1, 2)).to(dt)}
    p = Padded(choice, w.shape[0])
    dy = p.spread(s["dy"])
    return {"dx": p.gather(dy @ w.float()).to(dt), "dw": (dy.transpose(1, 2) @ p.spread(x)).to(dt)}


def plain_adapter(s):
    x, w, a, b, scale, choice = s["x"], s["w"], s["a"], s["b"], s["scale"], s["choice"]
    dt = x.dtype
    if "dy" not in s:
        y = x.float() @ w.float().T
        if x.shape[0] <= 2 * a.shape[0]:
            u = plain_rows(x, a, choice) * scale[choice.clamp(min=0).long()][:, None]
            return {"y": (y + plain_rows(u, b, choice)).to(dt)}
        p = Padded(choice, a.shape[0])
        u = (p.spread(x) @ a.float().transpose(1, 2)) * scale[:, None, None]
        return {"y": (y + p.gather(u @ b.float().transpose(1, 2))).to(dt)}
    p = Padded(choice, a.shape[0])
    dy, px = p.spread(s["dy"]), p.spread(x)
    u = (px @ a.float().transpose(1, 2)) * scale[:, None, None]
    v = (dy @ b.float()) * scale[:, None, None]
    dx = s["dy"].float() @ w.float() + p.gather(v @ a.float())
    return {"dx": dx.to(dt), "da": (v.transpose(1, 2) @ px).to(dt), "db": (dy.transpose(1, 2) @ u).to(dt)}


def plain_clip(s):
    grads = s["grads"]
    norm = torch.stack([g.float().square().sum() for g in grads]).sum().sqrt()
    coef = (s["max_norm"] / (norm + EPS)).clamp(max=1.0)
    return {"norm": norm, "grads": [(g.float() * coef).to(g.dtype) for g in grads]}


def run_plain(s):
    if s["op"] == "dispatch":
        offsets, order = plain_dispatch(s["choice"], s["groups"])
        return {"offsets": offsets, "order": order}
    return {"grouped": plain_grouped, "adapter": plain_adapter, "clip": plain_clip}[s["op"]](s)


def run(state):
    return run_own(state) if own else run_plain(state)


# ---- what a pass cannot do without --------------------------------------------------

def work(case):
    if case["op"] == "clip":
        n, b = sum(clip_sizes(case)), 4 if case["dtype"] == "f32" else 2
        return {"bytes": 2 * b * n + 4, "flops": 3 * n}
    T, G = case["rows"], case["groups"]
    dispatch = 4 * T + 4 * T + 4 * (G + 1)
    if case["op"] == "dispatch":
        return {"bytes": dispatch, "flops": 0}
    K, N, used = case["n_in"], case["n_out"], min(T, G)
    if case["op"] == "grouped":
        if not case["train"]:
            return {"bytes": 4 * T + 2 * (T * K + used * N * K + T * N), "flops": 2 * T * N * K}
        return {"bytes": 4 * T + 2 * (2 * T * K + T * N + used * N * K + G * N * K),
                "flops": 4 * T * N * K}
    R = case["rank"]
    low = used * R * (K + N)
    if not case["train"]:
        return {"bytes": 4 * T + 2 * (T * K + N * K + low + T * N) + 4 * G,
                "flops": 2 * T * (N * K + R * (K + N))}
    return {"bytes": 4 * T + 2 * (2 * T * K + T * N + N * K + low + G * R * (K + N)) + 4 * G,
            "flops": 2 * T * (N * K + 3 * R * (K + N))}


# ---- the definition in 64 bits --------------------------------------------------------

def exact(case, seed):
    if case["op"] == "dispatch":
        return None
    s = prepare(case, seed)
    if case["op"] == "clip":
        total = sum(float(torch.dot(g.double(), g.double())) for g in s["grads"])
        norm = math.sqrt(total)
        k = min(1.0, s["max_norm"] / (norm + EPS))
        return {"norm": torch.tensor(norm, dtype=torch.float64), "grads": [g.double() * k for g in s["grads"]]}
    x, w, choice = s["x"].double(), s["w"], s["choice"].cpu()
    T, K = x.shape
    N = case["n_out"]
    zeros = lambda *n: torch.zeros(*n, dtype=torch.float64, device=x.device)  # noqa: E731
    rows_of = [torch.nonzero(choice == g).flatten().to(x.device) for g in range(case["groups"])]
    if case["op"] == "grouped":
        if not case["train"]:
            y = zeros(T, N)
            for g, r in enumerate(rows_of):
                y[r] = x[r] @ w[g].double().T
            return {"y": y}
        dy, dx, dw = s["dy"].double(), zeros(T, K), zeros(*w.shape)
        for g, r in enumerate(rows_of):
            dx[r] = dy[r] @ w[g].double()
            dw[g] = dy[r].T @ x[r]
        return {"dx": dx, "dw": dw}
    wd, scale = w.double(), s["scale"].double()
    if not case["train"]:
        y = x @ wd.T
        for g, r in enumerate(rows_of):
            y[r] += scale[g] * ((x[r] @ s["a"][g].double().T) @ s["b"][g].double().T)
        return {"y": y}
    dy = s["dy"].double()
    dx, da, db = dy @ wd, zeros(*s["a"].shape), zeros(*s["b"].shape)
    for g, r in enumerate(rows_of):
        a, b = s["a"][g].double(), s["b"][g].double()
        v = scale[g] * (dy[r] @ b)
        dx[r] += v @ a
        da[g] = v.T @ x[r]
        db[g] = scale[g] * (dy[r].T @ (x[r] @ a.T))
    return {"dx": dx, "da": da, "db": db}
