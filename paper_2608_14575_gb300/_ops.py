"""Binding of the operators that follow a routing decision (include/hwr_ops.h).

``Operators`` wraps one context for CUDA tensors: it checks the arguments,
allocates the outputs and queues the library's kernels (csrc/ops_torch.cpp).  As
in ``_hwr`` there is no other path: without the built library it raises.  The C
functions keep their names in ``load_ops()``, their structures below.

    ops = Operators()
    plan = ops.dispatch(chosen, groups)                 # rows by their choice
    y = ops.grouped_forward(x, w, plan)                 # y[t] = W[c] x[t]
    dx, dw = ops.grouped_backward(dy, x, w, plan)
    y = ops.adapter_forward(x, w, a, b, scale, plan)    # W x + scale B (A x)
    dx, da, db = ops.adapter_backward(dy, x, w, a, b, scale, plan)
    norm = ops.clip_gradients([dw, ...], max_norm=1.0)  # in place
    state = ops.adamw_state([w32, ...], copies=[w, ...])
    ops.adamw_step(state, [dw, ...], lr=1e-3)           # w32 and w
    y = ops.expert_layer(x, w_in, w_out, scores=s, top=2)   # a decode step's few rows
    got = ops.token_logprobs(logits, token, top=5)
    dlogits = ops.token_logprobs_backward(a, logits, token, got)

Tensors are CUDA tensors of the context's device whose last dimension is
contiguous; other strides are free.  The context is bound to the torch stream
that is current when it is made.  A call made under another current stream is
ordered after that stream's work so far, and that stream after the call.

Nothing is recorded for autograd: results have no gradient function, whatever the
inputs require, and the ``_backward`` calls are made by hand (or from a
``torch.autograd.Function`` of the caller's).  Tensors that a call writes in place
(``out``, clipped gradients) count as modified, so that autograd notices where it
had saved them.

Calls can be captured into CUDA graphs once the workspace is large enough: after
a call of the same sizes, or ``reserve`` (a capture in which it would have to grow
raises HwrError).  What a graph uses of the workspace stays until ``close``.  A
replay shares it with the context's other calls, so order them: replay on the
context's stream, or on one that the other calls are ordered with.
"""
from __future__ import annotations

import ctypes as ct
import importlib.util
import os

from . import _hwr
from . import build as _build
from ._hwr import HwrError

HWR_F16 = 2
HWR_OPS_MAX_GROUPS = 1024
HWR_OPS_MAX_RANK = 256
HWR_EXPERTS_MAX_ROWS = 128
HWR_EXPERTS_MAX_TOP = 16
HWR_EXPERTS_MAX_OUT = 65536
HWR_EXPERTS_MAX_WIDTH = 262144
HWR_TOKENS_MAX_TOP = 32
HWR_ADAMW_BLOCK = 256
ACTIVATIONS = {"silu": 0, "gelu": 1, "relu": 2}

OPS_EXPORTS = ("hwr_ops_create", "hwr_ops_destroy", "hwr_ops_synchronize",
               "hwr_ops_last_error", "hwr_ops_reserve", "hwr_ops_after", "hwr_ops_before",
               "hwr_dispatch",
               "hwr_grouped_forward", "hwr_grouped_backward", "hwr_adapter_forward",
               "hwr_adapter_backward", "hwr_clip_gradients", "hwr_gradients_create",
               "hwr_gradients_clip", "hwr_gradients_destroy", "hwr_adamw_create",
               "hwr_adamw_step", "hwr_adamw_destroy", "hwr_expert_layer",
               "hwr_token_logprobs", "hwr_token_logprobs_backward")


class hwr_rows(ct.Structure):
    _fields_ = [("rows", ct.c_int32), ("groups", ct.c_int32), ("n_in", ct.c_int32),
                ("n_out", ct.c_int32), ("dtype", ct.c_int), ("offsets", ct.c_void_p),
                ("order", ct.c_void_p), ("x", ct.c_void_p), ("x_ld", ct.c_int64),
                ("w", ct.c_void_p), ("w_ld", ct.c_int64), ("w_group", ct.c_int64)]


class hwr_adapters(ct.Structure):
    _fields_ = [("rank", ct.c_int32), ("a", ct.c_void_p), ("b", ct.c_void_p),
                ("scale", ct.c_void_p)]


class hwr_gradient(ct.Structure):
    _fields_ = [("in_", ct.c_void_p), ("out", ct.c_void_p), ("n", ct.c_int64),
                ("dtype", ct.c_int)]


class hwr_adamw_tensor(ct.Structure):
    _fields_ = [("param", ct.c_void_p), ("copy", ct.c_void_p), ("copy_dtype", ct.c_int),
                ("m", ct.c_void_p), ("v", ct.c_void_p), ("m_scale", ct.c_void_p),
                ("v_scale", ct.c_void_p), ("n", ct.c_int64)]


class hwr_adamw_options(ct.Structure):
    _fields_ = [("lr", ct.c_double), ("beta1", ct.c_double), ("beta2", ct.c_double),
                ("eps", ct.c_double), ("weight_decay", ct.c_double), ("lr_device", ct.c_void_p),
                ("norm", ct.c_void_p), ("max_norm", ct.c_float), ("seed", ct.c_uint32)]


class hwr_experts(ct.Structure):
    _fields_ = [("rows", ct.c_int32), ("groups", ct.c_int32), ("top", ct.c_int32),
                ("n_in", ct.c_int32), ("hidden", ct.c_int32), ("n_out", ct.c_int32),
                ("dtype", ct.c_int), ("activation", ct.c_int), ("gated", ct.c_int32),
                ("over_all", ct.c_int32), ("x", ct.c_void_p), ("x_ld", ct.c_int64),
                ("w_in", ct.c_void_p), ("w_in_ld", ct.c_int64), ("w_in_group", ct.c_int64),
                ("w_out", ct.c_void_p), ("w_out_ld", ct.c_int64), ("w_out_group", ct.c_int64),
                ("scores", ct.c_void_p), ("scores_ld", ct.c_int64), ("choice", ct.c_void_p),
                ("gates", ct.c_void_p)]


class hwr_logits(ct.Structure):
    _fields_ = [("rows", ct.c_int32), ("vocab", ct.c_int32), ("dtype", ct.c_int),
                ("logits", ct.c_void_p), ("ld", ct.c_int64), ("token", ct.c_void_p)]


_ready = None


def load_ops():
    """libhwr with the operators' signatures set."""
    global _ready
    if _ready is None:
        lib = _hwr.load()
        P, L, I = ct.c_void_p, ct.c_int64, ct.c_int32
        lib.hwr_ops_create.argtypes = [P, ct.POINTER(P)]
        lib.hwr_ops_destroy.argtypes = [P]
        lib.hwr_ops_synchronize.argtypes = [P]
        lib.hwr_ops_last_error.argtypes = [P]
        lib.hwr_ops_reserve.argtypes = [P, ct.c_uint64]
        lib.hwr_ops_after.argtypes = lib.hwr_ops_before.argtypes = [P, P]
        lib.hwr_dispatch.argtypes = [P, I, I, P, P, P]
        lib.hwr_grouped_forward.argtypes = [P, P, P, L]
        lib.hwr_grouped_backward.argtypes = [P, P, P, L, P, L, P]
        lib.hwr_adapter_forward.argtypes = [P, P, P, P, L]
        lib.hwr_adapter_backward.argtypes = [P, P, P, P, L, P, L, P, P]
        lib.hwr_clip_gradients.argtypes = [P, I, P, ct.c_float, P]
        lib.hwr_gradients_create.argtypes = [P, I, P, ct.POINTER(P)]
        lib.hwr_gradients_clip.argtypes = [P, P, ct.c_float, P]
        lib.hwr_gradients_destroy.argtypes = [P, P]
        lib.hwr_adamw_create.argtypes = [P, I, P, I, P, ct.POINTER(P)]
        lib.hwr_adamw_step.argtypes = [P, P, P, P, P]
        lib.hwr_adamw_destroy.argtypes = [P, P]
        lib.hwr_expert_layer.argtypes = [P, P, P, L]
        lib.hwr_token_logprobs.argtypes = [P, P, I, P, P, P, P, P]
        lib.hwr_token_logprobs_backward.argtypes = [P, P, P, P, P, P, P, L]
        for n in OPS_EXPORTS:
            getattr(lib, n).restype = ct.c_int
        lib.hwr_ops_last_error.restype = ct.c_char_p
        _ready = lib
    return _ready


_native = None


def _binding():
    """The torch binding (csrc/ops_torch.cpp); raises if it is not built."""
    global _native
    if _native is None:
        import torch  # noqa: F401  (its libraries come first)
        load_ops()
        path = _build.torch_path()
        if not os.path.exists(path):
            raise RuntimeError(f"the operators' binding is not built ({path} missing); run "
                               "__graft_entry__.build() or paper_2608_14575_gb300/build.py")
        spec = importlib.util.spec_from_file_location("hwr_torch", path)
        native = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(native)
        native.set_error(HwrError)
        _native = native
    return _native


class Plan:
    """Rows grouped by choice: ``offsets`` [groups + 1] and ``order`` [rows]."""
    __slots__ = ("offsets", "order")

    def __init__(self, offsets, order):
        self.offsets, self.order = offsets, order

    @property
    def rows(self) -> int:
        return self.order.numel()

    @property
    def groups(self) -> int:
        return self.offsets.numel() - 1


class GradientList:
    """The gradients of a training loop, laid out once for ``clip_gradients``:
    made by ``Operators.gradient_list``."""

    def __init__(self, ops, grads, out):
        self.ops, self.grads, self.out = ops, grads, out     # (the tensors stay alive)
        self.handle = 0
        self.handle = ops.native.list_create(ops.ctx, ops._current(), grads, out)

    def close(self):
        if self.handle and self.ops.ctx:      # (a closed context has freed its lists)
            self.ops.native.list_destroy(self.ops.ctx, self.handle)
        self.handle = 0

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class TokenLogprobs:
    """Of a row of logits each: ``logprob`` of its token, ``entropy``, ``stats`` [rows][2]
    (largest logit, log of the sum of exp(z - largest)), ``top_token`` and
    ``top_logprob`` [rows][top] (None without alternatives)."""
    __slots__ = ("logprob", "entropy", "stats", "top_token", "top_logprob")

    def __init__(self, *values):
        self.logprob, self.entropy, self.stats, self.top_token, self.top_logprob = values


class AdamWState:
    """Parameters and moments of an optimizer, made by ``Operators.adamw_state``.  The
    tensors stay where they are; save and restore them in place.  ``m`` and ``v`` are
    fp32, or (8 bits) e4m3 values of m and sqrt(v) with a power of two for each
    ``HWR_ADAMW_BLOCK`` elements in ``m_scale`` and ``v_scale``; ``step`` [1] int32
    counts the steps done."""

    def __init__(self, ops, params, bits, copies, m, v, m_scale, v_scale, step):
        self.ops, self.params, self.bits, self.copies = ops, params, bits, copies
        self.m, self.v, self.m_scale, self.v_scale, self.step = m, v, m_scale, v_scale, step
        self.handle = 0
        self.handle = ops.native.adamw_create(ops.ctx, ops._current(), params, copies, m, v, m_scale,
                                              v_scale, bits, step)

    def moments(self, i: int):
        """(m, v) of tensor i in fp32."""
        if self.bits == 32:
            return self.m[i], self.v[i]

        def wide(values, scale):
            flat = values.float().view(-1)
            return (flat * scale.repeat_interleave(HWR_ADAMW_BLOCK)[:flat.numel()]).view(values.shape)
        return wide(self.m[i], self.m_scale[i]), wide(self.v[i], self.v_scale[i]).square()

    def close(self):
        if self.handle:
            self.ops.native.adamw_destroy(self.ops.ctx, self.handle)
        self.handle = 0

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Operators:
    """One context (see the module's text).  ``stream``: a torch stream other than
    the current one."""

    def __init__(self, stream=None):
        import torch
        self.ctx = 0
        self.native = _binding()
        if not torch.cuda.is_available():
            raise RuntimeError("no CUDA device")
        device = torch.cuda.current_device()
        self.stream = torch.cuda.current_stream() if stream is None else stream
        # the raw handle of the stream that is current at a call
        raw = torch._C._cuda_getCurrentRawStream
        self._current = lambda: raw(device)
        self.ctx = self.native.create(self.stream.cuda_stream, device)

    def dispatch(self, choice, groups: int) -> Plan:
        """Bring the rows of each choice together.  ``choice`` [rows] int32;
        values outside [0, groups) are rows without a choice."""
        return Plan(*self.native.dispatch(self.ctx, self._current(), choice, groups))

    def grouped_forward(self, x, w, plan: Plan, out=None):
        """y[t] = w[c] x[t] for x [rows][K], w [groups][N][K] -> [rows][N];
        rows without a choice get zeros."""
        y = self.native.grouped_forward(self.ctx, self._current(), x, w, plan.offsets, plan.order, out)
        return y if out is None else out

    def grouped_backward(self, dy, x, w, plan: Plan, need_dx=True, need_dw=True):
        """(dx [rows][K], dw laid out as w) from dy [rows][N]; None where not
        asked for."""
        return self.native.grouped_backward(self.ctx, self._current(), dy, x, w, plan.offsets,
                                            plan.order, need_dx, need_dw)

    def adapter_forward(self, x, w, a, b, scale, plan: Plan, out=None):
        """y[t] = w x[t] + scale[c] b[c] (a[c] x[t]) for w [N][K],
        a [groups][rank][K], b [groups][N][rank], scale [groups] fp32; rows
        without a choice get w x[t]."""
        y = self.native.adapter_forward(self.ctx, self._current(), x, w, a, b, scale, plan.offsets,
                                        plan.order, out)
        return y if out is None else out

    def adapter_backward(self, dy, x, w, a, b, scale, plan: Plan, need_dx=True, need_dab=True):
        """(dx, da, db) of ``adapter_forward`` from dy [rows][N] (the shared
        projection is not trained); None where not asked for."""
        return self.native.adapter_backward(self.ctx, self._current(), dy, x, w, a, b, scale,
                                            plan.offsets, plan.order, need_dx, need_dab)

    def gradient_list(self, grads, out=None) -> GradientList:
        """Lay out gradients that stay where they are for ``clip_gradients`` at
        every step.  ``out``: where the clipped ones go (default: in place)."""
        grads = list(grads)
        return GradientList(self, grads, grads if out is None else list(out))

    def clip_gradients(self, grads, max_norm: float, out=None):
        """Scale the gradients by min(1, max_norm / (norm + 1e-6)); returns the
        norm over all of them before that, a scalar tensor on the device.
        ``grads``: tensors (``out``: where the clipped ones go, default in
        place), or a ``gradient_list``."""
        if isinstance(grads, GradientList):
            if out is not None or grads.ops is not self or not grads.handle:
                raise ValueError("a gradient list has its outputs, its context, and is open")
            return self.native.list_clip(self.ctx, self._current(), grads.handle, max_norm, grads.out)
        grads = list(grads)
        return self.native.clip(self.ctx, self._current(), grads,
                                grads if out is None else list(out), max_norm)

    def adamw_state(self, params, bits: int = 32, copies=None, m=None, v=None, m_scale=None, v_scale=None,
                    step=None) -> AdamWState:
        """State of an AdamW run over fp32 tensors ``params``, with ``copies`` in bf16 or
        fp16 (None, or None for some) that each step rounds them to.  Moments of ``bits`` 32 or 8,
        zeros unless they are given (lists as in ``AdamWState``), like ``step``.  None of these
        tensors may overlap another."""
        import torch
        params = list(params)
        kind = torch.float8_e4m3fn if bits == 8 else torch.float32
        blocks = [-(-p.numel() // HWR_ADAMW_BLOCK) for p in params]

        def state(given, wanted, shapes=None, dtype=torch.float32):
            if given is not None or not wanted:
                return None if given is None else list(given)
            return [torch.zeros(s, dtype=dtype, device=p.device) for s, p in zip(shapes, params)]
        shapes = [p.shape for p in params]
        m, v = state(m, True, shapes, kind), state(v, True, shapes, kind)
        m_scale, v_scale = state(m_scale, bits == 8, blocks), state(v_scale, bits == 8, blocks)
        if step is None:
            step = torch.zeros(1, dtype=torch.int32, device=self.stream.device)
        return AdamWState(self, params, bits, state(copies, False), m, v, m_scale, v_scale, step)

    def adamw_step(self, state: AdamWState, grads, lr, betas=(0.9, 0.999), eps: float = 1e-8,
                   weight_decay: float = 0.01, norm=None, max_norm: float = float("inf"), seed: int = 0):
        """One step (``state.step`` counts it): ``grads`` a gradient (fp32, bf16, fp16;
        contiguous, of its shape) or None for each parameter, ``lr`` a number or an fp32 tensor on the
        device.  With ``norm``
        (of ``clip_gradients``, max_norm inf: left as they are) the gradients are taken times
        min(1, max_norm / (norm + 1e-6)), and a step whose norm is not finite is left
        out.  ``seed``: of the 8-bit moments' rounding."""
        if state.ops is not self or not state.handle:
            raise ValueError("a state has its context, and is open")
        self.native.adamw_step(self.ctx, self._current(), state.handle,
                               grads if type(grads) is list else list(grads), lr, betas[0], betas[1], eps,
                               weight_decay, norm, max_norm, seed)

    def expert_layer(self, x, w_in, w_out, scores=None, top: int = 1, over_all: bool = False, choice=None,
                     gates=None, activation: str = "silu", out=None):
        """A layer of experts for up to ``HWR_EXPERTS_MAX_ROWS`` rows x [rows][K]:
        y[t] = sum of p[t, j] w_out[e] h over the row's choices e, with
        w_in [groups][2 F][K] h = act(w_in[e][:F] x[t]) * (w_in[e][F:] x[t]), with
        [groups][F][K] h = act(w_in[e] x[t]); w_out [groups][N][F].  ``scores``
        [rows][groups] fp32: the ``top`` largest are the choices (never NaN or -inf), p the
        softmax over them (``over_all``: over all scores, NaN where one of those is).  Or
        ``choice`` [rows][top] int32 (outside [0, groups): none) and ``gates`` [rows][top]
        fp32, the p.  ``activation``: "silu", "gelu" (u Phi(u)), "relu"."""
        if activation not in ACTIVATIONS:
            raise ValueError(f"activation {activation!r}: want one of {', '.join(ACTIVATIONS)}")
        y = self.native.expert_layer(self.ctx, self._current(), x, w_in, w_out, scores, top, over_all, choice,
                                     gates, ACTIVATIONS[activation], out)
        return y if out is None else out

    def token_logprobs(self, logits, token=None, top: int = 0) -> TokenLogprobs:
        """Log probability of each row's ``token`` [rows] int32 (0 for one outside
        [0, vocab)) under softmax(logits [rows][vocab]), entropies, and the ``top`` most
        probable tokens."""
        return TokenLogprobs(*self.native.token_logprobs(self.ctx, self._current(), logits, token, top))

    def token_logprobs_backward(self, dlogprob, logits, token, got: TokenLogprobs, dentropy=None, out=None):
        """The gradient with respect to the logits of sum(dlogprob * logprob + dentropy *
        entropy) (either may be None), in the logits' type; ``out`` may be the logits."""
        dz = self.native.token_logprobs_backward(self.ctx, self._current(), dlogprob, logits, token, got.entropy,
                                                 got.stats, dentropy, out)
        return dz if out is None else out

    def reserve(self, nbytes: int):
        """Make the workspace at least ``nbytes`` large (before a stream capture)."""
        self.native.reserve(self.ctx, self._current(), nbytes)

    def synchronize(self):
        self.native.synchronize(self.ctx)

    def close(self):
        if self.ctx:
            self.native.destroy(self.ctx)
            self.ctx = 0

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
