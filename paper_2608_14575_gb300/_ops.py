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

OPS_EXPORTS = ("hwr_ops_create", "hwr_ops_destroy", "hwr_ops_synchronize",
               "hwr_ops_last_error", "hwr_ops_reserve", "hwr_ops_after", "hwr_ops_before",
               "hwr_dispatch",
               "hwr_grouped_forward", "hwr_grouped_backward", "hwr_adapter_forward",
               "hwr_adapter_backward", "hwr_clip_gradients", "hwr_gradients_create",
               "hwr_gradients_clip", "hwr_gradients_destroy")


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
