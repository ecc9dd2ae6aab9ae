"""Binding of the operators that follow a routing decision (include/hwr_ops.h).

``Operators`` wraps one context for CUDA tensors: it checks the arguments,
allocates the outputs and queues the library's kernels.  As in ``_hwr`` there is
no other path: without the built library the first call raises.

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
"""
from __future__ import annotations

import ctypes as ct

from . import _hwr
from ._hwr import HWR_BF16, HWR_F32, HWR_OK, HwrError

HWR_F16 = 2
HWR_OPS_MAX_GROUPS = 1024
HWR_OPS_MAX_RANK = 256

OPS_EXPORTS = ("hwr_ops_create", "hwr_ops_destroy", "hwr_ops_synchronize",
               "hwr_ops_last_error", "hwr_ops_reserve", "hwr_dispatch",
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


class Plan:
    """Rows grouped by choice: ``offsets`` [groups + 1] and ``order`` [rows]."""
    __slots__ = ("offsets", "order", "rows", "groups", "_po", "_pr")

    def __init__(self, offsets, order):
        self.offsets, self.order = offsets, order
        self.rows, self.groups = order.numel(), offsets.numel() - 1
        self._po, self._pr = offsets.data_ptr(), order.data_ptr()


class GradientList:
    """The gradients of a training loop, laid out once for ``clip_gradients``:
    made by ``Operators.gradient_list``."""

    def __init__(self, ops, grads, out):
        self.ops, self.grads, self.out = ops, grads, out     # (the tensors stay alive)
        self.handle = ct.c_void_p()
        ops._call(ops.lib.hwr_gradients_create, len(grads), ops._gradients(grads, out),
                  ct.byref(self.handle))

    def close(self):
        if self.handle and self.ops.ctx:
            self.ops.lib.hwr_gradients_destroy(self.ops.ctx, self.handle)
        self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Operators:
    def __init__(self, stream=None):
        import torch
        self.torch = torch
        self.lib = load_ops()
        self.ctx = None
        if not torch.cuda.is_available():
            raise RuntimeError("no CUDA device")
        self.device = torch.device("cuda", torch.cuda.current_device())
        self.stream = torch.cuda.current_stream() if stream is None else stream
        self._raw = self.stream.cuda_stream
        self._current = torch._C._cuda_getCurrentRawStream
        self._dtypes = {torch.bfloat16: HWR_BF16, torch.float16: HWR_F16}
        self._grad_dtypes = dict(self._dtypes) | {torch.float32: HWR_F32}
        ctx = ct.c_void_p()
        # the legacy default stream has the handle 1 (0 would ask for a new one)
        st = self.lib.hwr_ops_create(self._raw or 1, ct.byref(ctx))
        if st != HWR_OK:
            raise HwrError(st, self.lib.hwr_ops_last_error(None).decode())
        self.ctx = ctx
        self._rows, self._adapters = hwr_rows(), hwr_adapters()
        self._rows_ref, self._adapters_ref = ct.byref(self._rows), ct.byref(self._adapters)

    # ---- helpers -------------------------------------------------------------

    def _call(self, fn, *args):
        if self.ctx is None:
            raise RuntimeError("the context is closed")
        current = self._current(self.device.index)
        if current == self._raw:
            st = fn(self.ctx, *args)
        else:
            other = self.torch.cuda.current_stream(self.device)
            self.stream.wait_stream(other)
            st = fn(self.ctx, *args)
            other.wait_stream(self.stream)
        if st != HWR_OK:
            raise HwrError(st, self.lib.hwr_ops_last_error(self.ctx).decode())

    def _matrix(self, t, name, shape, dtype):
        """Checks a tensor and returns its address and its row's stride."""
        if t.shape != shape:
            raise ValueError(f"{name}: shape {tuple(t.shape)}, want {tuple(shape)}")
        if t.dtype is not dtype:
            raise TypeError(f"{name}: {t.dtype}, want {dtype}")
        if t.device != self.device:
            raise ValueError(f"{name} is on {t.device}, the context on {self.device}")
        st = t.stride()
        if st[-1] != 1 and shape[-1] != 1:
            raise ValueError(f"{name}: the last dimension is not contiguous")
        ld = st[-2]
        if ld < shape[-1]:                   # one row, or rows that overlap
            if shape[-2] > 1:
                raise ValueError(f"{name}: overlapping rows")
            ld = shape[-1]
        return t.data_ptr(), ld

    def _fill(self, x, w, plan, x_name, x_width, w_shape, with_x=True):
        """The call's hwr_rows from its tensors."""
        dt = x.dtype
        code = self._dtypes.get(dt)
        if code is None:
            raise TypeError(f"{x_name}: {dt}, want bfloat16 or float16")
        r = self._rows
        r.rows, r.groups, r.dtype = plan.rows, plan.groups, code
        r.n_out, r.n_in = w_shape[-2], w_shape[-1]
        r.offsets, r.order = plan._po, plan._pr
        if w.dim() != len(w_shape):
            raise ValueError(f"w has {w.dim()} dimensions, want {len(w_shape)}")
        r.w, r.w_ld = self._matrix(w, "w", w_shape, dt)
        r.w_group = w.stride(0) if len(w_shape) == 3 else 0
        if len(w_shape) == 3 and w_shape[0] == 1:
            r.w_group = r.w_ld * w_shape[1]
        return dt

    def _out(self, out, name, rows, width, like):
        if out is None:
            out = like.new_empty((rows, width))
            return out, out.data_ptr(), width
        return (out, *self._matrix(out, name, (rows, width), like.dtype))

    # ---- operators -------------------------------------------------------------

    def dispatch(self, choice, groups: int) -> Plan:
        """Bring the rows of each choice together.  ``choice`` [rows] int32;
        values outside [0, groups) are rows without a choice."""
        torch = self.torch
        if choice.dtype is not torch.int32 or choice.dim() != 1 or not choice.is_contiguous():
            raise TypeError("choice: want a contiguous int32 vector")
        if choice.device != self.device:
            raise ValueError(f"choice is on {choice.device}, the context on {self.device}")
        n, g = choice.numel(), int(groups)
        if g < 1:
            raise ValueError(f"groups {g}")
        both = choice.new_empty(g + 1 + n)
        p = both.data_ptr()
        self._call(self.lib.hwr_dispatch, n, g, choice.data_ptr(), p, p + 4 * (g + 1))
        return Plan(both[:g + 1], both[g + 1:])

    def grouped_forward(self, x, w, plan: Plan, out=None):
        """y[t] = w[c] x[t] for x [rows][K], w [groups][N][K] -> [rows][N];
        rows without a choice get zeros."""
        if w.dim() != 3:
            raise ValueError("w: want [groups][N][K]")
        _, N, K = w.shape
        self._fill(x, w, plan, "x", K, (plan.groups, N, K))
        r = self._rows
        r.x, r.x_ld = self._matrix(x, "x", (plan.rows, K), x.dtype)
        y, p, ld = self._out(out, "out", plan.rows, N, x)
        self._call(self.lib.hwr_grouped_forward, self._rows_ref, p, ld)
        return y

    def grouped_backward(self, dy, x, w, plan: Plan, need_dx=True, need_dw=True):
        """(dx [rows][K], dw like w) from dy [rows][N]; None where not asked for."""
        if w.dim() != 3:
            raise ValueError("w: want [groups][N][K]")
        _, N, K = w.shape
        dt = self._fill(dy, w, plan, "dy", N, (plan.groups, N, K))
        r = self._rows
        r.x, r.x_ld = self._matrix(x, "x", (plan.rows, K), dt)
        d, d_ld = self._matrix(dy, "dy", (plan.rows, N), dt)
        dx = dy.new_empty((plan.rows, K)) if need_dx else None
        dw = None
        if need_dw:
            # laid out as w
            dw = w.new_empty_strided(w.shape, (r.w_group, r.w_ld, 1))
        self._call(self.lib.hwr_grouped_backward, self._rows_ref, d, d_ld,
                   dx.data_ptr() if need_dx else None, K, dw.data_ptr() if need_dw else None)
        return dx, dw

    def _low_rank(self, x, a, b, scale, plan, N, K):
        if a.dim() != 3:
            raise ValueError("a: want [groups][rank][K]")
        R = a.shape[1]
        for t, name, shape in ((a, "a", (plan.groups, R, K)), (b, "b", (plan.groups, N, R))):
            if t.shape != shape:
                raise ValueError(f"{name}: shape {tuple(t.shape)}, want {shape}")
            if t.dtype is not x.dtype:
                raise TypeError(f"{name}: {t.dtype}, want {x.dtype}")
            if t.device != self.device or not t.is_contiguous():
                raise ValueError(f"{name}: want a contiguous tensor on {self.device}")
        if (scale.dtype is not self.torch.float32 or scale.shape != (plan.groups,)
                or scale.device != self.device or not scale.is_contiguous()):
            raise ValueError(f"scale: want {plan.groups} contiguous float32 on {self.device}")
        ad = self._adapters
        ad.rank, ad.a, ad.b, ad.scale = R, a.data_ptr(), b.data_ptr(), scale.data_ptr()

    def adapter_forward(self, x, w, a, b, scale, plan: Plan, out=None):
        """y[t] = w x[t] + scale[c] b[c] (a[c] x[t]) for w [N][K],
        a [groups][rank][K], b [groups][N][rank], scale [groups] fp32; rows
        without a choice get w x[t]."""
        N, K = w.shape
        self._fill(x, w, plan, "x", K, (N, K))
        self._low_rank(x, a, b, scale, plan, N, K)
        r = self._rows
        r.x, r.x_ld = self._matrix(x, "x", (plan.rows, K), x.dtype)
        y, p, ld = self._out(out, "out", plan.rows, N, x)
        self._call(self.lib.hwr_adapter_forward, self._rows_ref, self._adapters_ref, p, ld)
        return y

    def adapter_backward(self, dy, x, w, a, b, scale, plan: Plan, need_dx=True, need_dab=True):
        """(dx, da, db) of ``adapter_forward`` from dy [rows][N] (the shared
        projection is not trained); None where not asked for."""
        N, K = w.shape
        dt = self._fill(dy, w, plan, "dy", N, (N, K))
        self._low_rank(dy, a, b, scale, plan, N, K)
        r = self._rows
        r.x, r.x_ld = self._matrix(x, "x", (plan.rows, K), dt)
        d, d_ld = self._matrix(dy, "dy", (plan.rows, N), dt)
        dx = dy.new_empty((plan.rows, K)) if need_dx else None
        da = a.new_empty(a.shape) if need_dab else None
        db = b.new_empty(b.shape) if need_dab else None
        self._call(self.lib.hwr_adapter_backward, self._rows_ref, self._adapters_ref, d, d_ld,
                   dx.data_ptr() if need_dx else None, K,
                   da.data_ptr() if need_dab else None, db.data_ptr() if need_dab else None)
        return dx, da, db

    def _gradients(self, grads, out):
        if len(out) != len(grads):
            raise ValueError(f"{len(out)} outputs for {len(grads)} gradients")
        table = (hwr_gradient * max(1, len(grads)))()
        for e, g, o in zip(table, grads, out):
            code = self._grad_dtypes.get(g.dtype)
            if code is None:
                raise TypeError(f"gradient: {g.dtype}, want float32, bfloat16 or float16")
            if o.dtype is not g.dtype or o.shape != g.shape:
                raise ValueError("an output differs from its gradient in shape or type")
            for t in (g, o):
                if t.device != self.device or not t.is_contiguous():
                    raise ValueError(f"want contiguous gradients on {self.device}")
            e.in_, e.out, e.n, e.dtype = g.data_ptr(), o.data_ptr(), g.numel(), code
        return table

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
        norm = self.torch.empty((), dtype=self.torch.float32, device=self.device)
        if isinstance(grads, GradientList):
            if out is not None or grads.ops is not self or not grads.handle:
                raise ValueError("a gradient list has its outputs, its context, and is open")
            self._call(self.lib.hwr_gradients_clip, grads.handle, float(max_norm), norm.data_ptr())
        else:
            grads = list(grads)
            self._call(self.lib.hwr_clip_gradients, len(grads),
                       self._gradients(grads, grads if out is None else list(out)),
                       float(max_norm), norm.data_ptr())
        return norm

    def reserve(self, nbytes: int):
        """Make the workspace at least ``nbytes`` large (before a stream capture)."""
        self._call(self.lib.hwr_ops_reserve, int(nbytes))

    def synchronize(self):
        self._call(self.lib.hwr_ops_synchronize)

    def close(self):
        if getattr(self, "ctx", None):
            self.lib.hwr_ops_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
