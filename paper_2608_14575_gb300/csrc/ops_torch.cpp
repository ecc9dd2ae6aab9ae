// Torch binding of the operators in hwr_ops.h: checks the tensors of a call,
// allocates its outputs and makes the call.  Written against torch's C++ API
// because a small call's own time is that of its binding: with the checks in
// Python, a dispatch of 64 rows took 14.5 us of the host, its kernel 3.
//
// Exceptions do not leave a function: they become Python errors.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_strided.h>
#include <torch/csrc/autograd/python_variable.h>

#include <stdexcept>
#include <string>
#include <vector>

#include "hwr_ops.h"

namespace {

struct TypeError : std::runtime_error {
    using std::runtime_error::runtime_error;
};
struct ValueError : std::runtime_error {
    using std::runtime_error::runtime_error;
};
struct StatusError : std::runtime_error {
    hwr_status status;
    StatusError(hwr_status s, const char *text) : std::runtime_error(text), status(s) {}
};
struct PythonError {};      // an error that is already set

struct Context {
    hwr_ops *ops = nullptr;
    int device = 0;
    void *stream = nullptr;      // torch's handle (null: the default stream)
};

PyObject *g_hwr_error = nullptr;      // the package's HwrError

template <class F>
PyObject *guarded(F f) {
    try {
        return f();
    } catch (const TypeError &e) {
        PyErr_SetString(PyExc_TypeError, e.what());
    } catch (const ValueError &e) {
        PyErr_SetString(PyExc_ValueError, e.what());
    } catch (const StatusError &e) {
        PyObject *args = Py_BuildValue("(is)", (int)e.status, e.what());
        PyObject *err = args ? PyObject_CallObject(g_hwr_error, args) : nullptr;
        Py_XDECREF(args);
        if (err) {
            PyErr_SetObject(g_hwr_error, err);
            Py_DECREF(err);
        }
    } catch (const PythonError &) {
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
    }
    return nullptr;
}

void want(Py_ssize_t n, Py_ssize_t k) {
    if (n != k) throw TypeError("wrong number of arguments");
}

Context &context(PyObject *o) {
    Context *c = (Context *)PyLong_AsVoidPtr(o);
    if (PyErr_Occurred()) throw PythonError();
    if (!c) throw std::runtime_error("the context is closed");
    return *c;
}

void *address(PyObject *o) {
    void *p = PyLong_AsVoidPtr(o);
    if (PyErr_Occurred()) throw PythonError();
    return p;
}

bool truth(PyObject *o) {
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw PythonError();
    return v != 0;
}

double number(PyObject *o) {
    const double v = PyFloat_AsDouble(o);
    if (PyErr_Occurred()) throw PythonError();
    return v;
}

const at::Tensor &tensor(PyObject *o, const char *name) {
    if (!THPVariable_Check(o)) throw TypeError(std::string(name) + ": want a tensor");
    return THPVariable_Unpack(o);
}

std::string shape_of(at::IntArrayRef s) {
    std::string t = "[";
    for (size_t i = 0; i < s.size(); ++i) t += (i ? ", " : "") + std::to_string(s[i]);
    return t + "]";
}

void on_device(const Context &c, const at::Tensor &t, const char *name) {
    if (!t.is_cuda() || t.get_device() != c.device)
        throw ValueError(std::string(name) + " is not on the context's device");
}

void shaped(const at::Tensor &t, at::IntArrayRef shape, const char *name) {
    if (t.sizes() != shape)
        throw ValueError(std::string(name) + ": shape " + shape_of(t.sizes()) + ", want " + shape_of(shape));
}

void typed(const at::Tensor &t, at::ScalarType dtype, const char *name) {
    if (t.scalar_type() != dtype)
        throw TypeError(std::string(name) + ": " + c10::toString(t.scalar_type()) + ", want " + c10::toString(dtype));
}

int narrow(int64_t v, const char *what) {
    if (v > INT32_MAX) throw StatusError(HWR_ERR_UNSUPPORTED, (std::string(what) + " beyond 32 bits").c_str());
    return (int)v;
}

// A matrix (the last two dimensions) whose rows are contiguous: its row stride.
int64_t rows_stride(const Context &c, const at::Tensor &t, at::IntArrayRef shape, at::ScalarType dtype,
                    const char *name) {
    shaped(t, shape, name);
    typed(t, dtype, name);
    on_device(c, t, name);
    const auto st = t.strides();
    const size_t d = shape.size();
    if (st[d - 1] != 1 && shape[d - 1] != 1) throw ValueError(std::string(name) + ": the last dimension is not contiguous");
    if (st[d - 2] >= shape[d - 1]) return st[d - 2];
    if (shape[d - 2] > 1) throw ValueError(std::string(name) + ": overlapping rows");
    return shape[d - 1];
}

const void *contiguous(const Context &c, const at::Tensor &t, at::IntArrayRef shape, at::ScalarType dtype,
                       const char *name) {
    shaped(t, shape, name);
    typed(t, dtype, name);
    on_device(c, t, name);
    if (!t.is_contiguous()) throw ValueError(std::string(name) + ": want a contiguous tensor");
    return t.data_ptr();
}

hwr_dtype sixteen(const at::Tensor &t, const char *name) {
    if (t.scalar_type() == at::kBFloat16) return HWR_BF16;
    if (t.scalar_type() == at::kHalf) return HWR_F16;
    throw TypeError(std::string(name) + ": " + c10::toString(t.scalar_type()) + ", want bfloat16 or float16");
}

// The call, ordered after the current stream's work and that stream after it,
// where it is not the context's own; also when it fails (part of its work may be
// queued, and the caller's memory goes back to the current stream).
template <class F>
void call(Context &c, PyObject *raw, F f) {
    void *current = address(raw);
    const bool other = current != c.stream;
    auto check = [&](hwr_status s) {
        if (s != HWR_OK) throw StatusError(s, hwr_ops_last_error(c.ops));
    };
    if (other) check(hwr_ops_after(c.ops, current ? current : (void *)1));
    const hwr_status s = f();
    if (s != HWR_OK) {
        const StatusError error(s, hwr_ops_last_error(c.ops));
        if (other) hwr_ops_before(c.ops, current ? current : (void *)1);
        throw error;
    }
    if (other) check(hwr_ops_before(c.ops, current ? current : (void *)1));
}

// Tell autograd that the call has written a tensor of the caller's.
void written(const at::Tensor &t) {
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

void all_written(PyObject *list) {
    for (Py_ssize_t i = 0; i < PyList_GET_SIZE(list); ++i) written(tensor(PyList_GET_ITEM(list, i), "output"));
}

PyObject *wrap(at::Tensor t) {
    PyObject *o = THPVariable_Wrap(std::move(t));
    if (!o) throw PythonError();
    return o;
}

PyObject *wrap_or_none(at::Tensor t) {
    if (!t.defined()) Py_RETURN_NONE;
    return wrap(std::move(t));
}

PyObject *tuple(std::initializer_list<at::Tensor> ts) {
    PyObject *p = PyTuple_New((Py_ssize_t)ts.size());
    if (!p) throw PythonError();
    Py_ssize_t i = 0;
    for (const at::Tensor &t : ts) {
        PyObject *o;
        try {
            o = wrap_or_none(t);
        } catch (...) {
            Py_DECREF(p);
            throw;
        }
        PyTuple_SET_ITEM(p, i++, o);
    }
    return p;
}

// ---- calls: (context, current stream, ...) -------------------------------------

PyObject *create(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&] {
        want(n, 2);
        Context *c = new Context;
        c->stream = address(a[0]);
        c->device = (int)PyLong_AsLong(a[1]);
        // the legacy default stream has the handle 1 (null would ask for a new one)
        const hwr_status s = hwr_ops_create(c->stream ? c->stream : (void *)1, &c->ops);
        if (s != HWR_OK) {
            delete c;
            throw StatusError(s, hwr_ops_last_error(nullptr));
        }
        return PyLong_FromVoidPtr(c);
    });
}

PyObject *destroy(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        want(n, 1);
        Context &c = context(a[0]);
        hwr_ops_destroy(c.ops);
        delete &c;
        Py_RETURN_NONE;
    });
}

PyObject *synchronize(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        want(n, 1);
        Context &c = context(a[0]);
        hwr_status s;
        Py_BEGIN_ALLOW_THREADS
        s = hwr_ops_synchronize(c.ops);
        Py_END_ALLOW_THREADS
        if (s != HWR_OK) throw StatusError(s, hwr_ops_last_error(c.ops));
        Py_RETURN_NONE;
    });
}

PyObject *reserve(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        want(n, 3);
        Context &c = context(a[0]);
        const unsigned long long bytes = PyLong_AsUnsignedLongLong(a[2]);
        if (PyErr_Occurred()) throw PythonError();
        call(c, a[1], [&] { return hwr_ops_reserve(c.ops, bytes); });
        Py_RETURN_NONE;
    });
}

// choice, groups -> (offsets, order)
PyObject *dispatch(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&] {
        want(n, 4);
        Context &c = context(a[0]);
        const at::Tensor &choice = tensor(a[2], "choice");
        const long long groups = PyLong_AsLongLong(a[3]);
        if (PyErr_Occurred()) throw PythonError();
        if (choice.scalar_type() != at::kInt || choice.dim() != 1 || !choice.is_contiguous())
            throw TypeError("choice: want a contiguous int32 vector");
        on_device(c, choice, "choice");
        if (groups < 1) throw ValueError("groups " + std::to_string(groups));
        const int rows = narrow(choice.numel(), "rows"), g = narrow(groups, "groups");
        if (g > HWR_OPS_MAX_GROUPS)
            throw StatusError(HWR_ERR_UNSUPPORTED, ("groups " + std::to_string(g) + " > " + std::to_string(HWR_OPS_MAX_GROUPS)).c_str());
        at::Tensor offsets = at::empty({g + 1}, choice.options()), order = at::empty({rows}, choice.options());
        call(c, a[1], [&] {
            return hwr_dispatch(c.ops, rows, g, (const int32_t *)choice.data_ptr(), (int32_t *)offsets.data_ptr(),
                                (int32_t *)order.data_ptr());
        });
        return tuple({offsets, order});
    });
}

// The plan's part of a call.
void fill_plan(const Context &c, hwr_rows &r, PyObject *offsets, PyObject *order) {
    const at::Tensor &o = tensor(offsets, "offsets"), &p = tensor(order, "order");
    r.rows = narrow(p.numel(), "rows");
    r.groups = narrow(o.numel() - 1, "groups");
    r.offsets = (const int32_t *)contiguous(c, o, {o.numel()}, at::kInt, "offsets");
    r.order = (const int32_t *)contiguous(c, p, {p.numel()}, at::kInt, "order");
}

// w [groups][N][K] or [N][K] into the call.
void fill_weights(const Context &c, hwr_rows &r, const at::Tensor &w, at::ScalarType dtype, bool grouped) {
    if (w.dim() != (grouped ? 3 : 2)) throw ValueError(grouped ? "w: want [groups][N][K]" : "w: want [N][K]");
    const int64_t N = w.size(-2), K = w.size(-1);
    r.n_out = narrow(N, "n_out");
    r.n_in = narrow(K, "n_in");
    r.w_ld = grouped ? rows_stride(c, w, {r.groups, N, K}, dtype, "w") : rows_stride(c, w, {N, K}, dtype, "w");
    r.w_group = grouped ? (r.groups > 1 ? w.stride(0) : r.w_ld * N) : 0;
    r.w = w.data_ptr();
}

at::Tensor output(const Context &c, PyObject *given, int64_t rows, int64_t width, const at::Tensor &like,
                  int64_t *ld) {
    if (given == Py_None) {
        *ld = width;
        return at::empty({rows, width}, like.options());
    }
    const at::Tensor &t = tensor(given, "out");
    *ld = rows_stride(c, t, {rows, width}, like.scalar_type(), "out");
    return t;
}

// x, w, offsets, order, out
PyObject *grouped_forward(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&] {
        want(n, 7);
        Context &c = context(a[0]);
        const at::Tensor &x = tensor(a[2], "x"), &w = tensor(a[3], "w");
        hwr_rows r = {};
        r.dtype = sixteen(x, "x");
        fill_plan(c, r, a[4], a[5]);
        fill_weights(c, r, w, x.scalar_type(), true);
        r.x_ld = rows_stride(c, x, {r.rows, r.n_in}, x.scalar_type(), "x");
        r.x = x.data_ptr();
        int64_t ld;
        at::Tensor y = output(c, a[6], r.rows, r.n_out, x, &ld);
        call(c, a[1], [&] { return hwr_grouped_forward(c.ops, &r, y.data_ptr(), ld); });
        if (a[6] != Py_None) written(y);
        return wrap(std::move(y));
    });
}

// dy, x, w, offsets, order, need_dx, need_dw
PyObject *grouped_backward(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&] {
        want(n, 9);
        Context &c = context(a[0]);
        const at::Tensor &dy = tensor(a[2], "dy"), &x = tensor(a[3], "x"), &w = tensor(a[4], "w");
        hwr_rows r = {};
        r.dtype = sixteen(dy, "dy");
        fill_plan(c, r, a[5], a[6]);
        fill_weights(c, r, w, dy.scalar_type(), true);
        r.x_ld = rows_stride(c, x, {r.rows, r.n_in}, dy.scalar_type(), "x");
        r.x = x.data_ptr();
        const int64_t dy_ld = rows_stride(c, dy, {r.rows, r.n_out}, dy.scalar_type(), "dy");
        at::Tensor dx, dw;
        if (truth(a[7])) dx = at::empty({r.rows, r.n_in}, dy.options());
        if (truth(a[8])) dw = at::empty_strided(w.sizes(), {r.w_group, r.w_ld, 1}, w.options());     // laid out as w
        call(c, a[1], [&] {
            return hwr_grouped_backward(c.ops, &r, dy.data_ptr(), dy_ld, dx.defined() ? dx.data_ptr() : nullptr,
                                        r.n_in, dw.defined() ? dw.data_ptr() : nullptr);
        });
        return tuple({dx, dw});
    });
}

hwr_adapters fill_adapters(const Context &c, const hwr_rows &r, at::ScalarType dtype, const at::Tensor &a,
                           const at::Tensor &b, const at::Tensor &scale) {
    if (a.dim() != 3) throw ValueError("a: want [groups][rank][K]");
    hwr_adapters ad = {};
    const int64_t R = a.size(1);
    ad.rank = narrow(R, "rank");
    ad.a = contiguous(c, a, {r.groups, R, r.n_in}, dtype, "a");
    ad.b = contiguous(c, b, {r.groups, r.n_out, R}, dtype, "b");
    if (scale.scalar_type() != at::kFloat) throw ValueError("scale: want float32");
    ad.scale = (const float *)contiguous(c, scale, {r.groups}, at::kFloat, "scale");
    return ad;
}

// x, w, a, b, scale, offsets, order, out
PyObject *adapter_forward(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&] {
        want(n, 10);
        Context &c = context(a[0]);
        const at::Tensor &x = tensor(a[2], "x"), &w = tensor(a[3], "w");
        hwr_rows r = {};
        r.dtype = sixteen(x, "x");
        fill_plan(c, r, a[7], a[8]);
        fill_weights(c, r, w, x.scalar_type(), false);
        const hwr_adapters ad = fill_adapters(c, r, x.scalar_type(), tensor(a[4], "a"), tensor(a[5], "b"), tensor(a[6], "scale"));
        r.x_ld = rows_stride(c, x, {r.rows, r.n_in}, x.scalar_type(), "x");
        r.x = x.data_ptr();
        int64_t ld;
        at::Tensor y = output(c, a[9], r.rows, r.n_out, x, &ld);
        call(c, a[1], [&] { return hwr_adapter_forward(c.ops, &r, &ad, y.data_ptr(), ld); });
        if (a[9] != Py_None) written(y);
        return wrap(std::move(y));
    });
}

// dy, x, w, a, b, scale, offsets, order, need_dx, need_dab
PyObject *adapter_backward(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&] {
        want(n, 12);
        Context &c = context(a[0]);
        const at::Tensor &dy = tensor(a[2], "dy"), &x = tensor(a[3], "x"), &w = tensor(a[4], "w");
        const at::Tensor &A = tensor(a[5], "a"), &B = tensor(a[6], "b");
        hwr_rows r = {};
        r.dtype = sixteen(dy, "dy");
        fill_plan(c, r, a[8], a[9]);
        fill_weights(c, r, w, dy.scalar_type(), false);
        const hwr_adapters ad = fill_adapters(c, r, dy.scalar_type(), A, B, tensor(a[7], "scale"));
        r.x_ld = rows_stride(c, x, {r.rows, r.n_in}, dy.scalar_type(), "x");
        r.x = x.data_ptr();
        const int64_t dy_ld = rows_stride(c, dy, {r.rows, r.n_out}, dy.scalar_type(), "dy");
        at::Tensor dx, da, db;
        if (truth(a[10])) dx = at::empty({r.rows, r.n_in}, dy.options());
        if (truth(a[11])) {
            da = at::empty(A.sizes(), A.options());
            db = at::empty(B.sizes(), B.options());
        }
        call(c, a[1], [&] {
            return hwr_adapter_backward(c.ops, &r, &ad, dy.data_ptr(), dy_ld, dx.defined() ? dx.data_ptr() : nullptr,
                                        r.n_in, da.defined() ? da.data_ptr() : nullptr,
                                        db.defined() ? db.data_ptr() : nullptr);
        });
        return tuple({dx, da, db});
    });
}

// Lists of gradients and of where the clipped ones go.
std::vector<hwr_gradient> gradients(const Context &c, PyObject *grads, PyObject *out) {
    if (!PyList_Check(grads) || !PyList_Check(out)) throw TypeError("want lists of tensors");
    const Py_ssize_t n = PyList_GET_SIZE(grads);
    if (PyList_GET_SIZE(out) != n)
        throw ValueError(std::to_string(PyList_GET_SIZE(out)) + " outputs for " + std::to_string(n) + " gradients");
    std::vector<hwr_gradient> v((size_t)n);
    for (Py_ssize_t i = 0; i < n; ++i) {
        const at::Tensor &g = tensor(PyList_GET_ITEM(grads, i), "gradient"), &o = tensor(PyList_GET_ITEM(out, i), "output");
        hwr_gradient &e = v[(size_t)i];
        switch (g.scalar_type()) {
            case at::kFloat: e.dtype = HWR_F32; break;
            case at::kBFloat16: e.dtype = HWR_BF16; break;
            case at::kHalf: e.dtype = HWR_F16; break;
            default: throw TypeError("gradient: want float32, bfloat16 or float16");
        }
        if (o.scalar_type() != g.scalar_type() || o.sizes() != g.sizes())
            throw ValueError("an output differs from its gradient in shape or type");
        for (const at::Tensor *t : {&g, &o}) {
            on_device(c, *t, "a gradient");
            if (!t->is_contiguous()) throw ValueError("want contiguous gradients");
        }
        e.in = g.data_ptr();
        e.out = o.data_ptr();
        e.n = g.numel();
    }
    return v;
}

at::Tensor scalar(const Context &c) {
    return at::empty({}, at::TensorOptions().dtype(at::kFloat).device(at::kCUDA, (c10::DeviceIndex)c.device));
}

// grads, out, max_norm -> norm
PyObject *clip(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&] {
        want(n, 5);
        Context &c = context(a[0]);
        const std::vector<hwr_gradient> v = gradients(c, a[2], a[3]);
        const float max_norm = (float)number(a[4]);
        const int count = narrow((int64_t)v.size(), "gradients");
        at::Tensor norm = scalar(c);
        call(c, a[1], [&] { return hwr_clip_gradients(c.ops, count, v.data(), max_norm, (float *)norm.data_ptr()); });
        all_written(a[3]);
        return wrap(std::move(norm));
    });
}

// grads, out -> handle
PyObject *list_create(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&] {
        want(n, 4);
        Context &c = context(a[0]);
        const std::vector<hwr_gradient> v = gradients(c, a[2], a[3]);
        const int count = narrow((int64_t)v.size(), "gradients");
        hwr_gradients *l = nullptr;
        call(c, a[1], [&] { return hwr_gradients_create(c.ops, count, v.data(), &l); });
        return PyLong_FromVoidPtr(l);
    });
}

// handle, max_norm, the list's outputs -> norm
PyObject *list_clip(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&] {
        want(n, 5);
        if (!PyList_Check(a[4])) throw TypeError("want a list of tensors");
        Context &c = context(a[0]);
        const hwr_gradients *l = (const hwr_gradients *)address(a[2]);
        const float max_norm = (float)number(a[3]);
        at::Tensor norm = scalar(c);
        call(c, a[1], [&] { return hwr_gradients_clip(c.ops, l, max_norm, (float *)norm.data_ptr()); });
        all_written(a[4]);
        return wrap(std::move(norm));
    });
}

PyObject *list_destroy(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        want(n, 2);
        hwr_gradients_destroy(context(a[0]).ops, (hwr_gradients *)address(a[1]));
        Py_RETURN_NONE;
    });
}

PyObject *set_error(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        want(n, 1);
        Py_XDECREF(g_hwr_error);
        Py_INCREF(a[0]);
        g_hwr_error = a[0];
        Py_RETURN_NONE;
    });
}

#define METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(create), METHOD(destroy), METHOD(synchronize), METHOD(reserve), METHOD(dispatch),
                         METHOD(grouped_forward), METHOD(grouped_backward), METHOD(adapter_forward),
                         METHOD(adapter_backward), METHOD(clip), METHOD(list_create), METHOD(list_clip),
                         METHOD(list_destroy), METHOD(set_error), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "hwr_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_hwr_torch(void) { return PyModule_Create(&module); }
