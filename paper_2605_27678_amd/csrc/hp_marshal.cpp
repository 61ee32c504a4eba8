// The binding's way from lists of torch tensors to one call of the C ABI: checks
// every buffer as binding.py's _pointers does, collects the device pointers and
// makes the call, in one step.  In Python the same took 5 to 6 us a call, more
// than the launch (about 3.5 us) and, for small plans, than the kernel.
//
// call(fn, plan, desc, kind_a, list_a, kind_b, list_b, stream) -> the call's return
// code, or None for anything that is not plainly in order: the caller then goes
// the way through Python, which reports what is wrong (or copes with objects that
// are no plain tensors).  Nothing is kept from one call to the next.
//
// rotary(), norm(), norm_backward() and attend() do the same for the operators of
// operators.py, whose checks they repeat: None for whatever is not plainly in
// order.  In Python they took 11 to 13 us a call.
#include <c10/core/impl/VirtualGuardImpl.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <cstdint>

#include "hp.h"
#include "hp_operators.h"

namespace {

// Filled in once per plan by binding.py (Plan._desc); the same layout there.
struct Desc {
    int64_t n_src, n_dst, dst_rows, hidden, elem_bytes;
    const int64_t *src_rows;
};

enum Kind { kSrc = 0, kDst = 1, kAccum = 2 };     // kAccum: binary32 accumulators in the place of source buffers

typedef int (*Call)(const void *plan, const void *const *a, void *const *b, void *stream);

// The device pointers of a list (or tuple) of tensors; false if any of it is not plainly in order.
bool pointers(PyObject *list, Kind kind, const Desc &d, void **out) {
    const bool is_list = PyList_CheckExact(list);
    if (!is_list && !PyTuple_CheckExact(list)) return false;
    const int64_t n = is_list ? PyList_GET_SIZE(list) : PyTuple_GET_SIZE(list);
    if (n != (kind == kDst ? d.n_dst : d.n_src) || n > HP_MAX_BUFFERS) return false;
    const int64_t elem = kind == kAccum ? 4 : d.elem_bytes;
    for (int64_t i = 0; i < n; ++i) {
        PyObject *o = is_list ? PyList_GET_ITEM(list, i) : PyTuple_GET_ITEM(list, i);
        if (o == Py_None) {
            out[i] = nullptr;
            continue;
        }
        if (!THPVariable_CheckExact(o)) return false;
        const at::Tensor &t = THPVariable_Unpack(o);
        if (t.unsafeGetTensorImpl()->is_python_dispatch() || !t.has_storage()) return false;
        const int64_t rows = kind == kDst ? d.dst_rows : d.src_rows[i];
        if (!t.is_cuda() || !t.is_contiguous() || (int64_t)t.element_size() != elem || t.numel() < rows * d.hidden) return false;
        out[i] = t.numel() ? t.data_ptr() : nullptr;
    }
    return true;
}

// A stream argument: None, an object with a cuda_stream, or a number.
bool stream_of(PyObject *o, void **out) {
    if (o == Py_None) {
        *out = nullptr;
        return true;
    }
    PyObject *v = PyLong_CheckExact(o) ? Py_NewRef(o) : PyObject_GetAttrString(o, "cuda_stream");
    if (v) {
        *out = PyLong_AsVoidPtr(v);
        Py_DECREF(v);
    }
    if (PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    return true;
}

PyObject *call(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    if (n_args != 8) {
        PyErr_SetString(PyExc_TypeError, "call takes 8 arguments");
        return nullptr;
    }
    const Call fn = (Call)PyLong_AsVoidPtr(args[0]);
    const void *plan = PyLong_AsVoidPtr(args[1]);
    const Desc *desc = (const Desc *)PyLong_AsVoidPtr(args[2]);
    const long kind_a = PyLong_AsLong(args[3]), kind_b = PyLong_AsLong(args[5]);
    if (PyErr_Occurred()) return nullptr;
    if (!fn || !plan || !desc) Py_RETURN_NONE;
    void *a[HP_MAX_BUFFERS], *b[HP_MAX_BUFFERS], *stream = nullptr;
    try {
        if (!pointers(args[4], (Kind)kind_a, *desc, a) || !pointers(args[6], (Kind)kind_b, *desc, b) ||
            !stream_of(args[7], &stream))
            Py_RETURN_NONE;
    } catch (const std::exception &) {
        Py_RETURN_NONE;
    }
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = fn(plan, a, b, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// ---- the operators ----------------------------------------------------------------------------------------------

// A call's tensors: all on the current device, and of one element type (the others are named).
struct Checks {
    int device = c10::impl::VirtualGuardImpl(c10::DeviceType::CUDA).getDevice().index();
    at::ScalarType type = at::ScalarType::Undefined;
    bool ok = true;

    // The tensor, if it is a plain one of this type (Undefined: the call's) and number of dimensions with its last
    // dimension contiguous (whole: all of it); NULL and ok = false if not; NULL for None where that is allowed.
    const at::Tensor *take(PyObject *o, int64_t dims, bool whole = false, bool optional = false, at::ScalarType want = at::ScalarType::Undefined) {
        if (optional && o == Py_None) return nullptr;
        if (!ok || !THPVariable_CheckExact(o)) return fail();
        const at::Tensor &t = THPVariable_Unpack(o);
        if (t.unsafeGetTensorImpl()->is_python_dispatch() || !t.has_storage() || !t.is_cuda() || t.get_device() != device) return fail();
        if (want == at::ScalarType::Undefined) {
            if (type == at::ScalarType::Undefined) type = t.scalar_type();
            want = type;
            if (type != at::kBFloat16 && type != at::kFloat) return fail();
        }
        if (t.scalar_type() != want || (dims >= 0 && t.dim() != dims)) return fail();
        if (whole ? !t.is_contiguous() : dims > 0 && t.size(dims - 1) > 1 && t.stride(dims - 1) != 1) return fail();
        return &t;
    }
    const at::Tensor *shaped(PyObject *o, at::IntArrayRef sizes, bool whole = false, bool optional = false, at::ScalarType want = at::ScalarType::Undefined) {
        const at::Tensor *t = take(o, (int64_t)sizes.size(), whole, optional, want);
        return t && t->sizes() != sizes ? fail() : t;
    }
    const at::Tensor *fail() {
        ok = false;
        return nullptr;
    }
    int32_t dtype() const { return type == at::kFloat ? HP_F32 : HP_BF16; }
};

void *at_of(const at::Tensor *t) { return t && t->numel() ? t->data_ptr() : nullptr; }
hp_heads_t heads_of(const at::Tensor *t) { return t ? hp_heads_t{at_of(t), t->stride(0), t->stride(1)} : hp_heads_t{}; }

// Scratch memory: any contiguous tensor, or None.
bool scratch_of(PyObject *o, const Checks &c, void **at, int64_t *bytes) {
    *at = nullptr, *bytes = 0;
    if (o == Py_None) return true;
    if (!THPVariable_CheckExact(o)) return false;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (t.unsafeGetTensorImpl()->is_python_dispatch() || !t.has_storage() || !t.is_cuda() || t.get_device() != c.device || !t.is_contiguous()) return false;
    *at = at_of(&t);
    *bytes = t.numel() * (int64_t)t.element_size();
    return true;
}

// An operator's function: `n` arguments, a body that fills in the call; its code, or None.
template <class Body> PyObject *operate(PyObject *const *args, Py_ssize_t got, Py_ssize_t n, const Body &body) {
    if (got != n) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return nullptr;
    }
    void *fn = PyLong_AsVoidPtr(args[0]), *stream = nullptr;
    if (PyErr_Occurred()) return nullptr;
    int rc = 0;
    try {
        if (!fn || !stream_of(args[n - 1], &stream) || !body(fn, stream, &rc)) {
            if (PyErr_Occurred()) PyErr_Clear();
            Py_RETURN_NONE;
        }
    } catch (const std::exception &) {
        Py_RETURN_NONE;
    }
    return PyLong_FromLong(rc);
}

template <class F> int without_gil(const F &f) {
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f();
    Py_END_ALLOW_THREADS
    return rc;
}

// A list's or a tuple's entries, at most `cap`; -1 for anything else.
int entries(PyObject *list, PyObject **out, int cap) {
    const bool is_list = PyList_CheckExact(list);
    if (!is_list && !PyTuple_CheckExact(list)) return -1;
    const Py_ssize_t n = is_list ? PyList_GET_SIZE(list) : PyTuple_GET_SIZE(list);
    if (n > cap) return -1;
    for (Py_ssize_t i = 0; i < n; ++i) out[i] = is_list ? PyList_GET_ITEM(list, i) : PyTuple_GET_ITEM(list, i);
    return (int)n;
}

// An object that is neither leaves Python's error set.
bool truth(PyObject *o) { return PyObject_IsTrue(o) > 0; }

// rotary(fn, xs, outs, table, positions, interleaved, inverse, sections, stream)
PyObject *rotary(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    return operate(args, n_args, 9, [&](void *fn, void *stream, int *rc) {
        Checks c;
        hp_rotary_args_t a{};
        PyObject *xs[HP_ROTARY_MAX_TENSORS], *outs[HP_ROTARY_MAX_TENSORS], *sections[HP_ROTARY_MAX_AXES];
        a.n_tensors = entries(args[1], xs, HP_ROTARY_MAX_TENSORS);
        if (a.n_tensors < 1 || entries(args[2], outs, HP_ROTARY_MAX_TENSORS) != a.n_tensors) return false;
        for (int i = 0; i < a.n_tensors; ++i) {
            const at::Tensor *x = c.take(xs[i], 3);
            if (!x || (i && (x->size(0) != a.rows || x->size(2) != a.dim)) || x->size(1) > INT32_MAX || x->size(2) > INT32_MAX) return false;
            const at::Tensor *o = c.shaped(outs[i], x->sizes());
            if (!o) return false;
            a.rows = x->size(0), a.dim = (int32_t)x->size(2);
            a.heads[i] = (int32_t)x->size(1);
            a.x[i] = heads_of(x), a.out[i] = heads_of(o);
        }
        const at::Tensor *table = c.take(args[3], 3, true, false, at::kFloat);
        if (!table || table->size(2) != 2 || table->size(1) > (1 << 20)) return false;
        a.rot = 2 * (int32_t)table->size(1), a.table = (const float *)at_of(table), a.table_rows = table->size(0);
        a.n_axes = 1;
        if (args[7] != Py_None) {
            a.n_axes = entries(args[7], sections, HP_ROTARY_MAX_AXES);
            if (a.n_axes < 1) return false;
            int64_t sum = 0;
            for (int i = 0; i < a.n_axes; ++i) {
                const long v = PyLong_AsLong(sections[i]);
                if (PyErr_Occurred() || v < 0 || v > (1 << 20)) return false;
                sum += a.sections[i] = (int32_t)v;
            }
            if (sum != table->size(1)) return false;
        }
        const int64_t each[2] = {a.n_axes, a.rows};
        const at::Tensor *pos = args[7] == Py_None ? c.shaped(args[4], at::IntArrayRef(each + 1, 1), false, false, at::kInt)
                                                   : c.shaped(args[4], at::IntArrayRef(each, 2), false, false, at::kInt);
        if (!pos) return false;
        if (args[7] != Py_None) a.axis_stride = pos->stride(0);
        a.positions = (const int32_t *)at_of(pos);
        a.dtype = c.dtype(), a.interleaved = truth(args[5]), a.inverse = truth(args[6]);
        if (PyErr_Occurred()) return false;
        *rc = without_gil([&] { return ((int (*)(const hp_rotary_args_t *, void *))fn)(&a, stream); });
        return true;
    });
}

// x, y, w_post, gate, w_pre, gate_tanh, residual_scale, unit_offset, eps, rstd
constexpr int kNormArgs = 10;
bool norm_args(PyObject *const *p, Checks &c, hp_norm_args_t *a) {
    const at::Tensor *x = c.take(p[0], 2);
    if (!x || x->size(1) > INT32_MAX) return false;
    a->rows = x->size(0), a->hidden = (int32_t)x->size(1), a->x = at_of(x), a->x_stride = x->stride(0);
    const at::Tensor *y = c.shaped(p[1], x->sizes(), false, true), *w1 = c.shaped(p[2], x->sizes().slice(1), true, true);
    const at::Tensor *gate = c.take(p[3], 1, true, true), *w2 = c.shaped(p[4], x->sizes().slice(1), true, true);
    const int64_t lines[2] = {2, a->rows};
    const at::Tensor *rstd = c.shaped(p[9], at::IntArrayRef(lines, 2), true, true, at::kFloat);
    if (!c.ok || (gate && (gate->numel() < 1 || gate->numel() > INT32_MAX))) return false;
    if (y) a->y = at_of(y), a->y_stride = y->stride(0);
    a->w_post = at_of(w1), a->gate = at_of(gate), a->w_pre = at_of(w2), a->rstd = (float *)at_of(rstd);
    a->gate_size = gate ? (int32_t)gate->numel() : 0;
    a->gate_tanh = truth(p[5]), a->unit_offset = truth(p[7]);
    a->residual_scale = (float)PyFloat_AsDouble(p[6]), a->eps = (float)PyFloat_AsDouble(p[8]);
    a->dtype = c.dtype();
    return !PyErr_Occurred();
}

// norm(fn, <norm args>, h, z, stream)
PyObject *norm(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    return operate(args, n_args, kNormArgs + 4, [&](void *fn, void *stream, int *rc) {
        Checks c;
        hp_norm_args_t a{};
        if (!norm_args(args + 1, c, &a)) return false;
        const at::IntArrayRef sizes = THPVariable_Unpack(args[1]).sizes();
        const at::Tensor *h = c.shaped(args[kNormArgs + 1], sizes, false, true), *z = c.shaped(args[kNormArgs + 2], sizes, false, true);
        if (!c.ok) return false;
        if (h) a.h = at_of(h), a.h_stride = h->stride(0);
        if (z) a.z = at_of(z), a.z_stride = z->stride(0);
        *rc = without_gil([&] { return ((int (*)(const hp_norm_args_t *, void *))fn)(&a, stream); });
        return true;
    });
}

// norm_backward(fn, <norm args>, dh, dz, dx, dy, dw_post, dgate, dw_pre, workspace, stream)
PyObject *norm_backward(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    return operate(args, n_args, kNormArgs + 10, [&](void *fn, void *stream, int *rc) {
        Checks c;
        hp_norm_args_t a{};
        hp_norm_grads_t g{};
        if (!norm_args(args + 1, c, &a)) return false;
        PyObject *const *p = args + kNormArgs + 1;
        const at::IntArrayRef sizes = THPVariable_Unpack(args[1]).sizes();
        const at::Tensor *t[4];
        for (int i = 0; i < 4; ++i) t[i] = c.shaped(p[i], sizes, false, true);
        // a weight's gradient has the weight's shape; one without a weight is for the way through Python to refuse
        if ((p[4] != Py_None && !a.w_post) || (p[5] != Py_None && !a.gate) || (p[6] != Py_None && !a.w_pre)) return false;
        const int64_t gate[1] = {a.gate_size};
        const at::Tensor *w1 = c.shaped(p[4], sizes.slice(1), true, true), *dg = c.shaped(p[5], at::IntArrayRef(gate, 1), true, true);
        const at::Tensor *w2 = c.shaped(p[6], sizes.slice(1), true, true);
        if (!c.ok || !scratch_of(p[7], c, &g.workspace, &g.workspace_bytes)) return false;
        if (t[0]) g.dh = at_of(t[0]), g.dh_stride = t[0]->stride(0);
        if (t[1]) g.dz = at_of(t[1]), g.dz_stride = t[1]->stride(0);
        if (t[2]) g.dx = at_of(t[2]), g.dx_stride = t[2]->stride(0);
        if (t[3]) g.dy = at_of(t[3]), g.dy_stride = t[3]->stride(0);
        g.dw_post = at_of(w1), g.dgate = at_of(dg), g.dw_pre = at_of(w2);
        *rc = without_gil([&] { return ((int (*)(const hp_norm_args_t *, const hp_norm_grads_t *, void *))fn)(&a, &g, stream); });
        return true;
    });
}

// attend(fn, q, k, v, ranges, out, lse, scale, workspace, grads, stream); grads: None or (dout, dq, dk, dv)
PyObject *attend(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    return operate(args, n_args, 11, [&](void *fn, void *stream, int *rc) {
        Checks c;
        hp_attend_args_t a{};
        const at::Tensor *q = c.take(args[1], 3), *k = c.take(args[2], 3);
        if (!q || !k || k->size(2) != q->size(2)) return false;
        const int64_t pairs[2] = {q->size(0), 2};
        const at::Tensor *v = c.shaped(args[3], k->sizes()), *out = c.shaped(args[5], q->sizes());
        const at::Tensor *ranges = c.shaped(args[4], at::IntArrayRef(pairs, 2), true, true, at::kInt);
        const at::Tensor *lse = c.shaped(args[6], q->sizes().slice(0, 2), true, true, at::kFloat);
        if (!c.ok || q->size(1) > INT32_MAX || k->size(1) > INT32_MAX || q->size(2) > INT32_MAX) return false;
        if (!scratch_of(args[8], c, &a.workspace, &a.workspace_bytes)) return false;
        a.dtype = c.dtype(), a.rows = q->size(0), a.keys = k->size(0);
        a.heads_q = (int32_t)q->size(1), a.heads_k = (int32_t)k->size(1), a.dim = (int32_t)q->size(2);
        a.scale = (float)(args[7] == Py_None ? std::pow((double)a.dim, -0.5) : PyFloat_AsDouble(args[7]));
        if (PyErr_Occurred()) return false;
        a.q = heads_of(q), a.k = heads_of(k), a.v = heads_of(v), a.out = heads_of(out);
        a.ranges = (const int32_t *)at_of(ranges), a.lse = (float *)at_of(lse);
        if (args[9] != Py_None) {
            PyObject *g[4];
            if (entries(args[9], g, 4) != 4) return false;
            const at::Tensor *dout = c.shaped(g[0], q->sizes()), *dq = c.shaped(g[1], q->sizes());
            const at::Tensor *dk = c.shaped(g[2], k->sizes()), *dv = c.shaped(g[3], k->sizes());
            if (!c.ok) return false;
            a.dout = heads_of(dout), a.dq = heads_of(dq), a.dk = heads_of(dk), a.dv = heads_of(dv);
        }
        *rc = without_gil([&] { return ((int (*)(const hp_attend_args_t *, void *))fn)(&a, stream); });
        return true;
    });
}

#define HP_METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {HP_METHOD(call), HP_METHOD(rotary), HP_METHOD(norm), HP_METHOD(norm_backward), HP_METHOD(attend),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "hp_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_hp_marshal(void) {
    PyObject *m = PyModule_Create(&module);
    // a tensor's layout is that of the torch it was compiled against: the binding compares
    if (m && PyModule_AddStringConstant(m, "torch_version", HP_TORCH_VERSION) < 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
