// wm_seq_ext.cpp -- the Python side of include/wm_seq.h: tensors to pointers.
//
// A small CPython module: it checks types, shapes and strides, allocates outputs, takes the
// current stream and calls the C entry.  A call of a few kernels costs about as much on the
// host as on the device, and the same marshalling through ctypes took 15 us for one step of
// a scan, most of it in Python; here it takes 3 with its outputs given.  That an array is memory
// of the handle's device, and aligned, the C entries check.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <string>
#include <vector>

#include "wm_seq.h"

namespace {

PyObject *g_error = nullptr;  // raised with (status, message)

struct Refuse {  // becomes a ValueError
    std::string why;
};
struct Failed {  // a Python exception is set
};

std::string text(at::IntArrayRef s) {
    std::string t = "(";
    for (size_t i = 0; i < s.size(); ++i) t += (i ? ", " : "") + std::to_string(s[i]);
    return t + ")";
}

const at::Tensor *maybe(PyObject *o, const char *what) {
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) throw Refuse{std::string(what) + ": a tensor is needed"};
    return &THPVariable_Unpack(o);
}
const at::Tensor &tensor(PyObject *o, const char *what) {
    const at::Tensor *t = maybe(o, what);
    if (!t) throw Refuse{std::string(what) + ": a tensor is needed"};
    return *t;
}

int dtype_of(const at::Tensor &t) {
    if (t.scalar_type() == at::kFloat) return WM_FP32;
    if (t.scalar_type() == at::kBFloat16) return WM_BF16;
    throw Refuse{std::string("float32 or bfloat16 tensors are needed, got ") + toString(t.scalar_type())};
}

// Sizes that the C entries take as int.
int size(int64_t v) {
    if (v > 0x7fffffff) throw Refuse{"an axis is too long: " + std::to_string(v)};
    return (int)v;
}

// A dense tensor of this type and shape: its address (null for none).
template <class P = void>
P *flat(const at::Tensor *t, at::ScalarType type, at::IntArrayRef shape, const char *what) {
    if (!t) return nullptr;
    if (t->scalar_type() != type || t->sizes() != shape || !t->is_contiguous())
        throw Refuse{std::string(what) + ": a contiguous " + toString(type) + " tensor of shape " + text(shape) + " is needed, got " +
                     toString(t->scalar_type()) + " " + text(t->sizes())};
    return static_cast<P *>(t->data_ptr());
}

// A [T, N, H] (or, one step, [N, H]) tensor whose last axis is dense.
wm_seq_view view(const at::Tensor &t, at::ScalarType type, at::IntArrayRef shape, const char *what) {
    const auto st = t.strides();
    if (t.scalar_type() != type || t.sizes() != shape || (st.back() != 1 && shape.back() > 1))
        throw Refuse{std::string(what) + ": a " + toString(type) + " tensor of shape " + text(shape) +
                     " with a dense last axis is needed, got " + toString(t.scalar_type()) + " " + text(t.sizes())};
    return {t.data_ptr(), shape.size() == 3 ? st[0] : 0, st[shape.size() - 2]};
}

// The stride of a tensor's rows: its leading axes have to be one run of them.
long long row_stride(const at::Tensor &t, const char *what) {
    const int64_t n = t.dim();
    if (n < 1) throw Refuse{std::string(what) + " needs at least one axis"};
    if (t.is_contiguous()) return t.size(-1);
    const auto st = t.strides();
    const auto sz = t.sizes();
    if (sz[n - 1] > 1 && st[n - 1] != 1) throw Refuse{std::string(what) + ": its last axis must be dense"};
    bool any = false;
    long long row = sz[n - 1], span = 0;  // the rows' stride; the next axis's, of the axes seen so far from the last
    for (int64_t i = n - 2; i >= 0; --i) {
        if (sz[i] == 1) continue;
        if (!any) row = st[i];
        else if (st[i] != span) throw Refuse{std::string(what) + ": its leading axes must be one run of rows with a fixed stride"};
        any = true;
        span = st[i] * sz[i];
    }
    return row;
}

struct Call {
    wm_seq *h;
    int index;
    PyObject *const *a;
    Call(PyObject *const *args, Py_ssize_t n, Py_ssize_t want) : a(args + 2) {
        if (n != want + 2) throw Refuse{"wrong number of arguments"};
        if (args[0] == Py_None) throw Refuse{"the handle is closed"};
        h = static_cast<wm_seq *>(PyLong_AsVoidPtr(args[0]));
        index = (int)PyLong_AsLong(args[1]);
        if (PyErr_Occurred()) throw Failed{};
        if (!h) throw Refuse{"the handle is closed"};
    }
    at::Tensor fresh(at::IntArrayRef shape, at::ScalarType type) const {
        return at::empty(shape, at::TensorOptions().dtype(type).device(at::kCUDA, (c10::DeviceIndex)index));
    }
    void *stream() const { return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)index).stream(); }
    double number(int i) const {
        const double v = PyFloat_AsDouble(a[i]);
        if (v == -1.0 && PyErr_Occurred()) throw Failed{};
        return v;
    }
    bool yes(int i) const {
        const int v = PyObject_IsTrue(a[i]);
        if (v < 0) throw Failed{};
        return v;
    }
    // The C call, without the interpreter's lock: it may wait for the device (a workspace that grows), and what it
    // waits for may need another Python thread.  The arrays it takes are the caller's, who holds them meanwhile.
    template <class F>
    void run(F call) const {
        wm_status st;
        Py_BEGIN_ALLOW_THREADS;
        st = call();
        Py_END_ALLOW_THREADS;
        if (st == WM_OK) return;
        PyObject *args = Py_BuildValue("(is)", (int)st, wm_seq_last_error(h));
        if (args) {
            PyErr_SetObject(g_error ? g_error : PyExc_RuntimeError, args);
            Py_DECREF(args);
        }
        throw Failed{};
    }
};

PyObject *give(at::Tensor &t) { return THPVariable_Wrap(std::move(t)); }
// The tensor that a caller gave for an output, or the one that was made.
PyObject *give(PyObject *given, at::Tensor &made) {
    if (given == Py_None) return give(made);
    Py_INCREF(given);
    return given;
}
PyObject *none() {
    Py_INCREF(Py_None);
    return Py_None;
}
PyObject *tuple(std::initializer_list<PyObject *> items) {
    PyObject *t = PyTuple_New((Py_ssize_t)items.size());
    Py_ssize_t i = 0;
    for (PyObject *o : items) {
        if (!o || !t) {
            Py_XDECREF(t);
            throw Failed{};
        }
        PyTuple_SET_ITEM(t, i++, o);
    }
    return t;
}

PyObject *embed(const Call &c) {
    const at::Tensor &table = tensor(c.a[0], "table"), &tokens = tensor(c.a[1], "tokens");
    if (table.dim() != 2) throw Refuse{"table [V, D] is needed"};
    const auto type = table.scalar_type();
    const int dt = dtype_of(table);
    std::vector<int64_t> full(tokens.sizes().begin(), tokens.sizes().end());
    full.push_back(table.size(1));
    at::Tensor made;
    const at::Tensor *out = maybe(c.a[3], "out");
    const float scale = (float)c.number(2);
    const void *tp = flat(&table, type, table.sizes(), "table");
    const int32_t *kp = flat<int32_t>(&tokens, at::kInt, tokens.sizes(), "tokens");
    if (!out) out = &(made = c.fresh(full, type));
    void *op = flat(out, type, full, "out"), *s = c.stream();
    const long long n = tokens.numel();
    const int V = size(table.size(0)), D = size(table.size(1));
    c.run([&] { return wm_seq_embed(c.h, dt, n, V, D, tp, kp, scale, op, s); });
    return give(c.a[3], made);
}

PyObject *embed_backward(const Call &c) {
    const at::Tensor &tokens = tensor(c.a[0], "tokens"), &dout = tensor(c.a[1], "dout");
    const auto type = dout.scalar_type();
    const int dt = dtype_of(dout);
    const long long V = PyLong_AsLongLong(c.a[2]);
    if (V == -1 && PyErr_Occurred()) throw Failed{};
    if (dout.dim() < 1 || V < 1 || V > 0x7fffffff) throw Refuse{"dout [..., D] and 1 <= vocab < 2^31 are needed"};
    std::vector<int64_t> full(tokens.sizes().begin(), tokens.sizes().end());
    full.push_back(dout.size(-1));
    const int64_t shape[2] = {(int64_t)V, dout.size(-1)};
    const float scale = (float)c.number(3);
    const int32_t *kp = flat<int32_t>(&tokens, at::kInt, tokens.sizes(), "tokens");
    const void *dp = flat(&dout, type, full, "dout");
    at::Tensor made;
    const at::Tensor *out = maybe(c.a[4], "out");
    if (!out) out = &(made = c.fresh(shape, type));
    void *op = flat(out, type, shape, "out"), *s = c.stream();
    const long long n = tokens.numel();
    const int D = size(shape[1]);
    c.run([&] { return wm_seq_embed_backward(c.h, dt, n, (int)V, D, kp, dp, scale, op, s); });
    return give(c.a[4], made);
}

PyObject *layer_norm(const Call &c) {
    const at::Tensor &x = tensor(c.a[0], "x"), *w = maybe(c.a[1], "weight"), *b = maybe(c.a[2], "bias");
    const auto type = x.scalar_type();
    const int dt = dtype_of(x);
    const long long ldx = row_stride(x, "x");
    const int64_t D = x.size(-1), par[1] = {D};
    const auto lead = x.sizes().slice(0, x.dim() - 1);
    const float eps = (float)c.number(3), *wp = flat<float>(w, at::kFloat, par, "weight"), *bp = flat<float>(b, at::kFloat, par, "bias");
    const bool stats = c.yes(4);
    at::Tensor made, mean, rstd;
    const at::Tensor *out = maybe(c.a[5], "out");
    long long ldy = D;
    if (out) {
        if (out->sizes() != x.sizes() || out->scalar_type() != type) throw Refuse{"out must have x's shape and type"};
        ldy = row_stride(*out, "out");
    } else {
        out = &(made = c.fresh(x.sizes(), type));
    }
    if (stats) {
        mean = c.fresh(lead, at::kFloat);
        rstd = c.fresh(lead, at::kFloat);
    }
    const long long rows = D ? x.numel() / D : 0;
    const int d = size(D);
    const void *xp = x.data_ptr();
    void *op = out->data_ptr(), *s = c.stream();
    float *mp = stats ? (float *)mean.data_ptr() : nullptr, *rp = stats ? (float *)rstd.data_ptr() : nullptr;
    c.run([&] { return wm_seq_layer_norm(c.h, dt, rows, d, xp, ldx, wp, bp, eps, op, ldy, mp, rp, s); });
    if (!stats) return give(c.a[5], made);
    return tuple({give(c.a[5], made), give(mean), give(rstd)});
}

PyObject *layer_norm_backward(const Call &c) {
    const at::Tensor &x = tensor(c.a[0], "x"), *w = maybe(c.a[1], "weight"), &mean = tensor(c.a[2], "mean"),
                     &rstd = tensor(c.a[3], "rstd"), &dy = tensor(c.a[4], "dy");
    const auto type = x.scalar_type();
    const int dt = dtype_of(x);
    const long long ldx = row_stride(x, "x");
    if (dy.sizes() != x.sizes() || dy.scalar_type() != type) throw Refuse{"dy must have x's shape and type"};
    const long long lddy = row_stride(dy, "dy");
    const int64_t D = x.size(-1), par[1] = {D};
    const auto lead = x.sizes().slice(0, x.dim() - 1);
    const float *wp = flat<float>(w, at::kFloat, par, "weight"), *mp = flat<float>(&mean, at::kFloat, lead, "mean"),
                *rp = flat<float>(&rstd, at::kFloat, lead, "rstd");
    at::Tensor made, dw, db;
    const at::Tensor *dx = maybe(c.a[5], "dx");
    long long lddx = D;
    if (dx) {
        if (dx->sizes() != x.sizes() || dx->scalar_type() != type) throw Refuse{"dx must have x's shape and type"};
        lddx = row_stride(*dx, "dx");
    } else {
        dx = &(made = c.fresh(x.sizes(), type));
    }
    const bool params = c.yes(6);
    if (params) {
        dw = c.fresh(par, at::kFloat);
        db = c.fresh(par, at::kFloat);
    }
    const long long rows = D ? x.numel() / D : 0;
    const int d = size(D);
    const void *xp = x.data_ptr(), *yp = dy.data_ptr();
    void *op = dx->data_ptr(), *s = c.stream();
    float *wo = params ? (float *)dw.data_ptr() : nullptr, *bo = params ? (float *)db.data_ptr() : nullptr;
    c.run([&] { return wm_seq_layer_norm_backward(c.h, dt, rows, d, xp, ldx, wp, mp, rp, yp, lddy, op, lddx, wo, bo, s); });
    return tuple({give(c.a[5], made), params ? give(dw) : none(), params ? give(db) : none()});
}

// gate, x, h0, reset, lengths, out, want_last, h_last; STEP: [N, H] arrays, no lengths
template <bool STEP>
PyObject *scan(const Call &c) {
    const at::Tensor &gate = tensor(c.a[0], "gate"), &x = tensor(c.a[1], "x"), *h0 = maybe(c.a[2], "h0"), *reset = maybe(c.a[3], "reset"),
                     *lengths = maybe(c.a[4], "lengths"), *out = maybe(c.a[5], "out"), *last = maybe(c.a[7], "h_last");
    const auto type = gate.scalar_type();
    const int dt = dtype_of(gate);
    if (gate.dim() != (STEP ? 2 : 3)) throw Refuse{STEP ? "gate [N, H] is needed" : "gate [T, N, H] is needed"};
    const auto shape = gate.sizes();
    const int64_t T = STEP ? 1 : shape[0], N = shape[STEP ? 0 : 1], H = shape.back(), nh[2] = {N, H}, n1[1] = {N};
    const wm_seq_view vg = view(gate, type, shape, "gate"), vx = view(x, type, shape, "x");
    const float *p0 = flat<float>(h0, at::kFloat, nh, "h0");
    const uint8_t *pr = flat<uint8_t>(reset, at::kByte, STEP ? at::IntArrayRef(n1) : shape.slice(0, 2), "reset");
    const int32_t *pl = flat<int32_t>(lengths, at::kInt, n1, "lengths");
    at::Tensor made, made_last;
    if (!out) out = &(made = c.fresh(shape, type));
    const wm_seq_view vo = view(*out, type, shape, "out");
    if (!last && c.yes(6)) last = &(made_last = c.fresh(nh, at::kFloat));
    const int n = size(N), hh = size(H);
    float *pe = flat<float>(last, at::kFloat, nh, "h_last");
    void *s = c.stream();
    c.run([&] { return wm_seq_gated_scan(c.h, dt, T, n, hh, &vg, &vx, p0, pr, pl, &vo, pe, s); });
    return tuple({give(c.a[5], made), last ? give(c.a[7], made_last) : none()});
}

PyObject *scan_backward(const Call &c) {
    const at::Tensor &gate = tensor(c.a[0], "gate"), &x = tensor(c.a[1], "x"), &h = tensor(c.a[2], "h"), &dh = tensor(c.a[3], "dh"),
                     *dh_last = maybe(c.a[4], "dh_last"), *h0 = maybe(c.a[5], "h0"), *reset = maybe(c.a[6], "reset"),
                     *lengths = maybe(c.a[7], "lengths"), *dgate = maybe(c.a[8], "dgate"), *dx = maybe(c.a[9], "dx"), *dh0 = maybe(c.a[11], "dh0");
    const auto type = gate.scalar_type();
    const int dt = dtype_of(gate);
    if (gate.dim() != 3) throw Refuse{"gate [T, N, H] is needed"};
    const auto shape = gate.sizes();
    const int64_t N = shape[1], H = shape[2], nh[2] = {N, H}, n1[1] = {N};
    const wm_seq_view vg = view(gate, type, shape, "gate"), vx = view(x, type, shape, "x"), vh = view(h, type, shape, "h"),
                      vd = view(dh, type, shape, "dh");
    const float *pd = flat<float>(dh_last, at::kFloat, nh, "dh_last"), *p0 = flat<float>(h0, at::kFloat, nh, "h0");
    const uint8_t *pr = flat<uint8_t>(reset, at::kByte, shape.slice(0, 2), "reset");
    const int32_t *pl = flat<int32_t>(lengths, at::kInt, n1, "lengths");
    at::Tensor m0, m1, m2;
    if (!dgate) dgate = &(m0 = c.fresh(shape, type));
    if (!dx) dx = &(m1 = c.fresh(shape, type));
    const wm_seq_view v0 = view(*dgate, type, shape, "dgate"), v1 = view(*dx, type, shape, "dx");
    if (!dh0 && c.yes(10)) dh0 = &(m2 = c.fresh(nh, at::kFloat));
    const int n = size(N), hh = size(H);
    float *pe = flat<float>(dh0, at::kFloat, nh, "dh0");
    void *s = c.stream();
    const long long T = shape[0];
    c.run([&] { return wm_seq_gated_scan_backward(c.h, dt, T, n, hh, &vg, &vx, p0, pr, pl, &vh, &vd, pd, &v0, &v1, pe, s); });
    return tuple({give(c.a[8], m0), give(c.a[9], m1), dh0 ? give(c.a[11], m2) : none()});
}

PyObject *clip(const Call &c) {
    struct Ref {
        PyObject *o;
        ~Ref() { Py_XDECREF(o); }
    };
    // (tuples of their own: no other thread can take a tensor out of them while the lock is given up)
    const Ref grads{PySequence_Tuple(c.a[0])};
    if (!grads.o) throw Failed{};
    const Ref outs{c.a[2] == Py_None ? nullptr : PySequence_Tuple(c.a[2])};
    if (PyErr_Occurred()) throw Failed{};
    const Py_ssize_t n = PyTuple_GET_SIZE(grads.o);
    if (outs.o && PyTuple_GET_SIZE(outs.o) != n) throw Refuse{"out needs a tensor for each gradient"};
    std::vector<wm_seq_grad> table((size_t)n);
    for (Py_ssize_t i = 0; i < n; ++i) {
        const at::Tensor &g = tensor(PyTuple_GET_ITEM(grads.o, i), "grads");
        const at::Tensor &o = outs.o ? tensor(PyTuple_GET_ITEM(outs.o, i), "out") : g;
        if (!g.is_contiguous() || o.scalar_type() != g.scalar_type() || o.sizes() != g.sizes() || !o.is_contiguous())
            throw Refuse{"contiguous gradients, and out of the same shapes and types, are needed"};
        table[(size_t)i] = {g.data_ptr(), o.data_ptr(), g.numel(), dtype_of(g)};
    }
    const float max_norm = (float)c.number(1);
    at::Tensor norm = c.fresh({}, at::kFloat);
    const int count = size(n);
    float *np = (float *)norm.data_ptr();
    void *s = c.stream();
    c.run([&] { return wm_seq_clip(c.h, count, table.data(), max_norm, np, s); });
    return give(norm);
}

template <PyObject *(*F)(const Call &), int ARGS>
PyObject *entry(PyObject *, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    try {
        return F(Call(args, n, ARGS));
    } catch (const Refuse &r) {
        PyErr_SetString(PyExc_ValueError, r.why.c_str());
    } catch (const Failed &) {
    }
    return nullptr;
    END_HANDLE_TH_ERRORS
}

PyObject *set_error(PyObject *, PyObject *cls) {
    Py_INCREF(cls);
    Py_XSETREF(g_error, cls);
    Py_RETURN_NONE;
}

#define SEQ_ENTRY(NAME, F, ARGS) {NAME, (PyCFunction)(void *)entry<F, ARGS>, METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {
    SEQ_ENTRY("embed", embed, 4),
    SEQ_ENTRY("embed_backward", embed_backward, 5),
    SEQ_ENTRY("layer_norm", layer_norm, 6),
    SEQ_ENTRY("layer_norm_backward", layer_norm_backward, 7),
    SEQ_ENTRY("gated_scan", scan<false>, 8),
    SEQ_ENTRY("gated_step", scan<true>, 8),
    SEQ_ENTRY("gated_scan_backward", scan_backward, 12),
    SEQ_ENTRY("clip_grads", clip, 3),
    {"set_error", set_error, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_seq_ext", "Marshalling of the sequence operators.", -1, g_methods};

}  // namespace

PyMODINIT_FUNC PyInit__seq_ext() { return PyModule_Create(&g_module); }
