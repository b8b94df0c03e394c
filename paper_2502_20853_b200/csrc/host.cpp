// The host path of the binding's frequent calls, native: the quantized-matrix object and the marshalling of the linear layer's
// entry points.  A small layer's step is bound by the host (1024 x 192 -> 768: 23 us of device work).  Building the ctypes
// structures and converting their arguments cost more of it than the launches do; here a quantized matrix keeps its C
// description inside the object, and a call reads its arguments straight into the C call.  Python time of a call, without
// the launches, in us (ctypes / native): forward with a quantized weight 10.3 / 5.4, forward of a training step 18.5 / 7.4, backward
// 9.1 / 5.0, of which the allocations of the results are 2.7, 4.1 and 2.7.  1024 x 192 -> 768, whole step: 43 -> 33 us.
// The functions take the address of the library's entry point as their first argument: the library itself is loaded, and
// its absence reported, in binding.py.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <structmember.h>

#include "../../include/mxfp4.h"

namespace {

// ---- quantized matrix: the base of binding.QMat ----
struct Mat {
    PyObject_HEAD
    mxfp4_mat_t m;
    PyObject *buf, *data, *scales;   // one buffer for both (data, scales: views of it, made when asked for) or two tensors
    Py_ssize_t at;                   // where the codes start in buf
    PyObject *q4;                    // what binding.linear_fwd made of it besides (see there); gone once the matrix may have changed
};

int mat_traverse(PyObject *o, visitproc visit, void *arg)
{
    Mat *s = reinterpret_cast<Mat *>(o);
    Py_VISIT(s->buf);
    Py_VISIT(s->data);
    Py_VISIT(s->scales);
    Py_VISIT(s->q4);
    return 0;
}
int mat_clear(PyObject *o)
{
    Mat *s = reinterpret_cast<Mat *>(o);
    Py_CLEAR(s->buf);
    Py_CLEAR(s->data);
    Py_CLEAR(s->scales);
    Py_CLEAR(s->q4);
    return 0;
}
void mat_dealloc(PyObject *o)
{
    PyObject_GC_UnTrack(o);
    mat_clear(o);
    Py_TYPE(o)->tp_free(o);
}

PyObject *g_data_ptr;   // the name of the tensors' method

// Once the tensors of a matrix have been handed out (or came from the caller), its addresses are theirs: a program may give a
// tensor another storage.
bool refresh(Mat *s)
{
    if (s->data && s->data != Py_None) {
        PyObject *a = PyObject_CallMethodNoArgs(s->data, g_data_ptr);
        if (!a) return false;
        s->m.data = reinterpret_cast<void *>((uintptr_t)PyLong_AsUnsignedLongLongMask(a));
        Py_DECREF(a);
    }
    if (s->scales && s->scales != Py_None) {
        PyObject *a = PyObject_CallMethodNoArgs(s->scales, g_data_ptr);
        if (!a) return false;
        s->m.scales = reinterpret_cast<uint8_t *>((uintptr_t)PyLong_AsUnsignedLongLongMask(a));
        Py_DECREF(a);
    }
    return !PyErr_Occurred();
}
PyObject *mat_address(PyObject *o, void *scales)
{
    Mat *s = reinterpret_cast<Mat *>(o);
    return refresh(s) ? PyLong_FromVoidPtr(scales ? (void *)s->m.scales : s->m.data) : nullptr;
}
PyGetSetDef mat_getset[] = {{"data_addr", mat_address, nullptr, nullptr, nullptr}, {"scales_addr", mat_address, nullptr, nullptr, (void *)1}, {nullptr, nullptr, nullptr, nullptr, nullptr}};

PyMemberDef mat_members[] = {
    {"rows", T_LONGLONG, offsetof(Mat, m.rows), 0, nullptr},
    {"cols", T_LONGLONG, offsetof(Mat, m.cols), 0, nullptr},
    {"_buf", T_OBJECT, offsetof(Mat, buf), 0, nullptr},
    {"_data", T_OBJECT, offsetof(Mat, data), 0, nullptr},
    {"_scales", T_OBJECT, offsetof(Mat, scales), 0, nullptr},
    {"_at", T_PYSSIZET, offsetof(Mat, at), 0, nullptr},
    {"_q4", T_OBJECT, offsetof(Mat, q4), 0, nullptr},
    {nullptr, 0, 0, 0, nullptr}};

PyTypeObject mat_type = {PyVarObject_HEAD_INIT(nullptr, 0)};

// ---- arguments of a call ----
struct Args {
    PyObject *const *a;
    bool bad = false;

    uint64_t u64(int i)
    {
        const unsigned long long v = PyLong_AsUnsignedLongLongMask(a[i]);
        if (v == (unsigned long long)-1 && PyErr_Occurred()) bad = true;
        return v;
    }
    int64_t i64(int i) { return (int64_t)u64(i); }
    int32_t i32(int i) { return (int32_t)u64(i); }
    template <class T = void> T *ptr(int i) { return given(i) ? reinterpret_cast<T *>((uintptr_t)u64(i)) : nullptr; }
    bool given(int i) const { return a[i] != Py_None; }
    mxfp4_mat_t mat(int i)
    {
        if (PyObject_TypeCheck(a[i], &mat_type)) {
            Mat *s = reinterpret_cast<Mat *>(a[i]);
            if (!bad && !refresh(s)) bad = true;
            return s->m;
        }
        if (given(i) && !bad) {
            PyErr_SetString(PyExc_TypeError, "a quantized matrix (QMat) is expected");
            bad = true;
        }
        return mxfp4_mat_t{nullptr, nullptr, 0, 0};
    }
    // a matrix that the call writes
    mxfp4_mat_t dst(int i)
    {
        const mxfp4_mat_t m = mat(i);
        if (!bad && given(i)) Py_CLEAR(reinterpret_cast<Mat *>(a[i])->q4);
        return m;
    }
    // Runs the call without the interpreter lock and returns its status.
    template <class F> PyObject *run(F &&f)
    {
        if (bad) return nullptr;
        int32_t s;
        Py_BEGIN_ALLOW_THREADS
        s = f();
        Py_END_ALLOW_THREADS
        return PyLong_FromLong(s);
    }
};

bool counted(const char *name, Py_ssize_t n, Py_ssize_t want)
{
    if (n == want) return true;
    PyErr_Format(PyExc_TypeError, "%s: %zd arguments expected, %zd given", name, want, n);
    return false;
}

Py_ssize_t mat_bytes(int64_t rows, int64_t cols)   // codes and scales in one buffer, both on 256-byte boundaries
{
    const int64_t s = ((rows + 127) >> 7) * ((cols + 127) >> 7) * 512;
    return ((rows * (cols / 2) + 255) & ~int64_t(255)) + (s > 256 ? s : 256);
}

// nbytes(rows, cols, ...) -> bytes of one buffer for all of these matrices
PyObject *h_nbytes(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    Args r{a};
    Py_ssize_t sum = 0;
    for (int i = 0; i + 1 < n; i += 2) sum += mat_bytes(r.i64(i), r.i64(i + 1));
    return r.bad ? nullptr : PyLong_FromSsize_t(sum);
}

// place(matrix, buf, address of buf, rows, cols): puts the matrix into buf.
// place(class, buf, address of buf, rows, cols, rows, cols, ...) -> tuple of new matrices, one behind the other in buf.
PyObject *h_place(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    const bool one = n == 5 && PyObject_TypeCheck(a[0], &mat_type);
    if (!one && (n < 5 || (n & 1) == 0 || !PyType_Check(a[0]) || !PyType_IsSubtype(reinterpret_cast<PyTypeObject *>(a[0]), &mat_type))) {
        PyErr_SetString(PyExc_TypeError, "place(matrix or class, buf, address, rows, cols, ...)");
        return nullptr;
    }
    Args r{a};
    uint8_t *p = r.ptr<uint8_t>(2);
    const Py_ssize_t count = (n - 3) / 2;
    PyObject *all = one ? Py_NewRef(Py_None) : PyTuple_New(count);
    if (!all) return nullptr;
    Py_ssize_t at = 0;
    for (int i = 0; i < count; i++) {
        const int64_t rows = r.i64(3 + 2 * i), cols = r.i64(4 + 2 * i);
        PyTypeObject *cls = reinterpret_cast<PyTypeObject *>(a[0]);
        PyObject *o = r.bad ? nullptr : one ? a[0] : cls->tp_alloc(cls, 0);
        if (!o) {
            Py_DECREF(all);
            return nullptr;
        }
        Mat *s = reinterpret_cast<Mat *>(o);
        s->m = mxfp4_mat_t{p + at, p + at + ((rows * (cols / 2) + 255) & ~int64_t(255)), rows, cols};
        Py_XSETREF(s->buf, Py_NewRef(a[1]));
        Py_CLEAR(s->data);
        Py_CLEAR(s->scales);
        s->at = at;
        at += mat_bytes(rows, cols);
        if (!one) PyTuple_SET_ITEM(all, i, o);
    }
    return all;
}

PyObject *h_linear_fwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    // entry, x, ldx, m, k, w, n, bias, y, ldy, xq, wq, xq_t, wq_t, seed, scale_mode, epilogue, status, stream
    if (!counted("linear_fwd", n, 19)) return nullptr;
    Args r{a};
    const auto f = reinterpret_cast<decltype(&mxfp4_linear_fwd_ex)>(r.ptr(0));
    mxfp4_linear_ctx_t c{r.mat(10), r.given(5) ? r.dst(11) : r.mat(11), r.mat(12), r.u64(14), r.mat(13), r.u64(14)};
    const void *x = r.ptr(1), *w = r.ptr(5), *bias = r.ptr(7);
    void *y = r.ptr(8), *stream = r.ptr(18);
    const int64_t ldx = r.i64(2), m = r.i64(3), k = r.i64(4), nn = r.i64(6), ldy = r.i64(9);
    const int32_t mode = r.i32(15);
    const auto *epi = r.ptr<const mxfp4_epilogue_t>(16);
    auto *status = r.ptr<uint32_t>(17);
    return r.run([&] { return f(x, ldx, m, k, w, nn, bias, y, ldy, &c, mode, epi, status, stream); });
}

PyObject *h_linear_bwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    // entry, dy, lddy, dyq, dyq_t, xq, wq, xq_t, wq_t, ctx seed, seed, scale_mode, dx, lddx, dw, lddw, dw dtype, epilogue, workspace,
    // workspace bytes, status, stream
    if (!counted("linear_bwd", n, 22)) return nullptr;
    Args r{a};
    const auto f = reinterpret_cast<decltype(&mxfp4_linear_bwd_ex)>(r.ptr(0));
    const void *dy = r.ptr(1);
    const bool given = r.given(3), given_t = r.given(4);
    const mxfp4_mat_t dyq = r.mat(3), dyq_t = r.mat(4);
    const mxfp4_linear_ctx_t c{r.mat(5), r.mat(6), r.mat(7), r.u64(9), r.mat(8), r.u64(9)};
    const int64_t lddy = r.i64(2), lddx = r.i64(13), lddw = r.i64(15);
    const uint64_t seed = r.u64(10), ws_bytes = r.u64(19);
    const int32_t mode = r.i32(11), dwt = r.i32(16);
    void *dx = r.ptr(12), *dw = r.ptr(14), *ws = r.ptr(18), *stream = r.ptr(21);
    const auto *epi = r.ptr<const mxfp4_epilogue_t>(17);
    auto *status = r.ptr<uint32_t>(20);
    return r.run([&] {
        return f(dy, lddy, given ? &dyq : nullptr, given_t ? &dyq_t : nullptr, &c, seed, mode, dx, lddx, dw, lddw, dwt, epi, ws, ws_bytes, status, stream);
    });
}

PyObject *h_quantize(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    // entry, x, rows, cols, ld, dst, scale_mode, rounding, seed, stream_id, status, stream
    if (!counted("quantize", n, 12)) return nullptr;
    Args r{a};
    const auto f = reinterpret_cast<decltype(&mxfp4_quantize)>(r.ptr(0));
    const mxfp4_qparams_t qp{r.i32(6), r.i32(7), r.u64(8), (uint32_t)r.u64(9), 0u};
    const void *x = r.ptr(1);
    const int64_t rows = r.i64(2), cols = r.i64(3), ld = r.i64(4);
    const mxfp4_mat_t dst = r.dst(5);
    auto *status = r.ptr<uint32_t>(10);
    void *stream = r.ptr(11);
    return r.run([&] { return f(x, rows, cols, ld, dst, &qp, status, stream); });
}

PyObject *h_quantize_t(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    // entry, x, source matrix, rows, cols, ld, dst, scale_mode, rounding, seed, stream_id, status, stream
    if (!counted("quantize_t", n, 13)) return nullptr;
    Args r{a};
    const auto f = reinterpret_cast<decltype(&mxfp4_quantize_t)>(r.ptr(0));
    const mxfp4_qparams_t qp{r.i32(7), r.i32(8), r.u64(9), (uint32_t)r.u64(10), 0u};
    const void *x = r.ptr(1);
    const bool given = r.given(2);
    const mxfp4_mat_t src = r.mat(2), dst = r.dst(6);
    const int64_t rows = r.i64(3), cols = r.i64(4), ld = r.i64(5);
    auto *status = r.ptr<uint32_t>(11);
    void *stream = r.ptr(12);
    return r.run([&] { return f(x, given ? &src : nullptr, rows, cols, ld, dst, &qp, status, stream); });
}

PyObject *h_qema(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    // entry, w, ema, beta, update, n, k, dst, scale_mode, w_prev | None, wq_prev, dist_w, dist_q, status, stream
    if (!counted("qema_quantize", n, 15)) return nullptr;
    Args r{a};
    const auto f = reinterpret_cast<decltype(&mxfp4_qema_quantize)>(r.ptr(0));
    const double beta = PyFloat_AsDouble(a[3]);
    if (beta == -1.0 && PyErr_Occurred()) return nullptr;
    const void *w = r.ptr(1);
    float *ema = r.ptr<float>(2);
    const int32_t update = r.i32(4), mode = r.i32(8);
    const int64_t nn = r.i64(5), k = r.i64(6);
    const mxfp4_mat_t dst = r.dst(7);
    const bool osc = r.given(9);
    const mxfp4_osc_state_t o{r.ptr(9), r.dst(10), r.ptr<float>(11), r.ptr<float>(12)};
    auto *status = r.ptr<uint32_t>(13);
    void *stream = r.ptr(14);
    return r.run([&] { return f(w, ema, (float)beta, update, nn, k, dst, mode, osc ? &o : nullptr, status, stream); });
}

// ---- tensors as arguments (the operators around the linear layers) ----
// Attributes of a tensor read here cost a third of what they cost in Python (0.4 against 1.3 us for the five of a matrix).
PyObject *g_get_device, *g_dtype, *g_shape, *g_stride, *g_kind, *g_weight, *g_bias, *g_eps, *g_bf16, *g_fp32;

bool refuse(const char *what)
{
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_AssertionError, what);
    return false;
}
bool number(PyObject *o, int64_t &v)     // takes the reference
{
    if (!o) return false;
    v = PyLong_AsLongLong(o);
    Py_DECREF(o);
    return v != -1 || !PyErr_Occurred();
}
bool entries(PyObject *o, int n, int64_t *v)     // takes the reference: a tuple of n numbers
{
    if (!o) return false;
    bool ok = PyTuple_Check(o) && PyTuple_GET_SIZE(o) == n;
    for (int i = 0; ok && i < n; i++) {
        v[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(o, i));
        ok = v[i] != -1 || !PyErr_Occurred();
    }
    Py_DECREF(o);
    return ok;
}
struct Rows {
    void *p = nullptr;
    int64_t rows = 0, cols = 0, ld = 0;
    int32_t dtype = 0;
    bool given = false;
};
// dims 1 or 2 of bf16 or fp32 on `device`, the last one without gaps; one dimension counts as one row.
bool tensor(PyObject *t, int64_t device, int dims, Rows &r)
{
    int64_t dev, size[2], step[2];
    if (!number(PyObject_CallMethodNoArgs(t, g_get_device), dev)) return false;
    if (dev != device) return refuse("a tensor on the current device is expected");
    PyObject *dtype = PyObject_GetAttr(t, g_dtype);
    if (!dtype) return false;
    Py_DECREF(dtype);
    if (dtype != g_bf16 && dtype != g_fp32) return refuse("a tensor of bf16 or fp32 is expected");
    if (!entries(PyObject_GetAttr(t, g_shape), dims, size) || !entries(PyObject_CallMethodNoArgs(t, g_stride), dims, step))
        return refuse(dims == 2 ? "a matrix is expected" : "a vector is expected");
    if (size[dims - 1] > 1 && step[dims - 1] != 1) return refuse("the columns must lie side by side");
    PyObject *a = PyObject_CallMethodNoArgs(t, g_data_ptr);
    if (!a) return false;
    r.p = reinterpret_cast<void *>((uintptr_t)PyLong_AsUnsignedLongLongMask(a));
    Py_DECREF(a);
    r.dtype = dtype == g_fp32 ? MXFP4_OUT_FP32 : MXFP4_OUT_BF16;
    r.rows = dims == 2 ? size[0] : 1, r.cols = size[dims - 1];
    r.ld = dims == 2 && size[0] > 1 ? step[0] : r.cols;     // of a single row torch may say anything
    r.given = true;
    return !PyErr_Occurred();
}
// A matrix argument of `like`'s shape (if that is given) and of a type (-1: any).
bool matrix(PyObject *t, int64_t device, const Rows *like, int dtype, Rows &r)
{
    if (t == Py_None) return true;
    if (!tensor(t, device, 2, r)) return false;
    if (like && (r.rows != like->rows || r.cols != like->cols)) return refuse("a matrix of another shape is expected");
    return dtype < 0 || r.dtype == dtype || refuse("a matrix of another type is expected");
}
// One of the outputs that the binding allocates itself unless its caller gives them (a tensor, which the binding has looked at): then their
// address comes in their place, of `like`'s shape and without gaps.
bool output(PyObject *t, int64_t device, const Rows &like, int dtype, Rows &r)
{
    if (!PyLong_Check(t)) return matrix(t, device, &like, dtype, r);
    r = like;
    r.p = reinterpret_cast<void *>((uintptr_t)PyLong_AsUnsignedLongLongMask(t));
    r.ld = like.cols, r.dtype = dtype;
    return !PyErr_Occurred();
}
bool norm_of(PyObject *o, int64_t device, int64_t cols, mxfp4_norm_t &n)
{
    n = mxfp4_norm_t{MXFP4_NORM_NONE, 0, nullptr, nullptr, 0.0f, 0u};
    if (o == Py_None) return true;
    int64_t kind;
    if (!number(PyObject_GetAttr(o, g_kind), kind)) return false;
    n.kind = (int32_t)kind;
    PyObject *e = PyObject_GetAttr(o, g_eps);
    if (!e) return false;
    n.eps = (float)PyFloat_AsDouble(e);
    Py_DECREF(e);
    if (PyErr_Occurred()) return false;
    Rows side[2];
    PyObject *names[2] = {g_weight, g_bias};
    for (int k = 0; k < 2; k++) {
        PyObject *t = PyObject_GetAttr(o, names[k]);
        if (!t) return false;
        const bool ok = t == Py_None || tensor(t, device, 1, side[k]);
        Py_DECREF(t);
        if (!ok) return false;
        if (side[k].given && side[k].cols != cols) return refuse("weight and bias have a number for each column");
    }
    if (side[0].given && side[1].given && side[0].dtype != side[1].dtype) return refuse("weight and bias have one type");
    n.dtype = side[0].given ? side[0].dtype : side[1].dtype;
    n.weight = side[0].p, n.bias = side[1].p;
    return true;
}
// What residual_norm_fwd and _bwd share: arguments pre, post, gate, residual_scale, branch_scale at a[0 .. 4].
bool plan_of(PyObject *const *a, int64_t device, const Rows &x, int32_t x_dtype, mxfp4_residual_norm_t &n)
{
    n = mxfp4_residual_norm_t{};
    n.rows = x.rows, n.cols = x.cols, n.x_dtype = x_dtype;
    if (!norm_of(a[0], device, x.cols, n.pre) || !norm_of(a[1], device, x.cols, n.post)) return false;
    if (a[2] != Py_None) {
        Rows g;
        PyObject *shape = PyObject_GetAttr(a[2], g_shape);
        if (!shape) return false;
        const int dims = PyTuple_Check(shape) && PyTuple_GET_SIZE(shape) == 1 ? 1 : 2;
        Py_DECREF(shape);
        if (!tensor(a[2], device, dims, g)) return false;
        if (g.cols != x.cols) return refuse("the gate has a number for each column");
        if (g.rows == 0 && x.rows > 0) return refuse("a gate for each run of rows is expected");
        n.gate = g.p, n.gates = g.rows, n.ld_gate = g.ld, n.gate_dtype = g.dtype;
    }
    n.residual_scale = (float)PyFloat_AsDouble(a[3]);
    n.branch_scale = (float)PyFloat_AsDouble(a[4]);
    return !PyErr_Occurred();
}
mxfp4_ckpt_t ckpt_of(Args &r, int i, const Rows &x) { return mxfp4_ckpt_t{r.ptr<uint8_t>(i), r.ptr<uint8_t>(i + 1), r.given(i) ? x.rows : 0, r.given(i) ? x.cols : 0}; }

PyObject *h_norm_fwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    // entry, device, x, f, pre, post, gate, residual scale, branch scale, x_out, h, hq, stats, codes and scales of x^, of f^, scale_mode, status, stream
    if (!counted("residual_norm_fwd", n, 20)) return nullptr;
    Args r{a};
    const auto f = reinterpret_cast<decltype(&mxfp4_residual_norm_fwd)>(r.ptr(0));
    const int64_t device = r.i64(1);
    Rows x, b, xo, h;
    mxfp4_residual_norm_t plan;
    if (a[2] == Py_None) refuse("x is expected");
    if (a[2] == Py_None || !matrix(a[2], device, nullptr, -1, x) || !matrix(a[3], device, &x, MXFP4_OUT_BF16, b) || !plan_of(a + 4, device, x, x.dtype, plan) ||
        !output(a[9], device, x, x.dtype, xo) || !output(a[10], device, x, MXFP4_OUT_BF16, h))
        return nullptr;
    const mxfp4_mat_t hq = r.dst(11);
    const bool with_hq = r.given(11);
    float *stats = r.ptr<float>(12);
    const mxfp4_ckpt_t xc = ckpt_of(r, 13, x), fc = ckpt_of(r, 15, x);
    const int32_t mode = r.i32(17);
    auto *status = r.ptr<uint32_t>(18);
    void *stream = r.ptr(19);
    return r.run([&] { return f(&plan, x.p, x.ld, b.p, b.ld, xo.p, xo.ld, h.p, h.ld, with_hq ? &hq : nullptr, stats, xc, fc, mode, status, stream); });
}

PyObject *h_norm_bwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    // entry, device, dh, dx_out, pre, post, gate, residual scale, branch scale, stats, x, f, codes and scales of x^, of f^, dx, df, gradients of the
    // norms (4) and of the gate, workspace, its bytes, stream
    if (!counted("residual_norm_bwd", n, 26)) return nullptr;
    Args r{a};
    const auto f = reinterpret_cast<decltype(&mxfp4_residual_norm_bwd)>(r.ptr(0));
    const int64_t device = r.i64(1);
    Rows dx, dh, dxo, x, b, df, st;
    mxfp4_residual_norm_t plan;
    if (a[16] == Py_None) refuse("dx is expected");
    if (a[16] == Py_None || !matrix(a[16], device, nullptr, -1, dx) || !matrix(a[2], device, &dx, MXFP4_OUT_BF16, dh) || !matrix(a[3], device, &dx, dx.dtype, dxo) ||
        !plan_of(a + 4, device, dx, dx.dtype, plan) || !matrix(a[9], device, nullptr, MXFP4_OUT_FP32, st) || !matrix(a[10], device, &dx, dx.dtype, x) ||
        !matrix(a[11], device, &dx, MXFP4_OUT_BF16, b) || !output(a[17], device, dx, MXFP4_OUT_BF16, df))
        return nullptr;
    if (st.given && (st.rows != 4 || st.cols != dx.rows || (st.ld != st.cols && st.cols > 0))) {
        refuse("the statistics are [4, rows], without gaps");
        return nullptr;
    }
    mxfp4_residual_norm_bwd_t q{};
    q.dh_bf16 = dh.p, q.lddh = dh.ld, q.dx_out = dxo.p, q.lddxo = dxo.ld, q.stats = static_cast<const float *>(st.p);
    q.x_ckpt = ckpt_of(r, 12, dx), q.f_ckpt = ckpt_of(r, 14, dx);
    q.x_out = x.p, q.ldxo = x.ld, q.f_bf16 = b.p, q.ldf = b.ld, q.dx = dx.p, q.lddx = dx.ld, q.df_bf16 = df.p, q.lddf = df.ld;
    q.dw_pre = r.ptr<float>(18), q.db_pre = r.ptr<float>(19), q.dw_post = r.ptr<float>(20), q.db_post = r.ptr<float>(21), q.dgate = r.ptr<float>(22);
    void *ws = r.ptr(23), *stream = r.ptr(25);
    const uint64_t bytes = r.u64(24);
    return r.run([&] { return f(&plan, &q, ws, bytes, stream); });
}

PyObject *h_norm_workspace(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    // entry, rows, cols, gates
    if (!counted("residual_norm_workspace_bytes", n, 4)) return nullptr;
    Args r{a};
    const auto f = reinterpret_cast<decltype(&mxfp4_residual_norm_workspace_bytes)>(r.ptr(0));
    const int64_t rows = r.i64(1), cols = r.i64(2), gates = r.i64(3);
    return r.bad ? nullptr : PyLong_FromSize_t(f(rows, cols, gates));
}

PyObject *h_act_fwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    // entry, device, y, act, z, codes, scales, scale_mode, status, stream
    if (!counted("act_fwd", n, 10)) return nullptr;
    Args r{a};
    const auto f = reinterpret_cast<decltype(&mxfp4_act_fwd)>(r.ptr(0));
    const int64_t device = r.i64(1);
    const int32_t act = r.i32(3);
    Rows y, z;
    if (!matrix(a[2], device, nullptr, MXFP4_OUT_BF16, y) || !matrix(a[4], device, nullptr, MXFP4_OUT_BF16, z)) return nullptr;
    const int64_t halves = act == MXFP4_ACT_GEGLU || act == MXFP4_ACT_SWIGLU ? 2 : 1;
    if (z.rows != y.rows || z.cols * halves != y.cols) {
        refuse("z has y's shape, or half its columns where the activation is gated");
        return nullptr;
    }
    const mxfp4_ckpt_t c = ckpt_of(r, 5, y);
    const int32_t mode = r.i32(7);
    auto *status = r.ptr<uint32_t>(8);
    void *stream = r.ptr(9);
    return r.run([&] { return f(y.p, y.ld, z.rows, z.cols, act, z.p, z.ld, c, mode, status, stream); });
}

PyObject *h_act_bwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    // entry, device, dz, codes, scales, act, dy, stream
    if (!counted("act_bwd", n, 8)) return nullptr;
    Args r{a};
    const auto f = reinterpret_cast<decltype(&mxfp4_act_bwd)>(r.ptr(0));
    const int64_t device = r.i64(1);
    const int32_t act = r.i32(5);
    Rows dz, dy;
    if (!matrix(a[2], device, nullptr, MXFP4_OUT_BF16, dz) || !matrix(a[6], device, nullptr, MXFP4_OUT_BF16, dy)) return nullptr;
    const int64_t halves = act == MXFP4_ACT_GEGLU || act == MXFP4_ACT_SWIGLU ? 2 : 1;
    if (dz.rows != dy.rows || dz.cols * halves != dy.cols) {
        refuse("dz has dy's shape, or half its columns where the activation is gated");
        return nullptr;
    }
    const mxfp4_ckpt_t c = ckpt_of(r, 3, dy);
    void *stream = r.ptr(7);
    return r.run([&] { return f(dz.p, dz.ld, c, act, dy.p, dy.ld, stream); });
}

PyObject *h_ckpt(PyObject *, PyObject *const *a, Py_ssize_t n, bool store)
{
    // entry, device, the matrix, codes, scales, scale_mode, status, stream
    if (!counted("checkpoint", n, 8)) return nullptr;
    Args r{a};
    const int64_t device = r.i64(1);
    Rows x;
    if (!matrix(a[2], device, nullptr, -1, x)) return nullptr;
    const mxfp4_ckpt_t c = ckpt_of(r, 3, x);
    const int32_t mode = r.i32(5);
    auto *status = r.ptr<uint32_t>(6);
    void *entry = r.ptr(0), *stream = r.ptr(7);
    if (store) return r.run([&] { return reinterpret_cast<decltype(&mxfp4_checkpoint_store)>(entry)(x.p, x.dtype, x.ld, c, mode, status, stream); });
    return r.run([&] { return reinterpret_cast<decltype(&mxfp4_checkpoint_load)>(entry)(c, x.p, x.dtype, x.ld, stream); });
}
PyObject *h_ckpt_store(PyObject *, PyObject *const *a, Py_ssize_t n) { return h_ckpt(nullptr, a, n, true); }
PyObject *h_ckpt_load(PyObject *, PyObject *const *a, Py_ssize_t n) { return h_ckpt(nullptr, a, n, false); }

// types(torch.bfloat16, torch.float32): what the tensors' dtypes are compared with
PyObject *h_types(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!counted("types", n, 2)) return nullptr;
    Py_XSETREF(g_bf16, Py_NewRef(a[0]));
    Py_XSETREF(g_fp32, Py_NewRef(a[1]));
    Py_RETURN_NONE;
}

#define FAST(name, fn) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(fn)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST("nbytes", h_nbytes), FAST("place", h_place), FAST("linear_fwd", h_linear_fwd), FAST("linear_bwd", h_linear_bwd),
                         FAST("quantize", h_quantize), FAST("quantize_t", h_quantize_t), FAST("qema_quantize", h_qema),
                         FAST("residual_norm_fwd", h_norm_fwd), FAST("residual_norm_bwd", h_norm_bwd), FAST("residual_norm_workspace_bytes", h_norm_workspace),
                         FAST("act_fwd", h_act_fwd), FAST("act_bwd", h_act_bwd), FAST("checkpoint_store", h_ckpt_store), FAST("checkpoint_load", h_ckpt_load),
                         FAST("types", h_types), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_host", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__host()
{
    mat_type.tp_name = "paper_2502_20853_b200._host.Mat";
    mat_type.tp_basicsize = sizeof(Mat);
    mat_type.tp_flags = Py_TPFLAGS_DEFAULT | Py_TPFLAGS_BASETYPE | Py_TPFLAGS_HAVE_GC;
    mat_type.tp_new = PyType_GenericNew;
    mat_type.tp_dealloc = mat_dealloc;
    mat_type.tp_traverse = mat_traverse;
    mat_type.tp_clear = mat_clear;
    mat_type.tp_members = mat_members;
    mat_type.tp_getset = mat_getset;
    const struct {
        PyObject **at;
        const char *name;
    } names[] = {{&g_data_ptr, "data_ptr"}, {&g_get_device, "get_device"}, {&g_dtype, "dtype"}, {&g_shape, "shape"}, {&g_stride, "stride"},
                 {&g_kind, "kind"}, {&g_weight, "weight"}, {&g_bias, "bias"}, {&g_eps, "eps"}};
    for (const auto &n : names)
        if (!*n.at && !(*n.at = PyUnicode_InternFromString(n.name))) return nullptr;
    if (PyType_Ready(&mat_type) < 0) return nullptr;
    PyObject *m = PyModule_Create(&module);
    if (m && (PyModule_AddObjectRef(m, "Mat", reinterpret_cast<PyObject *>(&mat_type)) < 0 || PyModule_AddIntConstant(m, "interface", 3) < 0)) Py_CLEAR(m);
    return m;
}
