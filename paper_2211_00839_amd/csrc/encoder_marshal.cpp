// Argument marshalling of encoder.py and attention.py in C++: the checks, the results' allocation and the call into the C ABI.
//
// One sample through one operator is a kernel of 3 to 7 us.  Looking at five tensors attribute by attribute from Python and
// passing twenty numbers through ctypes took 10 to 18 us; here it takes about one, beside the allocations and the launch.  Nothing but
// marshalling is done here: the contracts are those of include/rcd.h.
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ATen.h>
#include <c10/core/GradMode.h>
#include <c10/core/impl/VirtualGuardImpl.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <string>
#include <utility>

#include "../../include/rcd.h"
#include "overlap.h"

namespace {

constexpr int64_t BLOCK = 32;
constexpr int NOT_ON_DEVICE = -1;

PyObject *g_error = nullptr;        // RcdError

struct Refusal {
    int status;
    std::string what;
};
[[noreturn]] void refuse(const std::string &what, int status = RCD_ERR_INVALID_ARG) { throw Refusal{status, what}; }

PyObject *raise(const Refusal &r)
{
    PyObject *e = g_error ? PyObject_CallFunction(g_error, "is", r.status, r.what.c_str()) : nullptr;
    if (e) {
        PyErr_SetObject(g_error, e);
        Py_DECREF(e);
    } else if (!PyErr_Occurred()) {
        PyErr_SetString(PyExc_RuntimeError, r.what.c_str());
    }
    return nullptr;
}

void check(int status)
{
    if (status == RCD_OK) return;
    std::string what = "rcd status " + std::to_string(status) + " (" + rcd_strerror(status);
    if (status == RCD_ERR_HIP) what += std::string(": ") + rcd_last_hip_error();
    throw Refusal{status, what + ")"};
}

// A call into the library, with the interpreter free meanwhile (a full launch queue is waited for).
template <typename Call> void run(Call call)
{
    PyThreadState *state = PyEval_SaveThread();
    const int status = call();
    PyEval_RestoreThread(state);
    check(status);
}

int code_of(at::ScalarType t)
{
    switch (t) {
    case at::kFloat: return RCD_F32;
    case at::kBFloat16: return RCD_BF16;
    case at::kFloat8_e4m3fn: return RCD_MXFP8;
    default: return -1;
    }
}

const at::Tensor *tensor(PyObject *o)
{
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) refuse("a tensor is expected");
    return &THPVariable_Unpack(o);
}

// A tensor whose gradients autograd would be expected to record, which these calls do not do: a result without a history must not
// be taken for one with.
void no_history(const std::string &name, const at::Tensor &t)
{
    if (t.requires_grad() && c10::GradMode::is_enabled())
        refuse(name + " requires grad, and this call records no history: call it under torch.no_grad() or inside an autograd.Function, "
                      "with the backward call beside it",
               RCD_ERR_UNSUPPORTED);
}

struct Matrix {
    const at::Tensor *t = nullptr;
    int64_t rows = 0, cols = 0, ld = 0;
    at::ScalarType type = at::kFloat;
    void *p() const { return t ? t->data_ptr() : nullptr; }
};

// A device matrix with contiguous rows.  rows, cols < 0: any; like: the call's first matrix, whose device it has to be on.
Matrix matrix(const char *name, PyObject *o, int64_t rows, int64_t cols, const at::ScalarType *type, const Matrix *like)
{
    const std::string n = name;
    if (!THPVariable_Check(o)) refuse(n + " must be a matrix");
    Matrix m;
    m.t = &THPVariable_Unpack(o);
    const at::Tensor &t = *m.t;
    no_history(n, t);
    if (t.dim() != 2) refuse(n + " must be a matrix");
    if (!t.is_cuda()) refuse(n + ": device tensor expected (there is no CPU path)", NOT_ON_DEVICE);
    m.type = t.scalar_type();
    if (code_of(m.type) < 0) refuse(n + ": float32, bfloat16 or float8_e4m3fn expected", RCD_ERR_UNSUPPORTED);
    if (type && m.type != *type) refuse(n + " must be " + c10::toString(*type), RCD_ERR_UNSUPPORTED);
    m.rows = t.size(0);
    m.cols = t.size(1);
    if ((rows >= 0 && m.rows != rows) || (cols >= 0 && m.cols != cols))
        refuse(n + " must be " + (rows < 0 ? "any" : std::to_string(rows)) + " x " + (cols < 0 ? "any" : std::to_string(cols)) + ", got " +
               std::to_string(m.rows) + " x " + std::to_string(m.cols));
    if (m.cols > 1 && m.rows > 0 && t.stride(1) != 1) refuse("the rows of " + n + " must be contiguous");
    if (m.rows > 1 && t.stride(0) < m.cols) refuse("the rows of " + n + " overlap");
    m.ld = m.rows > 1 ? t.stride(0) : std::max<int64_t>(m.cols, 1);     // (of one row the stride means nothing)
    if (like) {
        if (t.device() != like->t->device()) refuse(n + " is on another device");
    } else if (c10::impl::VirtualGuardImpl(at::kCUDA).getDevice() != t.device()) {
        refuse(n + " is on another device than the current one");
    }
    return m;
}
Matrix optional_matrix(const char *name, PyObject *o, int64_t rows, int64_t cols, at::ScalarType type, const Matrix &like)
{
    return o == Py_None ? Matrix{} : matrix(name, o, rows, cols, &type, &like);
}

const void *vector(const char *name, PyObject *o, int64_t n, at::ScalarType type, const Matrix &like)
{
    if (o == Py_None) return nullptr;
    const std::string s = name;
    if (!THPVariable_Check(o)) refuse(s + " must be a contiguous vector of " + std::to_string(n));
    const at::Tensor &t = THPVariable_Unpack(o);
    no_history(s, t);
    if (t.dim() != 1 || t.size(0) != n || (n > 1 && t.stride(0) != 1)) refuse(s + " must be a contiguous vector of " + std::to_string(n));
    if (t.scalar_type() != type) refuse(s + " must be " + c10::toString(type), RCD_ERR_UNSUPPORTED);
    if (t.device() != like.t->device()) refuse(s + " is on another device");
    return t.data_ptr();
}

struct Scale {
    const uint8_t *p = nullptr;
    int64_t ld = 0;
};
// The scales that belong to an 8-bit matrix; none for any other type.
Scale scale(const char *name, PyObject *o, const Matrix &of, const Matrix &like)
{
    const std::string s = name;
    Scale r;
    if (of.type != at::kFloat8_e4m3fn) {
        if (o != Py_None) refuse(s + " goes with float8_e4m3fn elements only");
        return r;
    }
    const int64_t blocks = (of.cols + BLOCK - 1) / BLOCK;
    if (!THPVariable_Check(o)) refuse(s + " (uint8 or float8_e8m0fnu) is missing");
    const at::Tensor &t = THPVariable_Unpack(o);
    if (t.scalar_type() != at::kByte && t.scalar_type() != at::kFloat8_e8m0fnu) refuse(s + " (uint8 or float8_e8m0fnu) is missing");
    if (t.dim() != 2 || t.size(0) != of.rows || t.size(1) != blocks || (blocks > 1 && of.rows > 0 && t.stride(1) != 1))
        refuse(s + " must be " + std::to_string(of.rows) + " x " + std::to_string(blocks) + " with contiguous rows");
    if (of.rows > 1 && t.stride(0) < blocks) refuse("the rows of " + s + " overlap");
    if (t.device() != like.t->device()) refuse(s + " is on another device");
    r.p = static_cast<const uint8_t *>(t.data_ptr());
    r.ld = of.rows > 1 ? t.stride(0) : blocks;
    return r;
}

at::Tensor fresh(const Matrix &like, at::IntArrayRef sizes, at::ScalarType type)
{
    return at::empty(sizes, like.t->options().dtype(type).requires_grad(false));
}

struct Room {
    at::Tensor held;
    void *p = nullptr;
    size_t bytes = 0;
};
Room room(PyObject *o, size_t need, const Matrix &like)
{
    Room r;
    if (o == Py_None) {
        if (need == 0) return r;
        r.held = fresh(like, {(int64_t)need}, at::kByte);
    } else {
        const char *what = "the workspace must be a contiguous uint8 tensor on the device";
        if (!THPVariable_Check(o)) refuse(what, RCD_ERR_WORKSPACE);
        r.held = THPVariable_Unpack(o);
        if (r.held.scalar_type() != at::kByte || !r.held.is_contiguous() || r.held.device() != like.t->device()) refuse(what, RCD_ERR_WORKSPACE);
    }
    r.p = r.held.data_ptr();
    r.bytes = (size_t)r.held.numel();
    return r;
}

long long number(PyObject *o)
{
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw python_error();
    return v;
}
bool truth(PyObject *o)
{
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw python_error();
    return v != 0;
}
void *stream(PyObject *o) { return reinterpret_cast<void *>((intptr_t)number(o)); }

PyObject *wrap(const at::Tensor &t)
{
    if (t.defined()) return THPVariable_Wrap(t);
    Py_RETURN_NONE;
}
template <typename... T> PyObject *tuple(const T &...t)
{
    PyObject *r = PyTuple_New(sizeof...(T));
    if (!r) throw python_error();
    Py_ssize_t i = 0;
    (PyTuple_SET_ITEM(r, i++, wrap(t)), ...);
    return r;
}

void *p(const at::Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; }

void expect(Py_ssize_t n, Py_ssize_t want)
{
    if (n != want) refuse("wrong number of arguments");
}

// The result of a product: `out` if there is one, else a new matrix of out_type (a code, -1: that of a, bfloat16 for 8 bits).
struct Result {
    at::Tensor t;
    Matrix m;
};
Result result(PyObject *out, PyObject *out_type, const Matrix &a, int64_t rows, int64_t cols)
{
    const long long code = number(out_type);
    at::ScalarType type = code == RCD_F32 ? at::kFloat : code == RCD_BF16 ? at::kBFloat16 : a.type == at::kFloat8_e4m3fn ? at::kBFloat16 : a.type;
    Result r;
    if (out == Py_None) {
        r.t = fresh(a, {rows, cols}, type);
        r.m.t = &r.t;
        r.m.rows = rows;
        r.m.cols = cols;
        r.m.ld = std::max<int64_t>(cols, 1);
        r.m.type = type;
        return r;
    }
    r.m = matrix("out", out, rows, cols, code >= 0 ? &type : nullptr, &a);
    if (r.m.type == at::kFloat8_e4m3fn) refuse("out must be float32 or bfloat16", RCD_ERR_UNSUPPORTED);
    r.t = *r.m.t;
    if (!r.t.is_inference()) r.t.unsafeGetTensorImpl()->bump_version();      // (autograd's check of what it has kept of it)
    return r;
}

#define MARSHAL_BEGIN \
    HANDLE_TH_ERRORS  \
    try {
#define MARSHAL_END                        \
    }                                      \
    catch (const Refusal &r) { return raise(r); } \
    END_HANDLE_TH_ERRORS

// x, weight, eps, residual, quantize, want_sum, want_rstd, stream -> (y, scale, sum, rstd)
PyObject *rms_norm(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    MARSHAL_BEGIN
    expect(n, 8);
    const Matrix x = matrix("x", a[0], -1, -1, nullptr, nullptr);
    const Matrix r = optional_matrix("residual", a[3], x.rows, x.cols, x.type, x);
    const void *w = vector("weight", a[1], x.cols, x.type, x);
    const double eps = PyFloat_AsDouble(a[2]);
    if (eps == -1.0 && PyErr_Occurred()) throw python_error();
    const bool quantize = truth(a[4]);
    const int64_t blocks = (x.cols + BLOCK - 1) / BLOCK;
    const int code = code_of(x.type);
    at::Tensor y = fresh(x, {x.rows, x.cols}, quantize ? at::kFloat8_e4m3fn : x.type), s, sum, rstd;
    if (quantize) s = fresh(x, {x.rows, blocks}, at::kFloat8_e8m0fnu);
    if (truth(a[5])) sum = fresh(x, {x.rows, x.cols}, x.type);
    if (truth(a[6])) rstd = fresh(x, {x.rows}, at::kFloat);
    void *const on = stream(a[7]);
    run([&] {
        return rcd_rms_norm(x.p(), code, x.rows, x.cols, x.ld, r.p(), r.ld, w, (float)eps, p(sum), x.cols, p(y),
                            quantize ? RCD_MXFP8 : code, x.cols, (uint8_t *)p(s), blocks, (float *)p(rstd), on);
    });
    return tuple(y, s, sum, rstd);
    MARSHAL_END
}

// dy, h, rstd, weight, dsum, want_dweight, workspace, stream -> (dx, dweight)
PyObject *rms_norm_backward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    MARSHAL_BEGIN
    expect(n, 8);
    const Matrix dy = matrix("dy", a[0], -1, -1, nullptr, nullptr);
    const Matrix h = matrix("h", a[1], dy.rows, dy.cols, &dy.type, &dy);
    if (a[2] == Py_None) refuse("rstd is missing");
    const float *rstd = (const float *)vector("rstd", a[2], dy.rows, at::kFloat, dy);
    const void *w = vector("weight", a[3], dy.cols, dy.type, dy);
    const Matrix ds = optional_matrix("dsum", a[4], dy.rows, dy.cols, dy.type, dy);
    const bool want = truth(a[5]);
    at::Tensor dx = fresh(dy, {dy.rows, dy.cols}, dy.type), dw;
    if (want) dw = fresh(dy, {dy.cols}, dy.type);
    const Room ws = room(a[6], want ? rcd_rms_norm_backward_workspace_bytes(dy.rows, dy.cols) : 0, dy);
    void *const on = stream(a[7]);
    run([&] {
        return rcd_rms_norm_backward(dy.p(), code_of(dy.type), dy.rows, dy.cols, dy.ld, h.p(), h.ld, rstd, w, ds.p(), ds.ld, p(dx), dy.cols,
                                     p(dw), ws.p, ws.bytes, on);
    });
    return tuple(dx, dw);
    MARSHAL_END
}

// x, stream -> (elements, scales)
PyObject *quantize_mxfp8(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    MARSHAL_BEGIN
    expect(n, 2);
    const Matrix x = matrix("x", a[0], -1, -1, nullptr, nullptr);
    const int64_t blocks = (x.cols + BLOCK - 1) / BLOCK;
    at::Tensor q = fresh(x, {x.rows, x.cols}, at::kFloat8_e4m3fn), s = fresh(x, {x.rows, blocks}, at::kFloat8_e8m0fnu);
    void *const on = stream(a[1]);
    run([&] {
        return rcd_quantize_mxfp8(x.p(), code_of(x.type), x.rows, x.cols, x.ld, (uint8_t *)p(q), x.cols, (uint8_t *)p(s), blocks, on);
    });
    return tuple(q, s);
    MARSHAL_END
}

// a, w, bias, act, residual, a_scale, w_scale, out_type, want_preact, out, workspace, stream -> (y, z)
PyObject *linear(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    MARSHAL_BEGIN
    expect(n, 12);
    const Matrix m = matrix("a", a[0], -1, -1, nullptr, nullptr);
    const Matrix w = matrix("w", a[1], -1, m.cols, &m.type, &m);
    const int64_t M = m.rows, N = w.rows, K = m.cols;
    const Scale sa = scale("a_scale", a[5], m, m), sw = scale("w_scale", a[6], w, m);
    const Result y = result(a[9], a[7], m, M, N);
    const void *b = vector("bias", a[2], N, y.m.type, m);
    const Matrix r = optional_matrix("residual", a[4], M, N, y.m.type, m);
    at::Tensor z;
    if (truth(a[8])) z = fresh(m, {M, N}, at::kFloat);
    const int code = code_of(m.type), act = (int)number(a[3]);
    const Room ws = room(a[10], rcd_linear_workspace_bytes(M, N, K, code), m);
    void *const on = stream(a[11]);
    run([&] {
        return rcd_linear(m.p(), sa.p, m.ld, sa.ld, w.p(), sw.p, w.ld, sw.ld, code, code_of(y.m.type), M, N, K, b, act, r.p(), r.ld,
                          (float *)p(z), N, p(y.t), y.m.ld, ws.p, ws.bytes, on);
    });
    return tuple(y.t, z);
    MARSHAL_END
}

// dy, a, w, preact, act, want_da, want_dw, want_dbias, workspace, stream -> (da, dw, dbias)
PyObject *linear_backward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    MARSHAL_BEGIN
    expect(n, 10);
    const Matrix dy = matrix("dy", a[0], -1, -1, nullptr, nullptr);
    const Matrix m = matrix("a", a[1], dy.rows, -1, &dy.type, &dy);
    const int64_t M = dy.rows, N = dy.cols, K = m.cols;
    const Matrix w = matrix("w", a[2], N, K, &dy.type, &dy);
    const int code = code_of(dy.type), act = (int)number(a[4]);
    if (a[3] == Py_None && act != RCD_ACT_NONE) refuse("preact is missing");
    const Matrix z = optional_matrix("preact", a[3], M, N, at::kFloat, dy);
    at::Tensor da, dw, db;
    if (truth(a[5])) da = fresh(dy, {M, K}, dy.type);
    if (truth(a[6])) dw = fresh(dy, {N, K}, dy.type);
    if (truth(a[7])) db = fresh(dy, {N}, dy.type);
    const Room ws = room(a[8], rcd_linear_backward_workspace_bytes(M, N, K, code), dy);
    void *const on = stream(a[9]);
    run([&] {
        return rcd_linear_backward(dy.p(), dy.ld, m.p(), m.ld, w.p(), w.ld, code, M, N, K, (const float *)z.p(), z.ld, act, p(da), K, p(dw),
                                   K, p(db), ws.p, ws.bytes, on);
    });
    return tuple(da, dw, db);
    MARSHAL_END
}

// a, w_gate, w_up, act, a_scale, gate_scale, up_scale, out_type, want_saved, out, workspace, stream -> (h, saved)
PyObject *gated_linear(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    MARSHAL_BEGIN
    expect(n, 12);
    const Matrix m = matrix("a", a[0], -1, -1, nullptr, nullptr);
    const Matrix g = matrix("w_gate", a[1], -1, m.cols, &m.type, &m);
    const int64_t M = m.rows, F = g.rows, K = m.cols;
    const Matrix u = matrix("w_up", a[2], F, K, &m.type, &m);
    const Scale sa = scale("a_scale", a[4], m, m), sg = scale("gate_scale", a[5], g, m), su = scale("up_scale", a[6], u, m);
    const Result h = result(a[9], a[7], m, M, F);
    at::Tensor saved;
    if (truth(a[8])) saved = fresh(m, {M, F, 2}, at::kFloat);
    const int code = code_of(m.type), act = (int)number(a[3]);
    const Room ws = room(a[10], rcd_gated_linear_workspace_bytes(M, F, K, code), m);
    void *const on = stream(a[11]);
    run([&] {
        return rcd_gated_linear(m.p(), sa.p, m.ld, sa.ld, g.p(), sg.p, g.ld, sg.ld, u.p(), su.p, u.ld, su.ld, code, code_of(h.m.type), M, F, K,
                                act, (float *)p(saved), p(h.t), h.m.ld, ws.p, ws.bytes, on);
    });
    return tuple(h.t, saved);
    MARSHAL_END
}

// dh, a, w_gate, w_up, saved, act, want_da, want_dw, workspace, stream -> (da, dw_gate, dw_up)
PyObject *gated_linear_backward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    MARSHAL_BEGIN
    expect(n, 10);
    const Matrix dh = matrix("dh", a[0], -1, -1, nullptr, nullptr);
    const Matrix m = matrix("a", a[1], dh.rows, -1, &dh.type, &dh);
    const int64_t M = dh.rows, F = dh.cols, K = m.cols;
    const Matrix g = matrix("w_gate", a[2], F, K, &dh.type, &dh), u = matrix("w_up", a[3], F, K, &dh.type, &dh);
    const at::Tensor *saved = tensor(a[4]);
    if (saved) no_history("saved", *saved);
    if (!saved || saved->dim() != 3 || saved->size(0) != M || saved->size(1) != F || saved->size(2) != 2 || saved->scalar_type() != at::kFloat ||
        !saved->is_contiguous() || saved->device() != dh.t->device())
        refuse("saved must be what gated_linear returned");
    const int code = code_of(dh.type), act = (int)number(a[5]);
    at::Tensor da, dg, du;
    if (truth(a[6])) da = fresh(dh, {M, K}, dh.type);
    if (truth(a[7])) {
        dg = fresh(dh, {F, K}, dh.type);
        du = fresh(dh, {F, K}, dh.type);
    }
    const Room ws = room(a[8], rcd_gated_linear_backward_workspace_bytes(M, F, K, code), dh);
    void *const on = stream(a[9]);
    run([&] {
        return rcd_gated_linear_backward(dh.p(), dh.ld, m.p(), m.ld, g.p(), g.ld, u.p(), u.ld, code, M, F, K, (const float *)saved->data_ptr(),
                                         act, p(da), K, p(dg), K, p(du), K, ws.p, ws.bytes, on);
    });
    return tuple(da, dg, du);
    MARSHAL_END
}

// ---- attention ------------------------------------------------------------------------------------------------------------

// Rows of heads: (batch, rows, heads, d), or (rows, heads, d) where offsets say which sequence a row belongs to.
struct Rows {
    const at::Tensor *t = nullptr;
    int64_t batch = 0, rows = 0, heads = 0, d = 0;
    rcd_heads h{};
};

// The strides of a tensor of heads; written: its elements may not share memory.
rcd_heads strides(const std::string &n, const at::Tensor &t, bool written)
{
    const int64_t dims = t.dim();
    if (t.size(dims - 1) > 1 && t.stride(dims - 1) != 1 && t.numel() > 0) refuse("the last dimension of " + n + " must be contiguous");
    int64_t s[4] = {0, 0, 0, 0};                // (of a dimension of one the stride means nothing)
    for (int64_t i = 0; i < dims; ++i) s[4 - dims + i] = t.size(i) > 1 ? t.stride(i) : 0;
    if (written && t.numel() > 0) {
        std::pair<int64_t, int64_t> by[4];
        int count = 0;
        for (int64_t i = 0; i < dims; ++i)
            if (t.size(i) > 1) by[count++] = {t.stride(i), t.size(i)};
        std::sort(by, by + count);
        int64_t extent = 1;
        for (int i = 0; i < count; ++i) {
            if (by[i].first < extent) refuse("elements of " + n + " overlap");
            extent += by[i].first * (by[i].second - 1);
        }
    }
    return {t.data_ptr(), s[0], s[1], s[2]};
}

Rows rows(const char *name, PyObject *o, bool ragged, const at::ScalarType *type, const at::Tensor *like, bool written = false)
{
    const std::string n = name, shape = ragged ? "(rows, heads, d)" : "(batch, rows, heads, d)";
    if (!THPVariable_Check(o)) refuse(n + " must be a tensor " + shape);
    Rows r;
    r.t = &THPVariable_Unpack(o);
    const at::Tensor &t = *r.t;
    no_history(n, t);
    if (t.dim() != (ragged ? 3 : 4)) refuse(n + " must be a tensor " + shape + (ragged ? " where it has offsets" : ""));
    if (!t.is_cuda()) refuse(n + ": device tensor expected (there is no CPU path)", NOT_ON_DEVICE);
    if (t.scalar_type() != at::kFloat && t.scalar_type() != at::kBFloat16) refuse(n + ": float32 or bfloat16 expected", RCD_ERR_UNSUPPORTED);
    if (type && t.scalar_type() != *type) refuse(n + " must be " + c10::toString(*type), RCD_ERR_UNSUPPORTED);
    if (like) {
        if (t.device() != like->device()) refuse(n + " is on another device");
    } else if (c10::impl::VirtualGuardImpl(at::kCUDA).getDevice() != t.device()) {
        refuse(n + " is on another device than the current one");
    }
    const int64_t d = t.dim();
    r.batch = ragged ? 1 : t.size(0);
    r.rows = t.size(d - 3);
    r.heads = t.size(d - 2);
    r.d = t.size(d - 1);
    r.h = strides(n, t, written);
    return r;
}
void same_shape(const char *name, const Rows &r, const Rows &as, const char *of)
{
    if (r.t->sizes() != as.t->sizes()) refuse(std::string(name) + " must have the shape of " + of);
}
const int32_t *indices(const char *name, PyObject *o, int64_t least, int64_t n, const at::Tensor &like, int64_t *count)
{
    if (o == Py_None) return nullptr;
    const std::string s = name;
    if (!THPVariable_Check(o)) refuse(s + " must be a contiguous int32 vector");
    const at::Tensor &t = THPVariable_Unpack(o);
    if (t.dim() != 1 || t.scalar_type() != at::kInt || !t.is_contiguous()) refuse(s + " must be a contiguous int32 vector");
    if (t.device() != like.device()) refuse(s + " is on another device");
    if (t.size(0) < least || (n >= 0 && t.size(0) != n)) refuse(s + " must have " + std::to_string(n >= 0 ? n : least) + " elements" + (n >= 0 ? "" : " at least"));
    if (count) *count = t.size(0);
    return static_cast<const int32_t *>(t.data_ptr());
}

// What both calls are told of the sequences: a[0] q_offsets, k_offsets, k_lengths, longest_q, longest_k, scale, causal, bias, a[8] borders.
struct Call {
    rcd_attention_shape s{};
    Rows q, k, v;
    at::ScalarType type;
    const at::Tensor *bias = nullptr, *q_offsets = nullptr, *k_offsets = nullptr, *k_lengths = nullptr;
};
Call attention_call(PyObject *q, PyObject *k, PyObject *v, PyObject *const *a)
{
    Call c;
    const bool q_ragged = a[0] != Py_None, k_ragged = a[1] != Py_None;
    c.q = rows("q", q, q_ragged, nullptr, nullptr);
    const at::Tensor &like = *c.q.t;
    c.type = like.scalar_type();
    c.k = rows("k", k, k_ragged, &c.type, &like);
    c.v = rows("v", v, k_ragged, &c.type, &like);
    same_shape("v", c.v, c.k, "k");
    if (c.k.d != c.q.d) refuse("k must have heads of q's size");
    int64_t ends = -1;
    c.s.q_offsets_dev = indices("q_offsets", a[0], 1, -1, like, &ends);
    c.s.k_offsets_dev = indices("k_offsets", a[1], 1, ends, like, &ends);
    c.s.batch = ends >= 0 ? ends - 1 : c.q.batch;
    if ((!q_ragged && c.q.batch != c.s.batch) || (!k_ragged && c.k.batch != c.s.batch)) refuse("q and k must have the same number of sequences");
    if (k_ragged && a[2] != Py_None) refuse("k_lengths go without k_offsets");
    c.s.k_lengths_dev = indices("k_lengths", a[2], 0, c.s.batch, like, nullptr);
    c.q_offsets = tensor(a[0]);
    c.k_offsets = tensor(a[1]);
    c.k_lengths = tensor(a[2]);
    c.s.longest_q = number(a[3]);
    c.s.longest_k = number(a[4]);
    if (c.s.longest_q < 0 || c.s.longest_k < 0) refuse("longest_q and longest_k must not be negative");
    if (c.k.heads < 1 || c.q.heads < 1 || c.q.heads % c.k.heads != 0) refuse("q's heads must be a multiple of k's");
    if (c.q.d < 1) refuse("heads must have elements");
    if (c.q.d > 128) refuse("heads of 128 elements at most", RCD_ERR_UNSUPPORTED);
    const double scale = a[5] == Py_None ? 1.0 / std::sqrt((double)c.q.d) : PyFloat_AsDouble(a[5]);
    if (scale == -1.0 && PyErr_Occurred()) throw python_error();
    c.s.scale = (float)scale;
    c.s.causal = truth(a[6]);
    c.s.dt = code_of(c.type);
    c.s.heads = c.q.heads;
    c.s.kv_heads = c.k.heads;
    c.s.d = c.q.d;
    c.s.q_rows = c.q.rows;
    c.s.k_rows = c.k.rows;
    if (a[7] != Py_None) {
        if (!THPVariable_Check(a[7])) refuse("bias must be a contiguous tensor (buckets, heads)");
        c.bias = &THPVariable_Unpack(a[7]);
        no_history("bias", *c.bias);
        if (c.bias->dim() != 2 || c.bias->size(1) != c.q.heads || !c.bias->is_contiguous()) refuse("bias must be a contiguous tensor (buckets, heads)");
        if (c.bias->scalar_type() != at::kFloat && c.bias->scalar_type() != c.type) refuse("bias must be float32 or of q's type", RCD_ERR_UNSUPPORTED);
        if (c.bias->device() != like.device()) refuse("bias is on another device");
        char *borders = nullptr;
        Py_ssize_t bytes = 0;
        if (PyBytes_AsStringAndSize(a[8], &borders, &bytes) < 0) throw python_error();
        c.s.bias_dev = c.bias->data_ptr();
        c.s.bias_dt = code_of(c.bias->scalar_type());
        c.s.buckets = c.bias->size(0);
        const int64_t each = c.s.causal ? c.s.buckets : c.s.buckets / 2;
        if (bytes < (each - 1) * 4) refuse("too few borders");
        c.s.borders_host = reinterpret_cast<const int32_t *>(borders);
    }
    return c;
}

// A result in the shape of `as`: `given`, or a new contiguous one (its rows that belong to no sequence are cleared by the call).
struct Made {
    at::Tensor t;
    rcd_heads h{};
};
Made made(const char *name, PyObject *given, const Rows &as, const Call &c)
{
    Made m;
    if (given == Py_None) {
        m.t = at::empty(as.t->sizes(), as.t->options().requires_grad(false));
        m.h = strides(name, m.t, true);
        return m;
    }
    const Rows r = rows(name, given, as.t->dim() == 3, &c.type, c.q.t, true);
    same_shape(name, r, as, "what it is of");
    m.t = *r.t;
    m.h = r.h;
    if (!m.t.is_inference()) m.t.unsafeGetTensorImpl()->bump_version();
    return m;
}
overlap::Array places(const at::Tensor &t)
{
    overlap::Array a;
    const int64_t dims = t.dim(), e = t.element_size();
    a.p = reinterpret_cast<uintptr_t>(t.data_ptr());
    if (t.is_contiguous()) {
        a.run = t.numel() * e;
        return a;
    }
    a.run = t.size(dims - 1) * e;               // (the last dimension of everything here is contiguous)
    for (int64_t i = 0; i + 1 < dims; ++i) a.dim(t.stride(i) * e, t.size(i));
    return a;
}
// A result that shares elements with an operand or another result would be read, or written again, while it is written.  (Where thousands of steps do
// not settle it, which the views of one buffer never take, it is the caller's part.)
void apart(const char *name, const Made &m, std::initializer_list<const at::Tensor *> others, const Room &ws, size_t need)
{
    const overlap::Array mine = places(m.t);
    overlap::Array used;
    used.p = reinterpret_cast<uintptr_t>(ws.p);
    used.run = (int64_t)std::min(need, ws.bytes);
    bool shared = overlap::of(mine, used) == overlap::SHARED;
    for (const at::Tensor *o : others) shared = shared || (o && overlap::of(mine, places(*o)) == overlap::SHARED);
    if (shared) refuse(std::string(name) + " shares elements with an operand, another result or the workspace");
}
Room room(PyObject *o, size_t need, const at::Tensor &like)
{
    Matrix m;
    m.t = &like;
    return room(o, need, m);
}

// q, k, v, [nine of attention_call], out, want_saved, workspace, stream -> (out, saved)
PyObject *attention(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    MARSHAL_BEGIN
    expect(n, 16);
    const Call c = attention_call(a[0], a[1], a[2], a + 3);
    const Made out = made("out", a[12], c.q, c);
    at::Tensor saved;
    if (truth(a[13])) {
        auto sizes = c.q.t->sizes().vec();
        sizes.back() = 2;
        saved = at::empty(sizes, c.q.t->options().dtype(at::kFloat).requires_grad(false));
    }
    const size_t need = rcd_attention_workspace_bytes(&c.s);
    const Room ws = room(a[14], need, *c.q.t);
    if (a[12] != Py_None) apart("out", out, {c.q.t, c.k.t, c.v.t, c.bias, c.q_offsets, c.k_offsets, c.k_lengths}, ws, need);
    void *const on = stream(a[15]);
    const int clear = a[12] == Py_None;
    run([&] { return rcd_attention(&c.s, &c.q.h, &c.k.h, &c.v.h, &out.h, (float *)p(saved), clear, ws.p, ws.bytes, on); });
    return tuple(out.t, saved);
    MARSHAL_END
}

// dout, q, k, v, out, saved, [nine of attention_call], dq, dk, dv, want_dbias, workspace, stream -> (dq, dk, dv, dbias)
PyObject *attention_backward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    MARSHAL_BEGIN
    expect(n, 21);
    const Call c = attention_call(a[1], a[2], a[3], a + 6);
    const bool q_ragged = c.q.t->dim() == 3;
    const Rows dout = rows("dout", a[0], q_ragged, &c.type, c.q.t), out = rows("out", a[4], q_ragged, &c.type, c.q.t);
    same_shape("dout", dout, c.q, "q");
    same_shape("out", out, c.q, "q");
    const at::Tensor *saved = tensor(a[5]);
    auto sizes = c.q.t->sizes().vec();
    sizes.back() = 2;
    if (saved) no_history("saved", *saved);
    if (!saved || saved->sizes() != at::IntArrayRef(sizes) || saved->scalar_type() != at::kFloat || !saved->is_contiguous() ||
        saved->device() != c.q.t->device())
        refuse("saved must be what attention returned");
    const int given = (a[15] != Py_None) + (a[16] != Py_None) + (a[17] != Py_None);
    if (given != 0 && given != 3) refuse("grads must be (dq, dk, dv)");
    const Made dq = made("dq", a[15], c.q, c), dk = made("dk", a[16], c.k, c), dv = made("dv", a[17], c.v, c);
    at::Tensor dbias;
    if (c.bias && truth(a[18])) dbias = at::empty(c.bias->sizes(), c.bias->options().requires_grad(false));
    const size_t need = rcd_attention_backward_workspace_bytes(&c.s);
    const Room ws = room(a[19], need, *c.q.t);
    if (given) {
        for (const auto &[name, made] : {std::pair("dq", &dq), std::pair("dk", &dk), std::pair("dv", &dv)})
            apart(name, *made, {dout.t, c.q.t, c.k.t, c.v.t, out.t, saved, c.bias, c.q_offsets, c.k_offsets, c.k_lengths}, ws, need);
        apart("dq", dq, {&dk.t, &dv.t}, ws, need);
        apart("dk", dk, {&dv.t}, ws, need);
    }
    void *const on = stream(a[20]);
    run([&] {
        return rcd_attention_backward(&c.s, &dout.h, &c.q.h, &c.k.h, &c.v.h, &out.h, (const float *)saved->data_ptr(), &dq.h, &dk.h, &dv.h, p(dbias),
                                      given == 0, ws.p, ws.bytes, on);
    });
    return tuple(dq.t, dk.t, dv.t, dbias);
    MARSHAL_END
}

PyObject *set_error(PyObject *, PyObject *cls)
{
    Py_XDECREF(g_error);
    Py_INCREF(cls);
    g_error = cls;
    Py_RETURN_NONE;
}

#define FAST(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(rms_norm),        FAST(rms_norm_backward), FAST(quantize_mxfp8),        FAST(linear),
                         FAST(linear_backward), FAST(gated_linear),      FAST(gated_linear_backward), FAST(attention),       FAST(attention_backward),
                         {"set_error", set_error, METH_O, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_encoder", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

} // namespace

PyMODINIT_FUNC PyInit__encoder() { return PyModule_Create(&module_def); }
