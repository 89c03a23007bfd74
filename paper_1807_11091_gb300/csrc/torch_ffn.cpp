// torch_ffn.cpp -- the feed-forward operators on torch tensors: checks, outputs
// and scratch from torch's allocator, and the call of the C entry point on
// torch's current stream.  Everything else is behind the C ABI (sadmm.h).
//
// This is native because on a few tokens the host is what a call costs: with
// the same steps in Python a layer norm of four rows took 14 us a call, its
// kernel 2.  sadmm.py holds the functions' signatures and documentation and
// passes their arguments on by position.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/core/LegacyTypeDispatch.h>
#include <ATen/ops/empty_strided.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <dlfcn.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>
#include <optional>
#include <stdexcept>
#include <string>

#include "sadmm.h"

namespace {

// ------------------------------------------------------------- the library --

struct Entry {
    decltype(&sadmm_layernorm_fwd) layernorm_fwd;
    decltype(&sadmm_layernorm_bwd_workspace_size) layernorm_bwd_size;
    decltype(&sadmm_layernorm_bwd) layernorm_bwd;
    decltype(&sadmm_linear_fwd_workspace_size) linear_fwd_size;
    decltype(&sadmm_linear_fwd) linear_fwd;
    decltype(&sadmm_linear_bwd_workspace_size) linear_bwd_size;
    decltype(&sadmm_linear_bwd) linear_bwd;
    decltype(&sadmm_gated_fwd_workspace_size) gated_fwd_size;
    decltype(&sadmm_gated_fwd) gated_fwd;
    decltype(&sadmm_gated_bwd_workspace_size) gated_bwd_size;
    decltype(&sadmm_gated_bwd) gated_bwd;
} entry;
PyObject* error_class;  // sadmm.SadmmError

struct PythonError {};  // a Python exception is set

[[noreturn]] void fail(PyObject* type, const std::string& what)
{
    PyErr_SetString(type, what.c_str());
    throw PythonError();
}

void ok(int status, const char* where)
{
    if (status == SADMM_OK) return;
    PyObject* e = PyObject_CallFunction(error_class, "is", status, where);
    if (e) PyErr_SetObject(error_class, e);
    Py_XDECREF(e);
    throw PythonError();
}

// --------------------------------------------------------------- arguments --

using at::ScalarType;
using at::Tensor;

const char* type_name(ScalarType t) { return c10::toString(t); }

int dtype_of(ScalarType t, const char* name)
{
    if (t == at::kBFloat16) return SADMM_BF16;
    if (t == at::kFloat) return SADMM_FP32;
    fail(PyExc_TypeError, std::string(name) + " must be bf16 or fp32, got " + type_name(t));
}

const Tensor& tensor(PyObject* o, const char* name)
{
    if (!THPVariable_Check(o)) fail(PyExc_TypeError, std::string(name) + " must be a tensor");
    const Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda()) fail(PyExc_TypeError, std::string(name) + " must be a CUDA tensor");
    return t;
}

// The call's x.  Its other tensors have to be on the same device, where the kernels
// run that are handed their pointers.
struct Named {
    PyObject* o;
    const char* name;
};
const Tensor& first(PyObject* o, std::initializer_list<Named> others)
{
    const Tensor& x = tensor(o, "x");
    for (const Named& n : others) {
        if (n.o == Py_None) continue;
        const Tensor& t = tensor(n.o, n.name);
        if (t.device() != x.device())
            fail(PyExc_ValueError, std::string(n.name) + " is on " + t.device().str() + ", x on " + x.device().str());
    }
    return x;
}

const Tensor* tensor_or_none(PyObject* o, const char* name) { return o == Py_None ? nullptr : &tensor(o, name); }

ScalarType dtype_arg(PyObject* o, ScalarType otherwise)
{
    if (o == Py_None) return otherwise;
    if (!THPDtype_Check(o)) fail(PyExc_TypeError, "a dtype argument is not a torch.dtype");
    return reinterpret_cast<THPDtype*>(o)->scalar_type;
}

bool flag(PyObject* o)
{
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw PythonError();
    return v != 0;
}

int number(PyObject* o)
{
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) throw PythonError();
    if (v != (int)v) fail(PyExc_OverflowError, "integer argument out of range");
    return (int)v;
}

// A tensor as a matrix [rows][cols]: any leading dimensions that view as one.
// The stride of a single row is free and taken as its width's next multiple of 8.
struct Matrix {
    void* p = nullptr;
    int64_t ld = 0, rows = 0, cols = 0;
    ScalarType type = at::kBFloat16;
};

Matrix matrix(const Tensor& t, const char* name)
{
    const int64_t d = t.dim();
    if (d < 1) fail(PyExc_TypeError, std::string(name) + " needs a last dimension");
    Matrix m;
    m.cols = t.size(d - 1);
    if (t.stride(d - 1) != 1 && m.cols > 1)
        fail(PyExc_TypeError, std::string(name) + "'s last dimension must be contiguous");
    m.rows = 1;
    for (int64_t i = 0; i < d - 1; ++i) m.rows *= t.size(i);
    m.ld = (m.cols + 7) / 8 * 8;
    if (m.rows > 1) {
        // the row stride is that of the last leading dimension longer than 1, and the ones before it follow on
        int64_t i = d - 2;
        while (t.size(i) == 1) --i;
        m.ld = t.stride(i);
        int64_t next = m.ld * t.size(i);
        for (--i; i >= 0; --i) {
            if (t.size(i) == 1) continue;
            if (t.stride(i) != next)
                fail(PyExc_TypeError, std::string(name) + "'s leading dimensions do not view as one");
            next *= t.size(i);
        }
    }
    m.p = t.data_ptr();
    m.type = t.scalar_type();
    return m;
}

Matrix matrix_of(const Tensor& t, const char* name, int64_t rows, int64_t cols, std::optional<ScalarType> type)
{
    if (type && t.scalar_type() != *type)
        fail(PyExc_TypeError, std::string(name) + " must be " + type_name(*type) + ", got " + type_name(t.scalar_type()));
    const Matrix m = matrix(t, name);
    if (m.cols != cols || (rows >= 0 && m.rows != rows))
        fail(PyExc_ValueError, std::string(name) + " is " + std::to_string(m.rows) + " x " + std::to_string(m.cols) +
                                   ", not " + std::to_string(rows >= 0 ? rows : m.rows) + " x " + std::to_string(cols));
    return m;
}

// The pointer of a contiguous fp32 vector of n elements.
float* vector(const Tensor& t, int64_t n, const char* name)
{
    if (t.scalar_type() != at::kFloat || t.numel() != n || !t.is_contiguous())
        fail(PyExc_TypeError,
             std::string(name) + " must be a contiguous fp32 CUDA tensor of " + std::to_string(n) + " elements");
    return static_cast<float*>(t.data_ptr());
}
float* vector_or_none(PyObject* o, int64_t n, const char* name)
{
    return o == Py_None ? nullptr : vector(tensor(o, name), n, name);
}

// ----------------------------------------------------------------- outputs --

struct Output {
    Tensor t;  // undefined: not wanted
    void* p = nullptr;
    int64_t ld = 0;
};

// [rows of `like`][cols] in like's leading dimensions, row stride ld.
Output allocate(const Tensor& like, int64_t cols, int64_t ld, ScalarType type)
{
    int64_t size[16], stride[16];
    const int64_t d = like.dim();
    if (d > 16) fail(PyExc_ValueError, "more than 16 dimensions");
    size[d - 1] = cols;
    stride[d - 1] = 1;
    int64_t next = ld;
    for (int64_t i = d - 2; i >= 0; --i) {
        size[i] = like.size(i);
        stride[i] = next;
        next *= size[i];
    }
    Output o;
    o.t = at::empty_strided(at::IntArrayRef(size, d), at::IntArrayRef(stride, d), like.options().dtype(type));
    o.p = o.t.data_ptr();
    o.ld = ld;
    return o;
}

// Rows on 32-byte boundaries, so that the next call reads them where they lie.
Output new_rows(const Tensor& like, int64_t cols, ScalarType type)
{
    const int64_t step = type == at::kBFloat16 ? 16 : 8;
    return allocate(like, cols, (cols + step - 1) / step * step, type);
}

// A weight's gradient: the weight's shape and row stride.
Output like_weight(const Tensor& w, const Matrix& m, ScalarType type)
{
    return allocate(w, m.cols, m.rows > 1 && m.ld > m.cols ? m.ld : m.cols, type);
}

Output new_vector(const Tensor& like, int64_t n)
{
    Output o;
    const int64_t size[1] = {n}, stride[1] = {1};
    o.t = at::empty_strided(at::IntArrayRef(size, 1), at::IntArrayRef(stride, 1), like.options().dtype(at::kFloat));
    o.p = o.t.data_ptr();
    return o;
}

Output given(PyObject* o, const Matrix& m)
{
    Output r;
    r.t = THPVariable_Unpack(o);
    r.p = m.p;
    r.ld = m.ld;
    return r;
}

PyObject* wrap(const Output& o)
{
    if (!o.t.defined()) Py_RETURN_NONE;
    return THPVariable_Wrap(o.t);
}

template <int N>
PyObject* wrap_all(const Output (&o)[N])
{
    PyObject* t = PyTuple_New(N);
    if (!t) throw PythonError();
    for (int i = 0; i < N; ++i) {
        PyObject* v = wrap(o[i]);
        if (!v) {
            Py_DECREF(t);
            throw PythonError();
        }
        PyTuple_SET_ITEM(t, i, v);
    }
    return t;
}

// ------------------------------------------------------------------ stream --

// The call's device, stream and scratch.  A stream other than torch's current one
// (given as its handle) is the current one while the call allocates: a block of the
// allocator's pool of another stream may be one that this stream's kernels, already
// enqueued, still use.  What the call is given is recorded on the stream, and what it
// returns on the caller's, where it will be read, so that neither's memory is handed
// out while it is in use there.  That the inputs are ready on the stream is for the
// caller to see to.
struct Call {
    c10::cuda::OptionalCUDAGuard guard;
    c10::cuda::OptionalCUDAStreamGuard current;
    at::AutoDispatchBelowADInplaceOrView no_autograd;
    c10::Device device;
    bool other;
    cudaStream_t stream;
    std::optional<c10::cuda::CUDAStream> callers, own;
    Tensor scratch;

    Call(const Tensor& t, PyObject* s) : device(t.device()), other(false)
    {
        if (device.index() != c10::cuda::current_device()) guard.set_device(device);
        callers = c10::cuda::getCurrentCUDAStream(device.index());
        stream = callers->stream();
        if (s == Py_None) return;
        const cudaStream_t given = static_cast<cudaStream_t>(PyLong_AsVoidPtr(s));
        if (PyErr_Occurred()) throw PythonError();
        if (given == stream) return;
        other = true;
        stream = given;
        own = c10::cuda::getStreamFromExternal(given, device.index());
        current.reset_stream(*own);
    }
    void* workspace(const Tensor& like, size_t bytes)
    {
        if (!bytes) return nullptr;
        const int64_t size[1] = {(int64_t)bytes}, stride[1] = {1};
        scratch = at::empty_strided(at::IntArrayRef(size, 1), at::IntArrayRef(stride, 1), like.options().dtype(at::kByte));
        return scratch.data_ptr();
    }
    // Before the launch: the n arguments of the call and its outputs.
    template <int N>
    void uses(PyObject* const* v, int n, const Output (&o)[N]) const
    {
        if (!other) return;
        for (int i = 0; i < n; ++i) {
            if (!THPVariable_Check(v[i])) continue;
            const Tensor& t = THPVariable_Unpack(v[i]);
            if (t.is_cuda()) t.record_stream(own->unwrap());  // (an argument that is not read may lie anywhere)
        }
        for (const Output& x : o)
            if (x.t.defined()) x.t.record_stream(callers->unwrap());
    }
};

// Rows off 16-byte boundaries are copied to scratch first.
bool apart(const Matrix& m) { return ((reinterpret_cast<uintptr_t>(m.p) | (uintptr_t)(m.ld * 2)) & 15) != 0; }

int width(int64_t n)
{
    if (n > 0x7fffffff) fail(PyExc_ValueError, "a matrix is too wide");
    return (int)n;
}

// --------------------------------------------------------------- operators --

// x, gamma, beta, eps, out_dtype, stats, out, stream
PyObject* layer_norm(PyObject* const* v)
{
    const Tensor& x = first(v[0], {{v[1], "gamma"}, {v[2], "beta"}, {v[6], "out"}});
    const Matrix m = matrix(x, "x");
    const double eps = PyFloat_AsDouble(v[3]);
    if (eps == -1.0 && PyErr_Occurred()) throw PythonError();
    const bool stats = flag(v[5]);
    Call call(x, v[7]);
    Output o[3];
    o[0] = v[6] != Py_None ? given(v[6], matrix_of(tensor(v[6], "out"), "out", m.rows, m.cols, std::nullopt))
                           : new_rows(x, m.cols, dtype_arg(v[4], m.type));
    if (stats) {
        o[1] = new_vector(x, m.rows);
        o[2] = new_vector(x, m.rows);
    }
    sadmm_layernorm_fwd_args a = {};
    a.rows = m.rows;
    a.cols = width(m.cols);
    a.x = m.p;
    a.ldx = m.ld;
    a.xdt = dtype_of(m.type, "x");
    a.gamma = vector_or_none(v[1], m.cols, "gamma");
    a.beta = vector_or_none(v[2], m.cols, "beta");
    a.eps = (float)eps;
    a.y = o[0].p;
    a.ldy = o[0].ld;
    a.ydt = dtype_of(o[0].t.scalar_type(), "out");
    a.mean = static_cast<float*>(o[1].p);
    a.rstd = static_cast<float*>(o[2].p);
    call.uses(v, 8, o);
    ok(entry.layernorm_fwd(&a, call.stream), "sadmm_layernorm_fwd");
    return stats ? wrap_all(o) : wrap(o[0]);
}

// dy, x, mean, rstd, gamma, dres, want_dx, want_dgamma, want_dbeta, stream
PyObject* layer_norm_backward(PyObject* const* v)
{
    const Tensor& x = first(v[1], {{v[0], "dy"}, {v[2], "mean"}, {v[3], "rstd"}, {v[4], "gamma"}, {v[5], "dres"}});
    const Matrix m = matrix(x, "x");
    const Matrix dy = matrix_of(tensor(v[0], "dy"), "dy", m.rows, m.cols, std::nullopt);
    Matrix dres;
    if (const Tensor* t = tensor_or_none(v[5], "dres")) dres = matrix_of(*t, "dres", m.rows, m.cols, m.type);
    Call call(x, v[9]);
    Output o[3];
    if (flag(v[6])) o[0] = new_rows(x, m.cols, m.type);
    if (flag(v[7])) o[1] = new_vector(x, m.cols);
    if (flag(v[8])) o[2] = new_vector(x, m.cols);
    sadmm_layernorm_bwd_args a = {};
    a.rows = m.rows;
    a.cols = width(m.cols);
    a.x = m.p;
    a.ldx = m.ld;
    a.xdt = dtype_of(m.type, "x");
    a.dy = dy.p;
    a.lddy = dy.ld;
    a.dydt = dtype_of(dy.type, "dy");
    a.gamma = vector_or_none(v[4], m.cols, "gamma");
    a.mean = vector(tensor(v[2], "mean"), m.rows, "mean");
    a.rstd = vector(tensor(v[3], "rstd"), m.rows, "rstd");
    a.dres = dres.p;
    a.lddres = dres.ld;
    a.dx = o[0].p;
    a.lddx = o[0].ld;
    a.dgamma = static_cast<float*>(o[1].p);
    a.dbeta = static_cast<float*>(o[2].p);
    const size_t n = entry.layernorm_bwd_size(&a);
    void* ws = call.workspace(x, n);
    call.uses(v, 10, o);
    ok(entry.layernorm_bwd(&a, ws, n, call.stream), "sadmm_layernorm_bwd");
    return wrap_all(o);
}

// x, W, bias, residual, act, out_dtype, save, out, stream
PyObject* linear(PyObject* const* v)
{
    const Tensor& x = first(v[0], {{v[1], "W"}, {v[2], "bias"}, {v[3], "residual"}, {v[7], "out"}});
    const Matrix m = matrix_of(x, "x", -1, x.dim() ? x.size(-1) : 0, at::kBFloat16);
    const Matrix w = matrix_of(tensor(v[1], "W"), "W", -1, m.cols, at::kBFloat16);
    const Tensor* residual = tensor_or_none(v[3], "residual");
    const bool save = flag(v[6]);
    Call call(x, v[8]);
    Output o[2];
    o[0] = v[7] != Py_None
               ? given(v[7], matrix_of(tensor(v[7], "out"), "out", m.rows, w.rows, std::nullopt))
               : new_rows(x, w.rows, dtype_arg(v[5], residual ? residual->scalar_type() : at::kBFloat16));
    if (save) o[1] = new_rows(x, w.rows, at::kBFloat16);
    Matrix r;
    if (residual) r = matrix_of(*residual, "residual", m.rows, w.rows, o[0].t.scalar_type());
    sadmm_linear_fwd_args a = {};
    a.tokens = m.rows;
    a.n_in = width(m.cols);
    a.n_out = width(w.rows);
    a.x = m.p;
    a.ldx = m.ld;
    a.w = w.p;
    a.ldw = w.ld;
    a.bias = vector_or_none(v[2], w.rows, "bias");
    a.residual = r.p;
    a.ldr = r.ld;
    a.act = number(v[4]);
    a.y = o[0].p;
    a.ldy = o[0].ld;
    a.ydt = dtype_of(o[0].t.scalar_type(), "out");
    a.z = o[1].p;
    a.ldz = o[1].ld;
    const size_t n = apart(m) || apart(w) ? entry.linear_fwd_size(&a) : 0;
    void* ws = call.workspace(x, n);
    call.uses(v, 9, o);
    ok(entry.linear_fwd(&a, ws, n, call.stream), "sadmm_linear_fwd");
    return save ? wrap_all(o) : wrap(o[0]);
}

// dy, x, W, z, act, want_dx, want_dw, want_db, dx_dtype, dw_dtype, stream
PyObject* linear_backward(PyObject* const* v)
{
    const int act = number(v[4]);
    const Tensor& x = first(v[1], {{v[0], "dy"}, {v[2], "W"}, {act != SADMM_ACT_NONE ? v[3] : Py_None, "z"}});
    const Tensor &dyt = tensor(v[0], "dy"), &wt = tensor(v[2], "W");
    const Matrix dy = matrix(dyt, "dy");
    const Matrix m = matrix_of(x, "x", dy.rows, x.dim() ? x.size(-1) : 0, at::kBFloat16);
    const Matrix w = matrix_of(wt, "W", dy.cols, m.cols, at::kBFloat16);
    Matrix z;
    if (act != SADMM_ACT_NONE) {
        if (v[3] == Py_None) fail(PyExc_TypeError, "the gradient of an activation needs z");
        z = matrix_of(tensor(v[3], "z"), "z", dy.rows, dy.cols, at::kBFloat16);
    }
    // types also of what is not wanted: the library then adds up in the same order whatever else is wanted
    const ScalarType xt = dtype_arg(v[8], at::kBFloat16), dwt = dtype_arg(v[9], at::kBFloat16);
    Call call(x, v[10]);
    Output o[3];
    if (flag(v[5])) o[0] = new_rows(x, m.cols, xt);
    if (flag(v[6])) o[1] = like_weight(wt, w, dwt);
    if (flag(v[7])) o[2] = new_vector(x, dy.cols);
    sadmm_linear_bwd_args a = {};
    a.tokens = dy.rows;
    a.n_in = width(m.cols);
    a.n_out = width(dy.cols);
    a.dy = dy.p;
    a.lddy = dy.ld;
    a.dydt = dtype_of(dy.type, "dy");
    a.x = m.p;
    a.ldx = m.ld;
    a.w = w.p;
    a.ldw = w.ld;
    a.z = z.p;
    a.ldz = z.ld;
    a.act = act;
    a.dx = o[0].p;
    a.lddx = o[0].ld;
    a.dxdt = dtype_of(xt, "dx");
    a.dw = o[1].p;
    a.lddw = o[1].ld;
    a.dwdt = dtype_of(dwt, "dW");
    a.db = static_cast<float*>(o[2].p);
    const size_t n = entry.linear_bwd_size(&a);
    void* ws = call.workspace(x, n);
    call.uses(v, 11, o);
    ok(entry.linear_bwd(&a, ws, n, call.stream), "sadmm_linear_bwd");
    return wrap_all(o);
}

// x, Wg, Wu, bg, bu, act, save, out, stream
PyObject* gated(PyObject* const* v)
{
    const Tensor& x = first(v[0], {{v[1], "Wg"}, {v[2], "Wu"}, {v[3], "bg"}, {v[4], "bu"}, {v[7], "out"}});
    const Matrix m = matrix_of(x, "x", -1, x.dim() ? x.size(-1) : 0, at::kBFloat16);
    const Matrix wg = matrix_of(tensor(v[1], "Wg"), "Wg", -1, m.cols, at::kBFloat16);
    const Matrix wu = matrix_of(tensor(v[2], "Wu"), "Wu", wg.rows, m.cols, at::kBFloat16);
    const bool save = flag(v[6]);
    Call call(x, v[8]);
    Output o[3];
    o[0] = v[7] != Py_None ? given(v[7], matrix_of(tensor(v[7], "out"), "out", m.rows, wg.rows, at::kBFloat16))
                           : new_rows(x, wg.rows, at::kBFloat16);
    if (save) {
        o[1] = new_rows(x, wg.rows, at::kBFloat16);
        o[2] = new_rows(x, wg.rows, at::kBFloat16);
    }
    sadmm_gated_fwd_args a = {};
    a.tokens = m.rows;
    a.n_in = width(m.cols);
    a.n_hidden = width(wg.rows);
    a.x = m.p;
    a.ldx = m.ld;
    a.wg = wg.p;
    a.ldwg = wg.ld;
    a.wu = wu.p;
    a.ldwu = wu.ld;
    a.bg = vector_or_none(v[3], wg.rows, "bg");
    a.bu = vector_or_none(v[4], wg.rows, "bu");
    a.act = number(v[5]);
    a.h = o[0].p;
    a.ldh = o[0].ld;
    a.g = o[1].p;
    a.ldg = o[1].ld;
    a.u = o[2].p;
    a.ldu = o[2].ld;
    const size_t n = apart(m) || apart(wg) || apart(wu) ? entry.gated_fwd_size(&a) : 0;
    void* ws = call.workspace(x, n);
    call.uses(v, 9, o);
    ok(entry.gated_fwd(&a, ws, n, call.stream), "sadmm_gated_fwd");
    return save ? wrap_all(o) : wrap(o[0]);
}

// dh, x, Wg, Wu, g, u, act, want_dx, want_dw, want_db, dx_dtype, dw_dtype, stream
PyObject* gated_backward(PyObject* const* v)
{
    const Tensor& x = first(v[1], {{v[0], "dh"}, {v[2], "Wg"}, {v[3], "Wu"}, {v[4], "g"}, {v[5], "u"}});
    const Tensor &dht = tensor(v[0], "dh"), &wgt = tensor(v[2], "Wg"), &wut = tensor(v[3], "Wu");
    const Matrix m = matrix_of(x, "x", -1, x.dim() ? x.size(-1) : 0, at::kBFloat16);
    const Matrix dh = matrix_of(dht, "dh", m.rows, dht.dim() ? dht.size(-1) : 0, at::kBFloat16);
    const Matrix wg = matrix_of(wgt, "Wg", dh.cols, m.cols, at::kBFloat16);
    const Matrix wu = matrix_of(wut, "Wu", dh.cols, m.cols, at::kBFloat16);
    const Matrix g = matrix_of(tensor(v[4], "g"), "g", m.rows, dh.cols, at::kBFloat16);
    const Matrix u = matrix_of(tensor(v[5], "u"), "u", m.rows, dh.cols, at::kBFloat16);
    const ScalarType xt = dtype_arg(v[10], at::kBFloat16), dwt = dtype_arg(v[11], at::kBFloat16);  // as in linear_backward
    Call call(x, v[12]);
    Output o[5];
    if (flag(v[7])) o[0] = new_rows(x, m.cols, xt);
    if (flag(v[8])) {
        o[1] = like_weight(wgt, wg, dwt);
        o[2] = like_weight(wut, wu, dwt);
    }
    if (flag(v[9])) {
        o[3] = new_vector(x, dh.cols);
        o[4] = new_vector(x, dh.cols);
    }
    sadmm_gated_bwd_args a = {};
    a.tokens = m.rows;
    a.n_in = width(m.cols);
    a.n_hidden = width(dh.cols);
    a.dh = dh.p;
    a.lddh = dh.ld;
    a.x = m.p;
    a.ldx = m.ld;
    a.wg = wg.p;
    a.ldwg = wg.ld;
    a.wu = wu.p;
    a.ldwu = wu.ld;
    a.g = g.p;
    a.ldg = g.ld;
    a.u = u.p;
    a.ldu = u.ld;
    a.act = number(v[6]);
    a.dx = o[0].p;
    a.lddx = o[0].ld;
    a.dxdt = dtype_of(xt, "dx");
    a.dwg = o[1].p;
    a.lddwg = o[1].ld;
    a.dwu = o[2].p;
    a.lddwu = o[2].ld;
    a.dwdt = dtype_of(dwt, "dW");
    a.dbg = static_cast<float*>(o[3].p);
    a.dbu = static_cast<float*>(o[4].p);
    const size_t n = entry.gated_bwd_size(&a);
    void* ws = call.workspace(x, n);
    call.uses(v, 13, o);
    ok(entry.gated_bwd(&a, ws, n, call.stream), "sadmm_gated_bwd");
    return wrap_all(o);
}

// ------------------------------------------------------------------ module --

// Every C++ exception ends here.
template <PyObject* (*F)(PyObject* const*), Py_ssize_t N>
PyObject* method(PyObject*, PyObject* const* v, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != N) {
        PyErr_Format(PyExc_TypeError, "%zd arguments, not %zd", N, n);
        return nullptr;
    }
    if (!entry.linear_fwd) {
        PyErr_SetString(PyExc_RuntimeError, "bind() has not been called");
        return nullptr;
    }
    try {
        return F(v);
    } catch (const PythonError&) {
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

// bind(path of libsadmm, SadmmError)
PyObject* bind(PyObject*, PyObject* const* v, Py_ssize_t n)
{
    if (n != 2) {
        PyErr_SetString(PyExc_TypeError, "bind(path, error class)");
        return nullptr;
    }
    const char* path = PyUnicode_AsUTF8(v[0]);
    if (!path) return nullptr;
    void* lib = dlopen(path, RTLD_NOW | RTLD_LOCAL);
    if (!lib) {
        PyErr_SetString(PyExc_OSError, dlerror());
        return nullptr;
    }
    bool all = true;
    auto get = [&](auto& f, const char* name) {
        void* p = dlsym(lib, name);
        all = all && p;
        f = reinterpret_cast<std::decay_t<decltype(f)>>(p);
    };
    Entry e = {};
    get(e.layernorm_fwd, "sadmm_layernorm_fwd");
    get(e.layernorm_bwd_size, "sadmm_layernorm_bwd_workspace_size");
    get(e.layernorm_bwd, "sadmm_layernorm_bwd");
    get(e.linear_fwd_size, "sadmm_linear_fwd_workspace_size");
    get(e.linear_fwd, "sadmm_linear_fwd");
    get(e.linear_bwd_size, "sadmm_linear_bwd_workspace_size");
    get(e.linear_bwd, "sadmm_linear_bwd");
    get(e.gated_fwd_size, "sadmm_gated_fwd_workspace_size");
    get(e.gated_fwd, "sadmm_gated_fwd");
    get(e.gated_bwd_size, "sadmm_gated_bwd_workspace_size");
    get(e.gated_bwd, "sadmm_gated_bwd");
    if (!all) {
        PyErr_SetString(PyExc_OSError, "the library lacks an entry point");
        return nullptr;
    }
    entry = e;
    Py_INCREF(v[1]);
    Py_XDECREF(error_class);
    error_class = v[1];
    Py_RETURN_NONE;
}

#define SADMM_METHOD(f, n) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&method<f, n>)), METH_FASTCALL, nullptr}

PyMethodDef methods[] = {
    {"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&bind)), METH_FASTCALL, nullptr},
    SADMM_METHOD(layer_norm, 8),
    SADMM_METHOD(layer_norm_backward, 10),
    SADMM_METHOD(linear, 9),
    SADMM_METHOD(linear_backward, 11),
    SADMM_METHOD(gated, 9),
    SADMM_METHOD(gated_backward, 13),
    {nullptr, nullptr, 0, nullptr},
};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "torch_ffn", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_torch_ffn() { return PyModule_Create(&module); }
