// torch_call.h -- what the bindings of torch tensors share (torch_ffn.cpp,
// torch_q8.h): arguments as matrices, outputs and scratch from torch's
// allocator, the call's stream, errors.
#pragma once

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

struct PythonError {};  // a Python exception is set

[[noreturn]] void fail(PyObject* type, const std::string& what)
{
    PyErr_SetString(type, what.c_str());
    throw PythonError();
}

PyObject* error_class;  // sadmm.SadmmError

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

}  // namespace
