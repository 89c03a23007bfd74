// torch_ffn.cpp -- the feed-forward operators on torch tensors: checks, outputs
// and scratch from torch's allocator, and the call of the C entry point on
// torch's current stream.  Everything else is behind the C ABI (sadmm.h).
//
// This is native because on a few tokens the host is what a call costs: with
// the same steps in Python a layer norm of four rows took 14 us a call, its
// kernel 2.  sadmm.py holds the functions' signatures and documentation and
// passes their arguments on by position.
#include "torch_call.h"
#include "torch_q8.h"

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
    Entry8 e8 = {};
    get(e8.rmsnorm_fwd, "sadmm_rmsnorm_fwd");
    get(e8.rmsnorm_bwd_size, "sadmm_rmsnorm_bwd_workspace_size");
    get(e8.rmsnorm_bwd, "sadmm_rmsnorm_bwd");
    get(e8.quantize, "sadmm_quantize");
    get(e8.linear8_fwd_size, "sadmm_linear8_fwd_workspace_size");
    get(e8.linear8_fwd, "sadmm_linear8_fwd");
    get(e8.linear8_bwd_size, "sadmm_linear8_bwd_workspace_size");
    get(e8.linear8_bwd, "sadmm_linear8_bwd");
    get(e8.gated8_fwd_size, "sadmm_gated8_fwd_workspace_size");
    get(e8.gated8_fwd, "sadmm_gated8_fwd");
    get(e8.gated8_bwd_size, "sadmm_gated8_bwd_workspace_size");
    get(e8.gated8_bwd, "sadmm_gated8_bwd");
    if (!all) {
        PyErr_SetString(PyExc_OSError, "the library lacks an entry point");
        return nullptr;
    }
    entry = e;
    entry8 = e8;
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
    SADMM_METHOD(rms_norm, 9),
    SADMM_METHOD(rms_norm_backward, 8),
    SADMM_METHOD(quantize, 5),
    SADMM_METHOD(linear8, 11),
    SADMM_METHOD(linear8_backward, 13),
    SADMM_METHOD(gated8, 12),
    SADMM_METHOD(gated8_backward, 16),
    {nullptr, nullptr, 0, nullptr},
};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "torch_ffn", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_torch_ffn() { return PyModule_Create(&module); }
