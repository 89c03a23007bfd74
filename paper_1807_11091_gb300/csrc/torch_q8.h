// torch_q8.h -- the feed-forward operators with 8-bit operands on torch tensors
// (part of torch_ffn.cpp).
#pragma once

#include "torch_call.h"

namespace {

struct Entry8 {
    decltype(&sadmm_rmsnorm_fwd) rmsnorm_fwd;
    decltype(&sadmm_rmsnorm_bwd_workspace_size) rmsnorm_bwd_size;
    decltype(&sadmm_rmsnorm_bwd) rmsnorm_bwd;
    decltype(&sadmm_quantize) quantize;
    decltype(&sadmm_linear8_fwd_workspace_size) linear8_fwd_size;
    decltype(&sadmm_linear8_fwd) linear8_fwd;
    decltype(&sadmm_linear8_bwd_workspace_size) linear8_bwd_size;
    decltype(&sadmm_linear8_bwd) linear8_bwd;
    decltype(&sadmm_gated8_fwd_workspace_size) gated8_fwd_size;
    decltype(&sadmm_gated8_fwd) gated8_fwd;
    decltype(&sadmm_gated8_bwd_workspace_size) gated8_bwd_size;
    decltype(&sadmm_gated8_bwd) gated8_bwd;
} entry8;

// The tensor that sets the call's device; the others have to be on it.
const Tensor& lead(PyObject* o, const char* name, std::initializer_list<Named> others)
{
    const Tensor& x = tensor(o, name);
    for (const Named& n : others) {
        if (n.o == Py_None) continue;
        const Tensor& t = tensor(n.o, n.name);
        if (t.device() != x.device())
            fail(PyExc_ValueError, std::string(n.name) + " is on " + t.device().str() + ", " + name + " on " + x.device().str());
    }
    return x;
}

int64_t blocks_of(int64_t n) { return (n + 127) / 128; }

// An 8-bit matrix: q [rows][cols] (rows < 0: any) and its scales, [rows][blocks] or for
// tiles of 128 rows [ceil(rows / 128)][blocks], of any strides.
struct Eight {
    sadmm_q8 m = {};
    int64_t rows = 0, cols = 0;
    bool apart() const { return ((reinterpret_cast<uintptr_t>(m.q) | (uintptr_t)m.ld) & 15) != 0; }
};
Eight eight(PyObject* qo, PyObject* so, const char* name, int64_t rows, int64_t cols)
{
    const Tensor &q = tensor(qo, name), &s = tensor(so, (std::string(name) + "'s scales").c_str());
    if (q.dim() < 1) fail(PyExc_TypeError, std::string(name) + " needs a last dimension");
    const Matrix m = matrix_of(q, name, rows, cols < 0 ? q.size(-1) : cols, at::kFloat8_e4m3fn);
    Eight e;
    e.rows = m.rows;
    e.cols = m.cols;
    e.m.q = m.p;
    e.m.ld = m.rows > 1 ? m.ld : (m.cols + 15) / 16 * 16;
    const std::string what = std::string(name) + "'s scales";
    if (s.scalar_type() != at::kFloat) fail(PyExc_TypeError, what + " must be fp32, got " + type_name(s.scalar_type()));
    const int64_t d = s.dim(), blocks = blocks_of(m.cols);
    if (d < 1) fail(PyExc_TypeError, what + " need a last dimension");
    int64_t n = 1;
    for (int64_t i = 0; i < d - 1; ++i) n *= s.size(i);
    const bool tile = n != m.rows && n == blocks_of(m.rows);
    if (s.size(d - 1) != blocks || (n != m.rows && !tile))
        fail(PyExc_ValueError, what + " are " + std::to_string(n) + " x " + std::to_string(s.size(d - 1)) + ", not " +
                                   std::to_string(m.rows) + " (or " + std::to_string(blocks_of(m.rows)) + ") x " +
                                   std::to_string(blocks));
    e.m.s = static_cast<const float*>(s.data_ptr());
    e.m.tile = tile;
    e.m.s_block = blocks > 1 ? s.stride(d - 1) : 1;
    e.m.s_row = 1;
    if (n > 1) {
        int64_t i = d - 2;
        while (s.size(i) == 1) --i;
        e.m.s_row = s.stride(i);
        int64_t next = e.m.s_row * s.size(i);
        for (--i; i >= 0; --i) {
            if (s.size(i) == 1) continue;
            if (s.stride(i) != next) fail(PyExc_TypeError, what + "' leading dimensions do not view as one");
            next *= s.size(i);
        }
    }
    return e;
}

// A new 8-bit matrix in like's leading dimensions (or [rows]): rows on 32-byte
// boundaries; scales of `rows / high` rows, those of a block neighbours.
struct NewEight {
    Output q, s;
    sadmm_q8_out m = {};
};
NewEight finish_eight(Output q, const Tensor& like, int64_t rows, const int64_t* size, int64_t d, int64_t cols)
{
    NewEight e;
    e.q = q;
    const int64_t blocks = blocks_of(cols), step = (rows + 3) / 4 * 4;
    int64_t shape[16], stride[16];
    int64_t next = 1;
    for (int64_t i = d - 1; i >= 0; --i) {
        shape[i] = size[i];
        stride[i] = next;
        next *= size[i];
    }
    shape[d] = blocks;
    stride[d] = step > 0 ? step : 1;
    e.s.t = at::empty_strided(at::IntArrayRef(shape, d + 1), at::IntArrayRef(stride, d + 1), like.options().dtype(at::kFloat));
    e.s.p = e.s.t.data_ptr();
    e.m.q = e.q.p;
    e.m.ld = e.q.ld;
    e.m.s = static_cast<float*>(e.s.p);
    e.m.s_row = 1;
    e.m.s_block = stride[d];
    return e;
}
Output new_bytes(const Tensor& like, int64_t rows, int64_t cols)
{
    const int64_t ld = (cols + 31) / 32 * 32, size[2] = {rows, cols}, stride[2] = {ld > 0 ? ld : 1, 1};
    Output o;
    o.t = at::empty_strided(at::IntArrayRef(size, 2), at::IntArrayRef(stride, 2), like.options().dtype(at::kFloat8_e4m3fn));
    o.p = o.t.data_ptr();
    o.ld = stride[0];
    return o;
}
NewEight new_eight(const Tensor& like, int64_t rows, int64_t cols)
{
    const int64_t d = like.dim() - 1;
    if (d > 14) fail(PyExc_ValueError, "more than 15 dimensions");
    return finish_eight(allocate(like, cols, (cols + 31) / 32 * 32, at::kFloat8_e4m3fn), like, rows, like.sizes().data(), d,
                        cols);
}
NewEight new_eight2(const Tensor& like, int64_t rows, int64_t cols, int64_t scale_rows)
{
    return finish_eight(new_bytes(like, rows, cols), like, scale_rows, &scale_rows, 1, cols);
}

Output new_matrix(const Tensor& like, int64_t rows, int64_t cols, ScalarType type)
{
    const int64_t step = type == at::kBFloat16 ? 16 : 8, ld = (cols + step - 1) / step * step;
    const int64_t size[2] = {rows, cols}, stride[2] = {ld, 1};
    Output o;
    o.t = at::empty_strided(at::IntArrayRef(size, 2), at::IntArrayRef(stride, 2), like.options().dtype(type));
    o.p = o.t.data_ptr();
    o.ld = ld;
    return o;
}

// The outputs there are: one by itself, or a tuple.
PyObject* wrap_there(const Output* o, int n)
{
    int there = 0;
    const Output* last = nullptr;
    for (int i = 0; i < n; ++i)
        if (o[i].t.defined()) ++there, last = &o[i];
    if (there == 1) return wrap(*last);
    PyObject* t = PyTuple_New(there);
    if (!t) throw PythonError();
    for (int i = 0, at = 0; i < n; ++i) {
        if (!o[i].t.defined()) continue;
        PyObject* v = wrap(o[i]);
        if (!v) {
            Py_DECREF(t);
            throw PythonError();
        }
        PyTuple_SET_ITEM(t, at++, v);
    }
    return t;
}

// An out of its own type cannot hold what out_dtype e4m3 asks for, q and scales.
void no_bits_in(PyObject* out, PyObject* out_dtype)
{
    if (out != Py_None && dtype_arg(out_dtype, at::kFloat) == at::kFloat8_e4m3fn)
        fail(PyExc_TypeError, "out_dtype float8_e4m3fn with an out: 8-bit results are the call's own tensors");
}

// x, gamma, residual, eps, out_dtype, stats, out, sum_out, stream
PyObject* rms_norm(PyObject* const* v)
{
    const Tensor& x = lead(v[0], "x", {{v[1], "gamma"}, {v[2], "residual"}, {v[6], "out"}, {v[7], "sum_out"}});
    const Matrix m = matrix(x, "x");
    const double eps = PyFloat_AsDouble(v[3]);
    if (eps == -1.0 && PyErr_Occurred()) throw PythonError();
    no_bits_in(v[6], v[4]);
    const ScalarType want = dtype_arg(v[4], m.type);
    const bool stats = flag(v[5]), bits = v[6] == Py_None && want == at::kFloat8_e4m3fn;
    Matrix r;
    if (v[2] != Py_None) r = matrix_of(tensor(v[2], "residual"), "residual", m.rows, m.cols, std::nullopt);
    if (v[7] != Py_None && !r.p) fail(PyExc_ValueError, "sum_out without a residual");
    Call call(x, v[8]);
    Output o[4];
    sadmm_rmsnorm_fwd_args a = {};
    a.rows = m.rows;
    a.cols = width(m.cols);
    a.x = m.p;
    a.ldx = m.ld;
    a.xdt = dtype_of(m.type, "x");
    a.gamma = vector_or_none(v[1], m.cols, "gamma");
    a.eps = (float)eps;
    if (bits) {
        const NewEight e = new_eight(x, m.rows, m.cols);
        o[0] = e.q;
        o[1] = e.s;
        a.ydt = SADMM_E4M3;
        a.y8 = e.m;
    } else {
        o[0] = v[6] != Py_None ? given(v[6], matrix_of(tensor(v[6], "out"), "out", m.rows, m.cols, std::nullopt))
                               : new_rows(x, m.cols, want);
        a.ydt = dtype_of(o[0].t.scalar_type(), "out");
        a.y = o[0].p;
        a.ldy = o[0].ld;
    }
    if (v[2] != Py_None) {
        a.rdt = dtype_of(r.type, "residual");
        a.residual = r.p;
        a.ldr = r.ld;
        o[2] = v[7] != Py_None ? given(v[7], matrix_of(tensor(v[7], "sum_out"), "sum_out", m.rows, m.cols, r.type))
                               : new_rows(x, m.cols, r.type);
        a.h = o[2].p;
        a.ldh = o[2].ld;
    }
    if (stats) o[3] = new_vector(x, m.rows);
    a.rstd = static_cast<float*>(o[3].p);
    call.uses(v, 9, o);
    ok(entry8.rmsnorm_fwd(&a, call.stream), "sadmm_rmsnorm_fwd");
    return wrap_there(o, 4);
}

// dy, h, rstd, gamma, dres, want_dx, want_dgamma, stream
PyObject* rms_norm_backward(PyObject* const* v)
{
    const Tensor& h = lead(v[1], "h", {{v[0], "dy"}, {v[2], "rstd"}, {v[3], "gamma"}, {v[4], "dres"}});
    const Matrix m = matrix(h, "h");
    const Matrix dy = matrix_of(tensor(v[0], "dy"), "dy", m.rows, m.cols, std::nullopt);
    Matrix dres;
    if (const Tensor* t = tensor_or_none(v[4], "dres")) dres = matrix_of(*t, "dres", m.rows, m.cols, m.type);
    Call call(h, v[7]);
    Output o[2];
    if (flag(v[5])) o[0] = new_rows(h, m.cols, m.type);
    if (flag(v[6])) o[1] = new_vector(h, m.cols);
    sadmm_rmsnorm_bwd_args a = {};
    a.rows = m.rows;
    a.cols = width(m.cols);
    a.h = m.p;
    a.ldh = m.ld;
    a.hdt = dtype_of(m.type, "h");
    a.dy = dy.p;
    a.lddy = dy.ld;
    a.dydt = dtype_of(dy.type, "dy");
    a.gamma = vector_or_none(v[3], m.cols, "gamma");
    a.rstd = vector(tensor(v[2], "rstd"), m.rows, "rstd");
    a.dres = dres.p;
    a.lddres = dres.ld;
    a.dx = o[0].p;
    a.lddx = o[0].ld;
    a.dgamma = static_cast<float*>(o[1].p);
    const size_t n = entry8.rmsnorm_bwd_size(&a);
    void* ws = call.workspace(h, n);
    call.uses(v, 8, o);
    ok(entry8.rmsnorm_bwd(&a, ws, n, call.stream), "sadmm_rmsnorm_bwd");
    return wrap_all(o);
}

// x, tiles, want_q, transposed, stream
PyObject* quantize(PyObject* const* v)
{
    const Tensor& x = tensor(v[0], "x");
    const Matrix m = matrix(x, "x");
    const bool tiles = flag(v[1]), want = flag(v[2]), turned = flag(v[3]);
    if (!want && !turned) fail(PyExc_ValueError, "neither the matrix nor its transpose is wanted");
    Call call(x, v[4]);
    Output o[4];
    sadmm_quantize_args a = {};
    a.rows = m.rows;
    a.cols = m.cols;
    a.x = m.p;
    a.ldx = m.ld;
    a.xdt = dtype_of(m.type, "x");
    a.tile = tiles;
    if (want) {
        const NewEight e = tiles ? new_eight2(x, m.rows, m.cols, blocks_of(m.rows)) : new_eight(x, m.rows, m.cols);
        o[0] = e.q;
        o[1] = e.s;
        a.out = e.m;
    }
    if (turned) {
        const NewEight e = new_eight2(x, m.cols, m.rows, tiles ? blocks_of(m.cols) : m.cols);
        o[2] = e.q;
        o[3] = e.s;
        a.out_t = e.m;
    }
    call.uses(v, 5, o);
    ok(entry8.quantize(&a, call.stream), "sadmm_quantize");
    return wrap_there(o, 4);
}

// x, xs, W, Ws, bias, residual, act, out_dtype, save, out, stream
PyObject* linear8(PyObject* const* v)
{
    const Tensor& x = lead(v[0], "x", {{v[1], "xs"}, {v[2], "W"}, {v[3], "Ws"}, {v[4], "bias"}, {v[5], "residual"}, {v[9], "out"}});
    const Eight m = eight(v[0], v[1], "x", -1, -1);
    const Eight w = eight(v[2], v[3], "W", -1, m.cols);
    const Tensor* residual = tensor_or_none(v[5], "residual");
    const bool save = flag(v[8]);
    no_bits_in(v[9], v[7]);
    Call call(x, v[10]);
    Output o[2];
    o[0] = v[9] != Py_None
               ? given(v[9], matrix_of(tensor(v[9], "out"), "out", m.rows, w.rows, std::nullopt))
               : new_rows(x, w.rows, dtype_arg(v[7], residual ? residual->scalar_type() : at::kBFloat16));
    if (save) o[1] = new_rows(x, w.rows, at::kBFloat16);
    Matrix r;
    if (residual) r = matrix_of(*residual, "residual", m.rows, w.rows, o[0].t.scalar_type());
    sadmm_linear8_fwd_args a = {};
    a.tokens = m.rows;
    a.n_in = width(m.cols);
    a.n_out = width(w.rows);
    a.x = m.m;
    a.w = w.m;
    a.bias = vector_or_none(v[4], w.rows, "bias");
    a.residual = r.p;
    a.ldr = r.ld;
    a.act = number(v[6]);
    a.y = o[0].p;
    a.ldy = o[0].ld;
    a.ydt = dtype_of(o[0].t.scalar_type(), "out");
    a.z = o[1].p;
    a.ldz = o[1].ld;
    const size_t n = m.apart() || w.apart() ? entry8.linear8_fwd_size(&a) : 0;
    void* ws = call.workspace(x, n);
    call.uses(v, 11, o);
    ok(entry8.linear8_fwd(&a, ws, n, call.stream), "sadmm_linear8_fwd");
    return wrap_there(o, 2);
}

// dy, xt, xts, Wt, Wts, z, act, want_dx, want_dw, want_db, dx_dtype, dw_dtype, stream
PyObject* linear8_backward(PyObject* const* v)
{
    const int act = number(v[6]);
    const bool dx = flag(v[7]), dw = flag(v[8]);
    PyObject* const none = Py_None;
    const Tensor& dyt = lead(v[0], "dy", {{dw ? v[1] : none, "xt"}, {dw ? v[2] : none, "xts"}, {dx ? v[3] : none, "Wt"},
                                          {dx ? v[4] : none, "Wts"}, {act != SADMM_ACT_NONE ? v[5] : none, "z"}});
    const Matrix dy = matrix(dyt, "dy");
    Eight xt, wt;
    if (dx) wt = eight(v[3], v[4], "Wt", -1, dy.cols);
    if (dw) xt = eight(v[1], v[2], "xt", dx ? wt.rows : -1, dy.rows);
    const int64_t n_in = dx ? wt.rows : dw ? xt.rows : 1;
    Matrix z;
    if (act != SADMM_ACT_NONE) {
        if (v[5] == Py_None) fail(PyExc_TypeError, "the gradient of an activation needs z");
        z = matrix_of(tensor(v[5], "z"), "z", dy.rows, dy.cols, at::kBFloat16);
    }
    const ScalarType dxt = dtype_arg(v[10], at::kBFloat16), dwt = dtype_arg(v[11], at::kBFloat16);
    Call call(dyt, v[12]);
    Output o[3];
    if (dx) o[0] = new_rows(dyt, n_in, dxt);
    if (dw) o[1] = new_matrix(dyt, dy.cols, n_in, dwt);
    if (flag(v[9])) o[2] = new_vector(dyt, dy.cols);
    sadmm_linear8_bwd_args a = {};
    a.tokens = dy.rows;
    a.n_in = width(n_in);
    a.n_out = width(dy.cols);
    a.dy = dy.p;
    a.lddy = dy.ld;
    a.dydt = dtype_of(dy.type, "dy");
    a.xt = xt.m;
    a.wt = wt.m;
    a.z = z.p;
    a.ldz = z.ld;
    a.act = act;
    a.dx = o[0].p;
    a.lddx = o[0].ld;
    a.dxdt = dtype_of(dxt, "dx");
    a.dw = o[1].p;
    a.lddw = o[1].ld;
    a.dwdt = dtype_of(dwt, "dW");
    a.db = static_cast<float*>(o[2].p);
    const size_t n = entry8.linear8_bwd_size(&a);
    void* ws = call.workspace(dyt, n);
    call.uses(v, 13, o);
    ok(entry8.linear8_bwd(&a, ws, n, call.stream), "sadmm_linear8_bwd");
    return wrap_all(o);
}

// x, xs, Wg, Wgs, Wu, Wus, bg, bu, act, out_dtype, save, stream
PyObject* gated8(PyObject* const* v)
{
    const Tensor& x = lead(v[0], "x", {{v[1], "xs"}, {v[2], "Wg"}, {v[3], "Wgs"}, {v[4], "Wu"}, {v[5], "Wus"}, {v[6], "bg"}, {v[7], "bu"}});
    const Eight m = eight(v[0], v[1], "x", -1, -1);
    const Eight wg = eight(v[2], v[3], "Wg", -1, m.cols), wu = eight(v[4], v[5], "Wu", wg.rows, m.cols);
    const ScalarType type = dtype_arg(v[9], at::kFloat8_e4m3fn);
    if (type != at::kFloat8_e4m3fn && type != at::kBFloat16)
        fail(PyExc_TypeError, std::string("out must be e4m3 or bf16, got ") + type_name(type));
    const bool save = flag(v[10]);
    Call call(x, v[11]);
    Output o[4];
    sadmm_gated8_fwd_args a = {};
    if (type == at::kFloat8_e4m3fn) {
        const NewEight e = new_eight(x, m.rows, wg.rows);
        o[0] = e.q;
        o[1] = e.s;
        a.hdt = SADMM_E4M3;
        a.h8 = e.m;
    } else {
        o[0] = new_rows(x, wg.rows, type);
        a.hdt = SADMM_BF16;
        a.h = o[0].p;
        a.ldh = o[0].ld;
    }
    if (save) {
        o[2] = new_rows(x, wg.rows, at::kBFloat16);
        o[3] = new_rows(x, wg.rows, at::kBFloat16);
    }
    a.tokens = m.rows;
    a.n_in = width(m.cols);
    a.n_hidden = width(wg.rows);
    a.x = m.m;
    a.wg = wg.m;
    a.wu = wu.m;
    a.bg = vector_or_none(v[6], wg.rows, "bg");
    a.bu = vector_or_none(v[7], wg.rows, "bu");
    a.act = number(v[8]);
    a.g = o[2].p;
    a.ldg = o[2].ld;
    a.u = o[3].p;
    a.ldu = o[3].ld;
    const size_t n = m.apart() || wg.apart() || wu.apart() ? entry8.gated8_fwd_size(&a) : 0;
    void* ws = call.workspace(x, n);
    call.uses(v, 12, o);
    ok(entry8.gated8_fwd(&a, ws, n, call.stream), "sadmm_gated8_fwd");
    return wrap_there(o, 4);
}

// dh, xt, xts, Wgt, Wgts, Wut, Wuts, g, u, act, want_dx, want_dw, want_db, dx_dtype, dw_dtype, stream
PyObject* gated8_backward(PyObject* const* v)
{
    const bool dx = flag(v[10]), dw = flag(v[11]);
    PyObject* const none = Py_None;
    const Tensor& dht = lead(v[0], "dh", {{dw ? v[1] : none, "xt"}, {dw ? v[2] : none, "xts"}, {dx ? v[3] : none, "Wgt"},
                                          {dx ? v[4] : none, "Wgts"}, {dx ? v[5] : none, "Wut"}, {dx ? v[6] : none, "Wuts"},
                                          {v[7], "g"}, {v[8], "u"}});
    const Matrix dh = matrix_of(dht, "dh", -1, dht.dim() ? dht.size(-1) : 0, at::kBFloat16);
    const Matrix g = matrix_of(tensor(v[7], "g"), "g", dh.rows, dh.cols, at::kBFloat16);
    const Matrix u = matrix_of(tensor(v[8], "u"), "u", dh.rows, dh.cols, at::kBFloat16);
    Eight xt, wgt, wut;
    if (dx) {
        wgt = eight(v[3], v[4], "Wgt", -1, dh.cols);
        wut = eight(v[5], v[6], "Wut", wgt.rows, dh.cols);
    }
    if (dw) xt = eight(v[1], v[2], "xt", dx ? wgt.rows : -1, dh.rows);
    const int64_t n_in = dx ? wgt.rows : dw ? xt.rows : 1;
    const ScalarType dxt = dtype_arg(v[13], at::kBFloat16), dwt = dtype_arg(v[14], at::kBFloat16);
    Call call(dht, v[15]);
    Output o[5];
    if (dx) o[0] = new_rows(dht, n_in, dxt);
    if (dw) {
        o[1] = new_matrix(dht, dh.cols, n_in, dwt);
        o[2] = new_matrix(dht, dh.cols, n_in, dwt);
    }
    if (flag(v[12])) {
        o[3] = new_vector(dht, dh.cols);
        o[4] = new_vector(dht, dh.cols);
    }
    sadmm_gated8_bwd_args a = {};
    a.tokens = dh.rows;
    a.n_in = width(n_in);
    a.n_hidden = width(dh.cols);
    a.dh = dh.p;
    a.lddh = dh.ld;
    a.xt = xt.m;
    a.wgt = wgt.m;
    a.wut = wut.m;
    a.g = g.p;
    a.ldg = g.ld;
    a.u = u.p;
    a.ldu = u.ld;
    a.act = number(v[9]);
    a.dx = o[0].p;
    a.lddx = o[0].ld;
    a.dxdt = dtype_of(dxt, "dx");
    a.dwg = o[1].p;
    a.lddwg = o[1].ld;
    a.dwu = o[2].p;
    a.lddwu = o[2].ld;
    a.dwdt = dtype_of(dwt, "dW");
    a.dbg = static_cast<float*>(o[3].p);
    a.dbu = static_cast<float*>(o[4].p);
    const size_t n = entry8.gated8_bwd_size(&a);
    void* ws = call.workspace(dht, n);
    call.uses(v, 16, o);
    ok(entry8.gated8_bwd(&a, ws, n, call.stream), "sadmm_gated8_bwd");
    return wrap_all(o);
}

}  // namespace
