// linear8.cu -- the feed-forward products of 8-bit operands: operands off 16-byte
// boundaries copied to where the tensor-memory accelerator can read them
// (k_q8_realign), a backward pass's dz (dg, du) made 8-bit (quant.cu), and the
// products (q8gemm.cu).
#include <string.h>

#include "q8.cuh"

namespace sadmm {
namespace {

// ------------------------------------------------------------ k_q8_realign --

struct Copies {
    const uint8_t* src[3];
    uint8_t* dst[3];
    long long ld[3], ldd[3], rows[3];
    int cols[3];
    int* status;
};

// Matrix blockIdx.y, 16 bytes a thread: rows of `words` 16-byte words, zeros past the
// row's end.
__global__ void __launch_bounds__(256) k_q8_realign(const Copies a)
{
    pdl_wait();
    pdl_trigger();
    const int m = blockIdx.y;
    const long long words = a.ldd[m] / 16, total = a.rows[m] * words;
    const Span span = {a.src[m], a.src[m] + (a.rows[m] - 1) * a.ld[m] + a.cols[m]};
    for (long long i = blockIdx.x * 256ll + threadIdx.x; i < total; i += gridDim.x * 256ll) {
        const long long r = total <= 0xffffffffll ? (long long)((uint32_t)i / (uint32_t)words) : i / words;
        const int c = (int)(i - r * words) * 16, n = min(16, a.cols[m] - c);
        if (!dbg_in(r, a.rows[m], a.status) || !dbg_run(c, n, a.cols[m], a.status)) continue;
        uint4 v = load16(a.src[m] + r * a.ld[m] + c, n, span);
        if (n < 16) {
            uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int left = n - 4 * j;
                if (left <= 0) w[j] = 0;
                else if (left < 4) w[j] &= (1u << (8 * left)) - 1u;
            }
            v = make_uint4(w[0], w[1], w[2], w[3]);
        }
        *reinterpret_cast<uint4*>(a.dst[m] + r * a.ldd[m] + c) = v;
    }
}

// -------------------------------------------------------------------- host --

// Places in the workspace, one after the other on 256-byte boundaries.
struct Arena {
    uint8_t* base;
    size_t used;
    void* take(size_t bytes)
    {
        void* p = base ? base + used : nullptr;
        used += (size_t)round_up((long long)bytes, 256);
        return p;
    }
};

// The operand of an 8-bit matrix, with a copy in the workspace where it needs one.
Q8Operand operand(const sadmm_q8& m, long long rows, long long k, Arena& ws, Copies& c, int& copies)
{
    Q8Operand o = {m.q, rows, k, m.ld, m.s, m.s_row, m.s_block, m.tile ? 7 : 0};
    if (q8_aligned(m.q, m.ld) || !m.q) return o;
    const long long ld = round_up(k, 16);
    void* to = ws.take((size_t)rows * (size_t)ld);
    c.src[copies] = static_cast<const uint8_t*>(m.q);
    c.dst[copies] = static_cast<uint8_t*>(to);
    c.ld[copies] = m.ld;
    c.ldd[copies] = ld;
    c.rows[copies] = rows;
    c.cols[copies] = (int)k;
    ++copies;
    o.p = to;
    o.ld = ld;
    return o;
}

sadmm_status run_copies(Copies& c, int n, cudaStream_t s)
{
    if (!n) return SADMM_OK;
    c.status = device_status_ptr();
    long long most = 0;
    for (int i = 0; i < n; ++i) {
        const long long blocks = (c.rows[i] * (c.ldd[i] / 16) + 255) / 256;
        if (blocks > most) most = blocks;
    }
    const long long cap = 16ll * device_sm_count();
    return launch_pdl(k_q8_realign, dim3((unsigned)(most < cap ? most : cap), (unsigned)n), dim3(256), 0, s, c) ==
                   cudaSuccess
               ? SADMM_OK
               : SADMM_ECUDA;
}

// A new 8-bit matrix in the workspace, blocks of one row; scales of a column block
// are neighbours.
sadmm_q8_out make_q8(long long rows, long long cols, Arena& ws)
{
    sadmm_q8_out o;
    o.ld = round_up(cols, 16);
    o.q = ws.take((size_t)rows * (size_t)o.ld);
    o.s_row = 1;
    o.s_block = round_up(rows, 4);
    o.s = static_cast<float*>(ws.take((size_t)o.s_block * (size_t)((cols + kQBlock - 1) / kQBlock) * 4));
    return o;
}
Q8Operand as_operand(const sadmm_q8_out& o, long long rows, long long k)
{
    return {o.q, rows, k, o.ld, o.s, o.s_row, o.s_block, 0};
}

TgMatrix matrix(void* p, long long ld, int dt) { return {p, ld, dt}; }
TgMatrix matrix(const void* p, long long ld, int dt) { return {const_cast<void*>(p), ld, dt}; }

Q8Problem problem(int mode, long long m, long long n)
{
    Q8Problem t;
    memset(&t, 0, sizeof(t));
    t.mode = mode;
    t.m = m;
    t.n = n;
    return t;
}

bool zero(void* p, long long ld, int dt, long long rows, long long cols, cudaStream_t s)
{
    const size_t es = dt == SADMM_BF16 ? 2 : 4;
    return !p || cudaMemset2DAsync(p, (size_t)ld * es, 0, (size_t)cols * es, (size_t)rows, s) == cudaSuccess;
}
bool zero(float* p, long long n, cudaStream_t s) { return !p || cudaMemsetAsync(p, 0, (size_t)n * 4, s) == cudaSuccess; }

// Whether the columns' operand (of a summand) has scales of single rows.
bool row_scales(const Q8Problem& t) { return t.b[0].shift == 0 || (t.mode != kTgSingle && t.b[1].shift == 0); }

// Whether CTA pairs take a product: where they are expected to be faster (8192 -> 2048 of 512 tokens:
// 32 us by pairs, 25 by single tiles; 4096 -> 16384 of 129: 21 and 47).
bool by_pairs(const Q8Problem& t)
{
    return !(t.mode == kTgGated && row_scales(t)) && time_q8_pair(t) < time_q8_product(t);
}

// Rows r .. r+m-1 and columns c .. c+n-1 of a product (no gated pair); r and c are multiples of 128.
Q8Problem part_of(const Q8Problem& t, long long r, long long m, long long c, long long n)
{
    Q8Problem p = t;
    p.m = m, p.n = n;
    for (int j = 0; j < (t.mode == kTgSum ? 2 : 1); ++j) {
        auto rows = [](Q8Operand& o, long long first, long long count) {
            o.p = static_cast<const uint8_t*>(o.p) + first * o.ld;
            o.s += (first >> o.shift) * o.s_row;
            o.rows = count;
        };
        rows(p.a[j], r, m);
        rows(p.b[j], c, n);
    }
    if (p.bias) p.bias += c;
    for (TgMatrix* o : {&p.y, &p.residual, &p.z})
        if (o->p) o->p = static_cast<uint8_t*>(o->p) + (r * o->ld + c) * (o->dt == SADMM_BF16 ? 2 : 4);
    return p;
}

// A product by CTA pairs: all of it, or whole rounds of their tiles and the remaining rows
// or columns by single tiles, which share a long contraction among more CTAs (weights' gradient of
// 8192 x 5120 -> 2048, 160 tiles on 76 pairs: the backward pass 280 us, so 252).
sadmm_status launch_pairs(const Q8Problem& t, cudaStream_t s)
{
    if (t.mode == kTgGated) return launch_q8_pair(&t, 1, s);
    long long rows, cols, best = time_q8_pair(t);
    q8_pair_less(t, rows, cols);
    Q8Problem most = t, rest = t;
    rest.m = 0;
    auto weigh = [&](const Q8Problem& a, const Q8Problem& b) {
        const long long time = time_q8_pair(a) + time_q8_product(b);
        if (time < best) best = time, most = a, rest = b;
    };
    if (rows > 0 && rows < t.m) weigh(part_of(t, 0, rows, 0, t.n), part_of(t, rows, t.m - rows, 0, t.n));
    if (cols > 0 && cols < t.n) weigh(part_of(t, 0, t.m, 0, cols), part_of(t, 0, t.m, cols, t.n - cols));
    const sadmm_status st = launch_q8_pair(&most, 1, s);
    return st == SADMM_OK && rest.m ? launch_q8_product(rest, s) : st;
}

sadmm_status launch_one(const Q8Problem& t, cudaStream_t s) { return by_pairs(t) ? launch_pairs(t, s) : launch_q8_product(t, s); }

// Two products of one shape that no call has one of alone: by CTA pairs in one launch, or by single tiles.
sadmm_status launch_two(const Q8Problem* t, cudaStream_t s)
{
    if (by_pairs(t[0]) && by_pairs(t[1])) return launch_q8_pair(t, 2, s);
    const sadmm_status st = launch_one(t[0], s);
    return st == SADMM_OK ? launch_one(t[1], s) : st;
}

// What a call runs, with its places in the workspace.
struct Forward {
    Q8Problem t;
    Copies c;
    int copies;
    size_t bytes;
};

Forward plan(const sadmm_linear8_fwd_args& a, void* base)
{
    Forward f;
    Arena ws = {static_cast<uint8_t*>(base), 0};
    memset(&f.c, 0, sizeof(f.c));
    f.copies = 0;
    f.t = problem(kTgSingle, a.tokens, a.n_out);
    if (a.tokens) {
        f.t.a[0] = operand(a.x, a.tokens, a.n_in, ws, f.c, f.copies);
        f.t.b[0] = operand(a.w, a.n_out, a.n_in, ws, f.c, f.copies);
    }
    f.t.bias = a.bias;
    f.t.act = a.act;
    f.t.y = matrix(a.y, a.ldy, a.ydt);
    f.t.residual = matrix(a.residual, a.ldr, a.ydt);
    f.t.z = matrix(a.z, a.ldz, SADMM_BF16);
    f.bytes = ws.used;
    return f;
}

Forward plan(const sadmm_gated8_fwd_args& a, void* base)
{
    Forward f;
    Arena ws = {static_cast<uint8_t*>(base), 0};
    memset(&f.c, 0, sizeof(f.c));
    f.copies = 0;
    f.t = problem(kTgGated, a.tokens, a.n_hidden);
    if (a.tokens) {
        f.t.a[0] = operand(a.x, a.tokens, a.n_in, ws, f.c, f.copies);
        f.t.b[0] = operand(a.wg, a.n_hidden, a.n_in, ws, f.c, f.copies);
        f.t.b[1] = operand(a.wu, a.n_hidden, a.n_in, ws, f.c, f.copies);
    }
    f.t.bias = a.bg;
    f.t.bias2 = a.bu;
    f.t.act = a.act;
    if (a.hdt == SADMM_E4M3)
        f.t.y8 = a.h8;
    else
        f.t.y = matrix(a.h, a.ldh, SADMM_BF16);
    f.t.z = matrix(a.g, a.ldg, SADMM_BF16);
    f.t.u = matrix(a.u, a.ldu, SADMM_BF16);
    f.bytes = ws.used;
    return f;
}

sadmm_status run(Forward f, cudaStream_t s)
{
    if (!f.t.m) return SADMM_OK;
    const sadmm_status st = run_copies(f.c, f.copies, s);
    return st != SADMM_OK ? st : launch_one(f.t, s);
}

// The gradients: a source made 8-bit by rows (for dx) and by columns (for the
// weights' gradients), then the products.
struct Backward {
    Q8Source src;
    void* src_ws;
    Q8Problem dx, dw[2];
    int dws;
    bool want_dx;
    Copies c;
    int copies;
    size_t bytes;
};

Backward plan(const sadmm_linear8_bwd_args& a, void* base)
{
    Backward b;
    memset(&b, 0, sizeof(b));
    Arena ws = {static_cast<uint8_t*>(base), 0};
    if (!a.tokens) return b;
    Q8Source& q = b.src;
    q.x = a.dy, q.ldx = a.lddy, q.xdt = a.dydt;
    q.z = a.act != SADMM_ACT_NONE ? a.z : nullptr, q.ldz = a.ldz, q.act = a.act;
    q.rows = a.tokens, q.cols = a.n_out;
    q.sums[0] = a.db;
    if (a.dx) {
        q.out[0] = make_q8(a.tokens, a.n_out, ws);
        b.want_dx = true;
        b.dx = problem(kTgSingle, a.tokens, a.n_in);
        b.dx.a[0] = as_operand(q.out[0], a.tokens, a.n_out);
        b.dx.b[0] = operand(a.wt, a.n_in, a.n_out, ws, b.c, b.copies);
        b.dx.y = matrix(a.dx, a.lddx, a.dxdt);
    }
    if (a.dw) {
        q.out_t[0] = make_q8(a.n_out, a.tokens, ws);
        b.dws = 1;
        b.dw[0] = problem(kTgSingle, a.n_out, a.n_in);
        b.dw[0].a[0] = as_operand(q.out_t[0], a.n_out, a.tokens);
        b.dw[0].b[0] = operand(a.xt, a.n_in, a.tokens, ws, b.c, b.copies);
        b.dw[0].y = matrix(a.dw, a.lddw, a.dwdt);
    }
    b.src_ws = ws.take(q8_source_bytes(q));
    b.bytes = ws.used;
    return b;
}

Backward plan(const sadmm_gated8_bwd_args& a, void* base)
{
    Backward b;
    memset(&b, 0, sizeof(b));
    Arena ws = {static_cast<uint8_t*>(base), 0};
    if (!a.tokens) return b;
    Q8Source& q = b.src;
    q.x = a.dh, q.ldx = a.lddh, q.xdt = SADMM_BF16;
    q.z = a.g, q.ldz = a.ldg, q.u = a.u, q.ldu = a.ldu, q.act = a.act;
    q.rows = a.tokens, q.cols = a.n_hidden;
    q.sums[0] = a.dbg, q.sums[1] = a.dbu;
    if (a.dx) {
        b.want_dx = true;
        b.dx = problem(kTgSum, a.tokens, a.n_in);
        for (int i = 0; i < 2; ++i) {
            q.out[i] = make_q8(a.tokens, a.n_hidden, ws);
            b.dx.a[i] = as_operand(q.out[i], a.tokens, a.n_hidden);
            b.dx.b[i] = operand(i ? a.wut : a.wgt, a.n_in, a.n_hidden, ws, b.c, b.copies);
        }
        b.dx.y = matrix(a.dx, a.lddx, a.dxdt);
    }
    if (a.dwg) {
        b.dws = 2;
        const Q8Operand x = operand(a.xt, a.n_in, a.tokens, ws, b.c, b.copies);
        for (int i = 0; i < 2; ++i) {
            q.out_t[i] = make_q8(a.n_hidden, a.tokens, ws);
            b.dw[i] = problem(kTgSingle, a.n_hidden, a.n_in);
            b.dw[i].a[0] = as_operand(q.out_t[i], a.n_hidden, a.tokens);
            b.dw[i].b[0] = x;
            b.dw[i].y = matrix(i ? a.dwu : a.dwg, i ? a.lddwu : a.lddwg, a.dwdt);
        }
    }
    b.src_ws = ws.take(q8_source_bytes(q));
    b.bytes = ws.used;
    return b;
}

sadmm_status run(Backward b, cudaStream_t s)
{
    sadmm_status st = run_copies(b.c, b.copies, s);
    if (st == SADMM_OK) st = launch_q8_source(b.src, b.src_ws, s);
    // (dx by itself: a launch that it shared with the weights' gradients gave it other bits than it has alone)
    if (st == SADMM_OK && b.want_dx) st = launch_one(b.dx, s);
    if (st == SADMM_OK && b.dws) st = b.dws == 2 ? launch_two(b.dw, s) : launch_one(b.dw[0], s);
    return st;
}

}  // namespace

size_t linear8_fwd_bytes(const sadmm_linear8_fwd_args& a) { return plan(a, nullptr).bytes; }
size_t linear8_bwd_bytes(const sadmm_linear8_bwd_args& a) { return plan(a, nullptr).bytes; }
size_t gated8_fwd_bytes(const sadmm_gated8_fwd_args& a) { return plan(a, nullptr).bytes; }
size_t gated8_bwd_bytes(const sadmm_gated8_bwd_args& a) { return plan(a, nullptr).bytes; }

sadmm_status launch_linear8_fwd(const sadmm_linear8_fwd_args& a, void* ws, cudaStream_t s) { return run(plan(a, ws), s); }
sadmm_status launch_gated8_fwd(const sadmm_gated8_fwd_args& a, void* ws, cudaStream_t s) { return run(plan(a, ws), s); }

sadmm_status launch_linear8_bwd(const sadmm_linear8_bwd_args& a, void* ws, cudaStream_t s)
{
    if (!a.tokens)
        return zero(a.dw, a.lddw, a.dwdt, a.n_out, a.n_in, s) && zero(a.db, a.n_out, s) ? SADMM_OK : SADMM_ECUDA;
    return run(plan(a, ws), s);
}

sadmm_status launch_gated8_bwd(const sadmm_gated8_bwd_args& a, void* ws, cudaStream_t s)
{
    if (!a.tokens)
        return zero(a.dwg, a.lddwg, a.dwdt, a.n_hidden, a.n_in, s) && zero(a.dwu, a.lddwu, a.dwdt, a.n_hidden, a.n_in, s) &&
                       zero(a.dbg, a.n_hidden, s) && zero(a.dbu, a.n_hidden, s)
                   ? SADMM_OK
                   : SADMM_ECUDA;
    return run(plan(a, ws), s);
}

}  // namespace sadmm
