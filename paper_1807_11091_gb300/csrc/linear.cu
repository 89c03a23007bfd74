// linear.cu -- the feed-forward products of the paper's method carried to a
// language model's layers: y = act(x W^T + b) + residual and the gated pair
// h = act(x Wg^T + bg) * (x Wu^T + bu), with their backward passes.  The
// products run in tgemm.cu; here are the passes around them:
//   k_dact     dz = dy act'(z), or dg and du of the gated pair, rounded to bf16
//              once for the tensor cores, and the bias gradients' partial sums
//              (fp32, taken before that rounding)
//   k_colsum   those partial sums added up in row-chunk order
//   k_realign  a matrix whose rows do not start on 16-byte boundaries, copied
//              to rows that do, which is what the tensor-memory accelerator reads
#include <string.h>

#include "act.cuh"
#include "common.cuh"
#include "internal.h"
#include "tgemm.cuh"

namespace sadmm {
namespace {

using bf16 = __nv_bfloat16;

// --------------------------------------------------------------- k_realign --

// A thread writes 8 elements (16 bytes) of a row.  Inside a row they come from
// the two aligned 16-byte words that hold them; at the row's ends one by one.
__global__ void __launch_bounds__(256) k_realign(const bf16* __restrict__ src, long long ld, bf16* __restrict__ dst,
                                                 long long ldd, long long rows, long long cols)
{
    pdl_wait();
    pdl_trigger();
    const long long per = ldd >> 3, n = rows * per;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256) {
        const long long r = i / per, c = (i - r * per) * 8;
        const bf16* p = src + r * ld + c;
        const int off = (int)((reinterpret_cast<uintptr_t>(p) & 15) >> 1);  // elements past a 16-byte boundary
        __align__(16) uint16_t e[8];
        if (c >= off && c + 16 <= cols) {
            const uint4* w = reinterpret_cast<const uint4*>(p - off);
            const uint4 lo = __ldg(w), hi = off ? __ldg(w + 1) : lo;
            const uint32_t v[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t a = 0, b = 0;  // words (off / 2) + j and the next
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    if (k == (off >> 1) + j) a = v[k];
                    if (k == (off >> 1) + j + 1) b = v[k];
                }
                const uint32_t u = (off & 1) ? __funnelshift_r(a, b, 16) : a;
                e[2 * j] = (uint16_t)(u & 0xffffu);
                e[2 * j + 1] = (uint16_t)(u >> 16);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                e[j] = c + j < cols ? __ldg(reinterpret_cast<const unsigned short*>(p) + j) : (uint16_t)0;
        }
        *reinterpret_cast<uint4*>(dst + r * ldd + c) = *reinterpret_cast<const uint4*>(e);
    }
}

sadmm_status realign(const void* src, long long ld, void* dst, long long ldd, long long rows, long long cols,
                     cudaStream_t s)
{
    const long long n = rows * (ldd >> 3);
    const long long blocks = (n + 255) / 256, most = (long long)device_sm_count() * 16;
    return launch_pdl(k_realign, dim3((unsigned)(blocks < most ? blocks : most)), dim3(256), 0, s,
                      static_cast<const bf16*>(src), ld, static_cast<bf16*>(dst), ldd, rows, cols) == cudaSuccess
               ? SADMM_OK
               : SADMM_ECUDA;
}

// ------------------------------------------------------------------ k_dact --

constexpr int kStrip = 256;  // columns of a CTA: 32 lanes x 8
constexpr int kWarps = 8;    // rows at a time

struct DactArgs {
    const void* dy;            // dy (dz = dy act'(z)) or dh, bf16 or fp32
    const bf16* z;             // z, or g; NULL: act' = 1
    const bf16* u;             // gated
    bf16* dz;                  // dz or dg; NULL: not written
    bf16* du;                  // gated
    float* part;               // [chunks][cols] partial column sums (gated: dg's, then du's at part_u); NULL: none
    float* part_u;
    long long lddy, ldz, ldu, ldd;
    long long rows, cols, chunk;
    int act;
    int dy_fp32;
};

// Eight consecutive elements; those at or past `left` read as zero.
SADMM_DEV void load8(const bf16* p, bool whole, long long left, float (&v)[8])
{
    if (whole) {
        const uint4 q = *reinterpret_cast<const uint4*>(p);
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[2 * j] = __uint_as_float(w[j] << 16);
            v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = j < left ? __bfloat162float(p[j]) : 0.0f;
    }
}

SADMM_DEV void load8(const float* p, bool whole, long long left, float (&v)[8])
{
    if (whole) {
        const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = j < left ? p[j] : 0.0f;
    }
}

// Eight consecutive elements of a row of the (aligned, padded) scratch copy.
SADMM_DEV void store8(bf16* p, const float (&v)[8])
{
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
        w[j] = *reinterpret_cast<const uint32_t*>(&h);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}

// A CTA takes a strip of 256 columns and a chunk of rows, a warp a row at a
// time, a lane 8 columns.  VEC: every matrix read starts its rows on 16-byte
// boundaries.  The scratch copies always do, and end their rows with zeros up
// to a multiple of 8 columns.
template <bool GATED, bool VEC>
__global__ void __launch_bounds__(kWarps * 32) k_dact(const DactArgs a)
{
    pdl_wait();
    pdl_trigger();
    __shared__ float red[kWarps][kStrip];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long long c = (long long)blockIdx.x * kStrip + lane * 8;
    const long long r0 = (long long)blockIdx.y * a.chunk, r1 = min(r0 + a.chunk, a.rows);
    const long long left = a.cols - c;
    const bool whole = VEC && left >= 8;
    float s[8], su[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) s[j] = su[j] = 0.0f;
    if (left > 0) {
        with_act(a.z ? a.act : SADMM_ACT_NONE, [&](auto tag) {
            constexpr int A = decltype(tag)::value;
#pragma unroll 2
            for (long long r = r0 + warp; r < r1; r += kWarps) {
                float d[8], z[8], u[8];
                if (a.dy_fp32)
                    load8(static_cast<const float*>(a.dy) + r * a.lddy + c, whole, left, d);
                else
                    load8(static_cast<const bf16*>(a.dy) + r * a.lddy + c, whole, left, d);
                if (A != SADMM_ACT_NONE || GATED) load8(a.z + r * a.ldz + c, whole, left, z);
                if (GATED) load8(a.u + r * a.ldu + c, whole, left, u);
                if (GATED) {
                    float du[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        du[j] = d[j] * act_f32<A>(z[j]);
                        d[j] = d[j] * u[j] * dact_f32<A>(z[j]);
                        s[j] += d[j];
                        su[j] += du[j];
                    }
                    store8(a.du + r * a.ldd + c, du);
                    store8(a.dz + r * a.ldd + c, d);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        if (A != SADMM_ACT_NONE) d[j] *= dact_f32<A>(z[j]);
                        s[j] += d[j];
                    }
                    if (a.dz) store8(a.dz + r * a.ldd + c, d);
                }
            }
        });
    }
    if (!a.part) return;
#pragma unroll
    for (int half = 0; half < (GATED ? 2 : 1); ++half) {
        if (half) __syncthreads();
#pragma unroll
        for (int j = 0; j < 8; ++j) red[warp][j * 32 + lane] = half ? su[j] : s[j];
        __syncthreads();
        // thread t adds up column 8 (t % 32) + t / 32 of the strip
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) v += red[w][threadIdx.x];
        const long long col = (long long)blockIdx.x * kStrip + lane * 8 + warp;
        if (col < a.cols) (half ? a.part_u : a.part)[(long long)blockIdx.y * a.cols + col] = v;
    }
}

// db[c] = the sum of part[0 .. chunks-1][c], eight groups of chunks at a time.
// blockIdx.y selects the second sum of the gated pair.
__global__ void __launch_bounds__(256) k_colsum(const float* __restrict__ part, const float* __restrict__ part2,
                                                float* __restrict__ out, float* __restrict__ out2, long long cols,
                                                int chunks)
{
    pdl_wait();
    pdl_trigger();
    __shared__ float red[8][32];
    const float* p = blockIdx.y ? part2 : part;
    float* o = blockIdx.y ? out2 : out;
    const int g = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long long c = (long long)blockIdx.x * 32 + lane;
    float v = 0.0f;
    if (c < cols)
        for (int k = g; k < chunks; k += 8) v += p[k * cols + c];
    red[g][lane] = v;
    __syncthreads();
    if (g == 0 && c < cols && o) {
        for (int k = 1; k < 8; ++k) v += red[k][lane];
        o[c] = v;
    }
}

// Rows of a chunk: enough CTAs to fill the device, at most 128 partial sums a column.
long long dact_chunk(long long rows)
{
    long long c = (rows + 127) / 128;
    if (c < 64) c = 64;
    return round_up(c, kWarps);
}
long long dact_chunks(long long rows) { return (rows + dact_chunk(rows) - 1) / dact_chunk(rows); }

sadmm_status launch_dact(DactArgs a, bool gated, cudaStream_t s)
{
    a.chunk = dact_chunk(a.rows);
    const dim3 grid((unsigned)((a.cols + kStrip - 1) / kStrip), (unsigned)dact_chunks(a.rows));
    bool vec = (reinterpret_cast<uintptr_t>(a.dy) & 15) == 0 && a.lddy % (a.dy_fp32 ? 4 : 8) == 0;
    if (a.z) vec = vec && tg_aligned(a.z, a.ldz);
    if (a.u) vec = vec && tg_aligned(a.u, a.ldu);
    auto k = gated ? (vec ? k_dact<true, true> : k_dact<true, false>)
                   : (vec ? k_dact<false, true> : k_dact<false, false>);
    return launch_pdl(k, grid, dim3(kWarps * 32), 0, s, a) == cudaSuccess ? SADMM_OK : SADMM_ECUDA;
}

// ------------------------------------------------------------------- parts --

// Scratch handed out in order, each piece on a 256-byte boundary.  With base
// NULL it only adds up the sizes.
struct Scratch {
    char* base;
    size_t used;
    void* take(size_t bytes)
    {
        void* p = base ? base + used : nullptr;
        used += (size_t)round_up((long long)bytes, 256);
        return p;
    }
};

// A matrix as the products read it: where it lies, or a copy in scratch.
struct Source {
    const void* p;
    long long ld;
    void* copy;
};
Source place(Scratch& w, const void* p, long long rows, long long cols, long long ld)
{
    Source o = {p, ld, nullptr};
    if (!tg_aligned(p, ld)) {
        o.ld = round_up(cols, 8);
        o.copy = w.take((size_t)rows * (size_t)o.ld * 2);
    }
    return o;
}
sadmm_status fill(Source& o, const void* p, long long rows, long long cols, long long ld, cudaStream_t s)
{
    if (tg_aligned(p, ld)) return SADMM_OK;
    o.p = o.copy;
    return realign(p, ld, o.copy, o.ld, rows, cols, s);
}

TgOperand kmajor(const Source& o, long long rows, long long k) { return {o.p, rows, k, o.ld, true}; }
TgOperand across(const Source& o, long long rows, long long k) { return {o.p, rows, k, o.ld, false}; }

// rows x cols zeros, for an empty sum
sadmm_status zero(void* p, long long ld, int dt, long long rows, long long cols, cudaStream_t s)
{
    const size_t es = dt == SADMM_BF16 ? 2 : 4;
    return !p || cudaMemset2DAsync(p, (size_t)ld * es, 0, (size_t)cols * es, (size_t)rows, s) == cudaSuccess
               ? SADMM_OK
               : SADMM_ECUDA;
}

struct LinearFwdPlan {
    Source x, w;
};
LinearFwdPlan plan_linear_fwd(const sadmm_linear_fwd_args& a, Scratch& w)
{
    return {place(w, a.x, a.tokens, a.n_in, a.ldx), place(w, a.w, a.n_out, a.n_in, a.ldw)};
}

struct LinearBwdPlan {
    Source x, w, dz;
    bool own_dz;  // dz is formed in scratch (an activation, fp32 or unaligned dy)
    float* part;
};
LinearBwdPlan plan_linear_bwd(const sadmm_linear_bwd_args& a, Scratch& w)
{
    LinearBwdPlan p;
    memset(&p, 0, sizeof(p));
    if (a.dw) p.x = place(w, a.x, a.tokens, a.n_in, a.ldx);
    if (a.dx) p.w = place(w, a.w, a.n_out, a.n_in, a.ldw);
    p.own_dz = (a.dx || a.dw) && (a.act != SADMM_ACT_NONE || a.dydt != SADMM_BF16 || !tg_aligned(a.dy, a.lddy));
    p.dz = {a.dy, a.lddy, nullptr};
    if (p.own_dz) {
        p.dz.ld = round_up(a.n_out, 8);
        p.dz.p = p.dz.copy = w.take((size_t)a.tokens * (size_t)p.dz.ld * 2);
    }
    if (a.db) p.part = static_cast<float*>(w.take((size_t)dact_chunks(a.tokens) * (size_t)a.n_out * 4));
    return p;
}

struct GatedFwdPlan {
    Source x, wg, wu;
};
GatedFwdPlan plan_gated_fwd(const sadmm_gated_fwd_args& a, Scratch& w)
{
    return {place(w, a.x, a.tokens, a.n_in, a.ldx), place(w, a.wg, a.n_hidden, a.n_in, a.ldwg),
            place(w, a.wu, a.n_hidden, a.n_in, a.ldwu)};
}

struct GatedBwdPlan {
    Source x, wg, wu, dg, du;
    float *part_g, *part_u;
};
GatedBwdPlan plan_gated_bwd(const sadmm_gated_bwd_args& a, Scratch& w)
{
    GatedBwdPlan p;
    memset(&p, 0, sizeof(p));
    if (a.dwg) p.x = place(w, a.x, a.tokens, a.n_in, a.ldx);
    if (a.dx) {
        p.wg = place(w, a.wg, a.n_hidden, a.n_in, a.ldwg);
        p.wu = place(w, a.wu, a.n_hidden, a.n_in, a.ldwu);
    }
    const long long ld = round_up(a.n_hidden, 8);
    p.dg.ld = p.du.ld = ld;
    p.dg.p = p.dg.copy = w.take((size_t)a.tokens * (size_t)ld * 2);
    p.du.p = p.du.copy = w.take((size_t)a.tokens * (size_t)ld * 2);
    if (a.dbg || a.dbu) {
        const size_t bytes = (size_t)dact_chunks(a.tokens) * (size_t)a.n_hidden * 4;
        p.part_g = static_cast<float*>(w.take(bytes));
        p.part_u = static_cast<float*>(w.take(bytes));
    }
    return p;
}

}  // namespace

sadmm_status launch_colsum(const float* part, const float* part2, float* out, float* out2, long long cols, int parts,
                           cudaStream_t s)
{
    const dim3 grid((unsigned)((cols + 31) / 32), part2 ? 2u : 1u);
    return launch_pdl(k_colsum, grid, dim3(256), 0, s, part, part2, out, out2, cols, parts) == cudaSuccess
               ? SADMM_OK
               : SADMM_ECUDA;
}

#define SADMM_TRY(call)                          \
    do {                                         \
        const sadmm_status st_ = (call);         \
        if (st_ != SADMM_OK) return st_;         \
    } while (0)

size_t linear_fwd_bytes(const sadmm_linear_fwd_args& a)
{
    Scratch w = {nullptr, 0};
    plan_linear_fwd(a, w);
    return w.used;
}

size_t linear_bwd_bytes(const sadmm_linear_bwd_args& a)
{
    Scratch w = {nullptr, 0};
    plan_linear_bwd(a, w);
    return w.used;
}

size_t gated_fwd_bytes(const sadmm_gated_fwd_args& a)
{
    Scratch w = {nullptr, 0};
    plan_gated_fwd(a, w);
    return w.used;
}

size_t gated_bwd_bytes(const sadmm_gated_bwd_args& a)
{
    Scratch w = {nullptr, 0};
    plan_gated_bwd(a, w);
    return w.used;
}

sadmm_status launch_linear_fwd(const sadmm_linear_fwd_args& a, void* ws, cudaStream_t s)
{
    if (a.tokens == 0) return SADMM_OK;
    Scratch w = {static_cast<char*>(ws), 0};
    LinearFwdPlan p = plan_linear_fwd(a, w);
    SADMM_TRY(fill(p.x, a.x, a.tokens, a.n_in, a.ldx, s));
    SADMM_TRY(fill(p.w, a.w, a.n_out, a.n_in, a.ldw, s));
    TgProblem t;
    memset(&t, 0, sizeof(t));
    t.mode = kTgSingle;
    t.a[0] = kmajor(p.x, a.tokens, a.n_in);
    t.b[0] = kmajor(p.w, a.n_out, a.n_in);
    t.m = a.tokens;
    t.n = a.n_out;
    t.bias = a.bias;
    t.act = a.act;
    t.y = {a.y, a.ldy, a.ydt};
    t.residual = {const_cast<void*>(a.residual), a.ldr, a.ydt};
    t.z = {a.z, a.ldz, SADMM_BF16};
    return launch_tgemm(&t, 1, s);
}

sadmm_status launch_linear_bwd(const sadmm_linear_bwd_args& a, void* ws, cudaStream_t s)
{
    if (a.tokens == 0) {
        SADMM_TRY(zero(a.dw, a.lddw, a.dwdt, a.n_out, a.n_in, s));
        return zero(a.db, a.n_out, SADMM_FP32, 1, a.n_out, s);
    }
    Scratch w = {static_cast<char*>(ws), 0};
    LinearBwdPlan p = plan_linear_bwd(a, w);
    if (p.own_dz || a.db) {
        DactArgs d;
        memset(&d, 0, sizeof(d));
        d.dy = a.dy;
        d.lddy = a.lddy;
        d.dy_fp32 = a.dydt == SADMM_FP32;
        d.z = a.act == SADMM_ACT_NONE ? nullptr : static_cast<const bf16*>(a.z);
        d.ldz = a.ldz;
        d.dz = static_cast<bf16*>(p.dz.copy);
        d.ldd = p.dz.ld;
        d.part = p.part;
        d.rows = a.tokens;
        d.cols = a.n_out;
        d.act = a.act;
        SADMM_TRY(launch_dact(d, false, s));
    }
    if (a.dx) SADMM_TRY(fill(p.w, a.w, a.n_out, a.n_in, a.ldw, s));
    if (a.dw) SADMM_TRY(fill(p.x, a.x, a.tokens, a.n_in, a.ldx, s));
    TgProblem t[2];
    memset(t, 0, sizeof(t));
    t[0].mode = t[1].mode = kTgSingle;
    t[0].a[0] = kmajor(p.dz, a.tokens, a.n_out);
    t[0].b[0] = across(p.w, a.n_in, a.n_out);
    t[0].m = a.tokens;
    t[0].n = t[1].n = a.n_in;
    t[0].y = {a.dx, a.lddx, a.dxdt};
    t[0].skip = !a.dx;
    t[1].a[0] = across(p.dz, a.n_out, a.tokens);
    t[1].b[0] = across(p.x, a.n_in, a.tokens);
    t[1].m = a.n_out;
    t[1].y = {a.dw, a.lddw, a.dwdt};
    t[1].skip = !a.dw;
    SADMM_TRY(launch_tgemm(t, 2, s));
    if (a.db) SADMM_TRY(launch_colsum(p.part, nullptr, a.db, nullptr, a.n_out, (int)dact_chunks(a.tokens), s));
    return SADMM_OK;
}

sadmm_status launch_gated_fwd(const sadmm_gated_fwd_args& a, void* ws, cudaStream_t s)
{
    if (a.tokens == 0) return SADMM_OK;
    Scratch w = {static_cast<char*>(ws), 0};
    GatedFwdPlan p = plan_gated_fwd(a, w);
    SADMM_TRY(fill(p.x, a.x, a.tokens, a.n_in, a.ldx, s));
    SADMM_TRY(fill(p.wg, a.wg, a.n_hidden, a.n_in, a.ldwg, s));
    SADMM_TRY(fill(p.wu, a.wu, a.n_hidden, a.n_in, a.ldwu, s));
    TgProblem t;
    memset(&t, 0, sizeof(t));
    t.mode = kTgGated;
    t.a[0] = t.a[1] = kmajor(p.x, a.tokens, a.n_in);
    t.b[0] = kmajor(p.wg, a.n_hidden, a.n_in);
    t.b[1] = kmajor(p.wu, a.n_hidden, a.n_in);
    t.m = a.tokens;
    t.n = a.n_hidden;
    t.bias = a.bg;
    t.bias2 = a.bu;
    t.act = a.act;
    t.y = {a.h, a.ldh, SADMM_BF16};
    t.z = {a.g, a.ldg, SADMM_BF16};
    t.u = {a.u, a.ldu, SADMM_BF16};
    return launch_tgemm(&t, 1, s);
}

sadmm_status launch_gated_bwd(const sadmm_gated_bwd_args& a, void* ws, cudaStream_t s)
{
    if (a.tokens == 0) {
        SADMM_TRY(zero(a.dwg, a.lddwg, a.dwdt, a.n_hidden, a.n_in, s));
        SADMM_TRY(zero(a.dwu, a.lddwu, a.dwdt, a.n_hidden, a.n_in, s));
        SADMM_TRY(zero(a.dbg, a.n_hidden, SADMM_FP32, 1, a.n_hidden, s));
        return zero(a.dbu, a.n_hidden, SADMM_FP32, 1, a.n_hidden, s);
    }
    Scratch w = {static_cast<char*>(ws), 0};
    GatedBwdPlan p = plan_gated_bwd(a, w);
    DactArgs d;
    memset(&d, 0, sizeof(d));
    d.dy = a.dh;
    d.lddy = a.lddh;
    d.z = static_cast<const bf16*>(a.g);
    d.ldz = a.ldg;
    d.u = static_cast<const bf16*>(a.u);
    d.ldu = a.ldu;
    d.dz = static_cast<bf16*>(p.dg.copy);
    d.du = static_cast<bf16*>(p.du.copy);
    d.ldd = p.dg.ld;
    d.part = p.part_g;
    d.part_u = p.part_u;
    d.rows = a.tokens;
    d.cols = a.n_hidden;
    d.act = a.act;
    SADMM_TRY(launch_dact(d, true, s));
    if (a.dx) {
        SADMM_TRY(fill(p.wg, a.wg, a.n_hidden, a.n_in, a.ldwg, s));
        SADMM_TRY(fill(p.wu, a.wu, a.n_hidden, a.n_in, a.ldwu, s));
    }
    if (a.dwg) SADMM_TRY(fill(p.x, a.x, a.tokens, a.n_in, a.ldx, s));
    TgProblem t[3];
    memset(t, 0, sizeof(t));
    t[0].mode = kTgSum;
    t[0].a[0] = kmajor(p.dg, a.tokens, a.n_hidden);
    t[0].a[1] = kmajor(p.du, a.tokens, a.n_hidden);
    t[0].b[0] = across(p.wg, a.n_in, a.n_hidden);
    t[0].b[1] = across(p.wu, a.n_in, a.n_hidden);
    t[0].m = a.tokens;
    t[0].n = a.n_in;
    t[0].y = {a.dx, a.lddx, a.dxdt};
    t[0].skip = !a.dx;
    for (int i = 1; i < 3; ++i) {
        t[i].mode = kTgSingle;
        t[i].a[0] = across(i == 1 ? p.dg : p.du, a.n_hidden, a.tokens);
        t[i].b[0] = across(p.x, a.n_in, a.tokens);
        t[i].m = a.n_hidden;
        t[i].n = a.n_in;
        t[i].y = i == 1 ? TgMatrix{a.dwg, a.lddwg, a.dwdt} : TgMatrix{a.dwu, a.lddwu, a.dwdt};
        t[i].skip = !a.dwg;
    }
    SADMM_TRY(launch_tgemm(t, 3, s));
    if (p.part_g) SADMM_TRY(launch_colsum(p.part_g, p.part_u, a.dbg, a.dbu, a.n_hidden, (int)dact_chunks(a.tokens), s));
    return SADMM_OK;
}

}  // namespace sadmm
