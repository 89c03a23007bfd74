// linear.cu -- the feed-forward products of the paper's method carried to a
// language model's layers: y = act(x W^T + b) + residual and the gated pair
// h = act(x Wg^T + bg) * (x Wu^T + bu), with their backward passes.  The
// products run in tgemm.cu; here are the passes around them:
//   k_dact     dz = dy act'(z), or dg and du of the gated pair, rounded to bf16
//              once for the tensor cores, and the bias gradients (fp32 sums,
//              taken before that rounding)
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

struct Copies {
    const bf16* src[3];
    bf16* dst[3];
    long long ld[3], ldd[3], rows[3];
    int cols[3];
    int* status;
};

// Matrix blockIdx.y, a warp a row's 1024 elements (segments blockIdx.z, blockIdx.z +
// gridDim.z, ...), a lane 8 elements (16 bytes) at a time, all in flight together.
// Inside a row they come from the two aligned 16-byte words that hold them (funnel
// shifts), at the row's ends one by one.
__global__ void __launch_bounds__(256) k_realign(const Copies a)
{
    pdl_wait();
    pdl_trigger();
    const int m = blockIdx.y, lane = threadIdx.x & 31;
    const int cols = a.cols[m], words = (int)(a.ldd[m] >> 3);
    const long long step = (long long)gridDim.x * 8;
    for (long long r = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); r < a.rows[m]; r += step) {
        const bf16* row = a.src[m] + r * a.ld[m];
        uint4* to = reinterpret_cast<uint4*>(a.dst[m] + r * a.ldd[m]);
        // elements of the row's first 16-byte word that lie before the row
        const int off = (int)((reinterpret_cast<uintptr_t>(row) & 15) >> 1);
        const uint4* from = reinterpret_cast<const uint4*>(row - off);
        const int sh = (off & 1) * 16, w0 = off >> 1;
        for (int z = blockIdx.z * 128 + lane; z < words; z += gridDim.z * 128) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int i = z + 32 * k;
                if (i >= words) break;
                const int c = i * 8;
                uint4 o;
                if (c >= off && c + 16 <= cols && dbg_run(c - off, 16, cols, a.status)) {
                    const uint4 lo = __ldg(from + i), hi = __ldg(from + i + 1);
                    // words w0 .. w0 + 4 of the eight (w0 is the row's: the same for the warp)
                    uint32_t v0, v1, v2, v3, v4;
                    if (w0 == 0) v0 = lo.x, v1 = lo.y, v2 = lo.z, v3 = lo.w, v4 = hi.x;
                    else if (w0 == 1) v0 = lo.y, v1 = lo.z, v2 = lo.w, v3 = hi.x, v4 = hi.y;
                    else if (w0 == 2) v0 = lo.z, v1 = lo.w, v2 = hi.x, v3 = hi.y, v4 = hi.z;
                    else v0 = lo.w, v1 = hi.x, v2 = hi.y, v3 = hi.z, v4 = hi.w;
                    o = make_uint4(__funnelshift_r(v0, v1, sh), __funnelshift_r(v1, v2, sh), __funnelshift_r(v2, v3, sh),
                                   __funnelshift_r(v3, v4, sh));
                } else {
                    uint32_t e[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        e[j] = c + j < cols ? __ldg(reinterpret_cast<const unsigned short*>(row) + c + j) : 0u;
                    o = make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
                }
                if (dbg_run(c, 8, a.ldd[m], a.status)) to[i] = o;
            }
        }
    }
}

// ------------------------------------------------------------------ k_dact --

constexpr int kStrip = 64;        // columns of a CTA
constexpr int kDactThreads = 256;
constexpr int kDactCluster = 8;   // CTAs that share a strip's column sums

struct DactArgs {
    const void* dy;            // dy (dz = dy act'(z)) or dh, bf16 or fp32
    const bf16* z;             // z, or g; NULL: act' = 1
    const bf16* u;             // gated
    bf16* dz;                  // dz or dg; NULL: not written
    bf16* du;                  // gated
    float* db;                 // column sums of dz (dg); NULL: none
    float* dbu;                // of du
    long long lddy, ldz, ldu, ldd;
    long long rows, cols, chunk;
    int act;
    int cluster;               // CTAs of a strip, in one cluster where sums are wanted
    int sums;
    int* status;
};

// N consecutive elements, as they lie in memory.
template <typename T, int N>
struct Raw {
    T e[N];
};

// Eight neighbours by 16-byte loads; one element otherwise.
SADMM_DEV void load_raw(const bf16* p, Raw<bf16, 8>& r)
{
    *reinterpret_cast<uint4*>(r.e) = *reinterpret_cast<const uint4*>(p);
}
SADMM_DEV void load_raw(const float* p, Raw<float, 8>& r)
{
    reinterpret_cast<float4*>(r.e)[0] = reinterpret_cast<const float4*>(p)[0];
    reinterpret_cast<float4*>(r.e)[1] = reinterpret_cast<const float4*>(p)[1];
}
template <typename T>
SADMM_DEV void load_raw(const T*, Raw<T, 2>&)  // (not called: two columns are loaded one by one)
{
}
SADMM_DEV float f32(bf16 v) { return __bfloat162float(v); }
SADMM_DEV float f32(float v) { return v; }

// A CTA takes a strip of 64 columns and a chunk of rows.  VEC: every matrix read
// starts its rows on 16-byte boundaries; a thread takes 8 neighbouring columns
// (where all are inside) of every 32nd row, else columns 32 apart of every 8th,
// so that a warp's loads are neighbours either way.  Several rows' loads are in
// flight before the first is used (bound by memory).  The scratch copies start
// rows on 16-byte boundaries, with zeros up to a multiple of 8 columns.  Column
// sums: over a thread's rows in order, then the CTA's threads, then the
// cluster's CTAs in rank order.  Measured: the sums alone of 8192 x 2048 bf16 6 us
// (from L2), the gated pair's of 4096 x 5464 45 us (224 MB: 34 us of a copy),
// act' of 1025 x 2731 off 16-byte boundaries 7.8 us.
template <bool GATED, bool VEC, typename DY>
__global__ void __launch_bounds__(kDactThreads, GATED || !VEC ? 3 : 4) k_dact(const DactArgs a)
{
    constexpr int N = VEC ? 8 : 2;              // columns of a thread
    constexpr int L = VEC ? 32 : 8;             // rows at a time
    __shared__ float red[GATED ? 2 : 1][L][kStrip + 1];
    __shared__ float csum[2][kStrip];
    pdl_wait();
    if (!a.sums) pdl_trigger();  // (clusters do not: see common.cuh)
    const int rank = (int)(blockIdx.x % (unsigned)a.cluster);
    const long long c0 = (long long)(blockIdx.x / (unsigned)a.cluster) * kStrip;
    const int cl = VEC ? threadIdx.x & 7 : threadIdx.x & 31, rl = VEC ? threadIdx.x >> 3 : threadIdx.x >> 5;
    auto col = [&](int j) { return VEC ? cl * 8 + j : cl + 32 * j; };  // of the strip
    const long long left = a.cols - c0;
    const long long padded = ((a.cols + 7) & ~7ll) - c0;  // columns of the copies
    const long long r0 = (long long)rank * a.chunk, r1 = min(r0 + a.chunk, a.rows);
    const bool whole = VEC && cl * 8 + 8 <= left;
    const DY* dy = static_cast<const DY*>(a.dy) + c0;
    const bf16 *zp = a.z + c0, *up = a.u + c0;
    float s[N], su[N];
#pragma unroll
    for (int j = 0; j < N; ++j) s[j] = su[j] = 0.0f;

    with_act(a.z ? a.act : SADMM_ACT_NONE, [&](auto tag) {
        constexpr int A = decltype(tag)::value;
        constexpr bool Z = GATED || A != SADMM_ACT_NONE;
        constexpr int U = VEC && !Z ? 4 : VEC ? 2 : 4;  // turns whose loads are in flight together
        // one row's values: sums them up and writes the copies
        auto row = [&](long long r, const Raw<DY, N>& rd, const Raw<bf16, N>& rz, const Raw<bf16, N>& ru) {
            float d[N], e[N];
#pragma unroll
            for (int j = 0; j < N; ++j) {
                d[j] = f32(rd.e[j]);
                float act = 0.0f, slope = 1.0f;
                if (Z) act_slope_f32<A>(f32(rz.e[j]), act, slope);
                // (products and sums not fused: the sums' bits do not depend on whether the products are also stored)
                if (GATED) {
                    e[j] = __fmul_rn(d[j], act);
                    d[j] = __fmul_rn(__fmul_rn(d[j], f32(ru.e[j])), slope);
                    su[j] = __fadd_rn(su[j], e[j]);
                } else if (A != SADMM_ACT_NONE) {
                    d[j] = __fmul_rn(d[j], slope);
                }
                s[j] = __fadd_rn(s[j], d[j]);
            }
            if (VEC) {
                if (a.dz && cl * 8 < left && dbg_run(c0 + cl * 8, 8, a.ldd, a.status) && dbg_in(r, a.rows, a.status)) {
                    __align__(16) Raw<bf16, 8> o;
#pragma unroll
                    for (int j = 0; j < N; ++j) o.e[j] = __float2bfloat16_rn(d[j]);
                    *reinterpret_cast<uint4*>(a.dz + r * a.ldd + c0 + cl * 8) = *reinterpret_cast<const uint4*>(o.e);
                    if (GATED) {
#pragma unroll
                        for (int j = 0; j < N; ++j) o.e[j] = __float2bfloat16_rn(e[j]);
                        *reinterpret_cast<uint4*>(a.du + r * a.ldd + c0 + cl * 8) = *reinterpret_cast<const uint4*>(o.e);
                    }
                }
            } else if (a.dz) {
#pragma unroll
                for (int j = 0; j < N; ++j)
                    if (col(j) < padded && dbg_in(c0 + col(j), a.ldd, a.status) && dbg_in(r, a.rows, a.status)) {
                        a.dz[r * a.ldd + c0 + col(j)] = __float2bfloat16_rn(d[j]);
                        if (GATED) a.du[r * a.ldd + c0 + col(j)] = __float2bfloat16_rn(e[j]);
                    }
            }
        };
        auto load = [&](auto inside, long long r, Raw<DY, N>& rd, Raw<bf16, N>& rz, Raw<bf16, N>& ru) {
            if constexpr (decltype(inside)::value) {
                if (!dbg_run(c0 + cl * 8, 8, a.cols, a.status) || !dbg_in(r, a.rows, a.status)) {
                    rd = {}, rz = {}, ru = {};
                    return;
                }
                load_raw(dy + r * a.lddy + cl * 8, rd);
                if (Z) load_raw(zp + r * a.ldz + cl * 8, rz);
                if (GATED) load_raw(up + r * a.ldu + cl * 8, ru);
            } else {
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    // past the end: zeros
                    const bool in = col(j) < left && dbg_in(c0 + col(j), a.cols, a.status) && dbg_in(r, a.rows, a.status);
                    rd.e[j] = in ? dy[r * a.lddy + col(j)] : DY(0.0f);
                    if (Z) rz.e[j] = in ? zp[r * a.ldz + col(j)] : bf16(0.0f);
                    if (GATED) ru.e[j] = in ? up[r * a.ldu + col(j)] : bf16(0.0f);
                }
            }
        };
        // (the choice outside the loop: inside it the loads of several rows would not be in flight together)
        auto rows = [&](auto inside) {
            long long r = r0 + rl;
            for (; r + (U - 1) * L < r1; r += U * L) {
                __align__(16) Raw<DY, N> rd[U];
                __align__(16) Raw<bf16, N> rz[U], ru[U];
#pragma unroll
                for (int i = 0; i < U; ++i) load(inside, r + i * L, rd[i], rz[i], ru[i]);
#pragma unroll
                for (int i = 0; i < U; ++i) row(r + i * L, rd[i], rz[i], ru[i]);
            }
            for (; r < r1; r += L) {
                __align__(16) Raw<DY, N> rd;
                __align__(16) Raw<bf16, N> rz, ru;
                load(inside, r, rd, rz, ru);
                row(r, rd, rz, ru);
            }
        };
        if constexpr (VEC) {
            if (whole)
                rows(ActTag<1>());
            else if (cl * 8 < left)
                rows(ActTag<0>());
        } else {
            rows(ActTag<0>());
        }
    });
    if (!a.sums) return;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        red[0][rl][col(j)] = s[j];
        if (GATED) red[GATED ? 1 : 0][rl][col(j)] = su[j];
    }
    __syncthreads();
    if (threadIdx.x < (GATED ? 2 : 1) * kStrip) {
        const int which = threadIdx.x / kStrip, c = threadIdx.x % kStrip;
        float v = 0.0f;
#pragma unroll 8
        for (int i = 0; i < L; ++i) v += red[which][i][c];
        csum[which][c] = v;
    }
    cluster_sync();
    const int share = kStrip / a.cluster;  // columns that this CTA finishes
    if ((int)threadIdx.x < (GATED ? 2 : 1) * share) {
        const int which = threadIdx.x / share, c = rank * share + threadIdx.x % share;
        float v = 0.0f;
        for (int i = 0; i < a.cluster; ++i) v += ld_cluster_f32(map_rank(smem_u32(&csum[which][c]), (uint32_t)i));
        float* out = which ? a.dbu : a.db;
        if (out && c < left && dbg_in(c0 + c, a.cols, a.status)) out[c0 + c] = v;
    }
    cluster_sync();  // the others have read this CTA's sums
}

template <bool GATED, bool VEC, typename DY>
sadmm_status run_dact(const DactArgs& a, cudaStream_t s)
{
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)a.cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((a.cols + kStrip - 1) / kStrip) * (unsigned)a.cluster);
    cfg.blockDim = dim3(kDactThreads);
    cfg.stream = s;
    cfg.attrs = attr;
    cfg.numAttrs = a.sums ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, k_dact<GATED, VEC, DY>, a) == cudaSuccess ? SADMM_OK : SADMM_ECUDA;
}

sadmm_status launch_dact(DactArgs a, bool gated, bool fp32, cudaStream_t s)
{
    a.sums = a.db || a.dbu;
    a.status = device_status_ptr();
    // with sums at most a cluster's CTAs share a strip's rows, of at least 32 each; without, chunks of 128
    if (a.sums) {
        a.cluster = 1;
        while (a.cluster < kDactCluster && a.rows > 32ll * a.cluster) a.cluster *= 2;
    } else {
        a.cluster = (int)((a.rows + 127) / 128 < 4096 ? (a.rows + 127) / 128 : 4096);
    }
    a.chunk = (a.rows + a.cluster - 1) / a.cluster;
    bool vec = (reinterpret_cast<uintptr_t>(a.dy) & 15) == 0 && a.lddy % (fp32 ? 4 : 8) == 0;
    if (a.z) vec = vec && tg_aligned(a.z, a.ldz);
    if (a.u) vec = vec && tg_aligned(a.u, a.ldu);
    if (gated) return vec ? run_dact<true, true, bf16>(a, s) : run_dact<true, false, bf16>(a, s);
    if (fp32) return vec ? run_dact<false, true, float>(a, s) : run_dact<false, false, float>(a, s);
    return vec ? run_dact<false, true, bf16>(a, s) : run_dact<false, false, bf16>(a, s);
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
// The copies that a call's sources need, in one launch.
struct Filler {
    Copies c;
    int n = 0;
    long long rows = 0, widest = 0;
    void add(Source& o, const void* p, long long rows_, long long cols, long long ld)
    {
        if (tg_aligned(p, ld)) return;
        o.p = o.copy;
        c.src[n] = static_cast<const bf16*>(p);
        c.dst[n] = static_cast<bf16*>(o.copy);
        c.ld[n] = ld;
        c.ldd[n] = o.ld;
        c.rows[n] = rows_;
        c.cols[n] = (int)cols;
        if (rows_ > rows) rows = rows_;
        if (o.ld > widest) widest = o.ld;
        ++n;
    }
    sadmm_status run(cudaStream_t s)
    {
        if (!n) return SADMM_OK;
        c.status = device_status_ptr();
        const long long blocks = (rows + 7) / 8, most = 8ll * device_sm_count();
        const long long segments = (widest + 1023) / 1024;
        const dim3 grid((unsigned)(blocks < most ? blocks : most), (unsigned)n,
                        (unsigned)(segments < 65535 ? segments : 65535));
        return launch_pdl(k_realign, grid, dim3(256), 0, s, c) == cudaSuccess
                   ? SADMM_OK
                   : SADMM_ECUDA;
    }
};

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
    if (few_linear(a)) return {};
    return {place(w, a.x, a.tokens, a.n_in, a.ldx), place(w, a.w, a.n_out, a.n_in, a.ldw)};
}

struct LinearBwdPlan {
    Source x, w, dz;
    bool own_dz;  // dz is formed in scratch (an activation, fp32 or unaligned dy)
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
    return p;
}

struct GatedFwdPlan {
    Source x, wg, wu;
};
GatedFwdPlan plan_gated_fwd(const sadmm_gated_fwd_args& a, Scratch& w)
{
    if (few_gated(a)) return {};
    return {place(w, a.x, a.tokens, a.n_in, a.ldx), place(w, a.wg, a.n_hidden, a.n_in, a.ldwg),
            place(w, a.wu, a.n_hidden, a.n_in, a.ldwu)};
}

struct GatedBwdPlan {
    Source x, wg, wu, dg, du;
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
    return p;
}

}  // namespace

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
    if (few_linear(a)) return launch_few_linear(a, s);
    Scratch w = {static_cast<char*>(ws), 0};
    LinearFwdPlan p = plan_linear_fwd(a, w);
    Filler f;
    f.add(p.x, a.x, a.tokens, a.n_in, a.ldx);
    f.add(p.w, a.w, a.n_out, a.n_in, a.ldw);
    SADMM_TRY(f.run(s));
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
        d.z = a.act == SADMM_ACT_NONE ? nullptr : static_cast<const bf16*>(a.z);
        d.ldz = a.ldz;
        d.dz = static_cast<bf16*>(p.dz.copy);
        d.ldd = p.dz.ld;
        d.db = a.db;
        d.rows = a.tokens;
        d.cols = a.n_out;
        d.act = a.act;
        SADMM_TRY(launch_dact(d, false, a.dydt == SADMM_FP32, s));
    }
    Filler f;
    if (a.dx) f.add(p.w, a.w, a.n_out, a.n_in, a.ldw);
    if (a.dw) f.add(p.x, a.x, a.tokens, a.n_in, a.ldx);
    SADMM_TRY(f.run(s));
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
    return SADMM_OK;
}

sadmm_status launch_gated_fwd(const sadmm_gated_fwd_args& a, void* ws, cudaStream_t s)
{
    if (a.tokens == 0) return SADMM_OK;
    if (few_gated(a)) return launch_few_gated(a, s);
    Scratch w = {static_cast<char*>(ws), 0};
    GatedFwdPlan p = plan_gated_fwd(a, w);
    Filler f;
    f.add(p.x, a.x, a.tokens, a.n_in, a.ldx);
    f.add(p.wg, a.wg, a.n_hidden, a.n_in, a.ldwg);
    f.add(p.wu, a.wu, a.n_hidden, a.n_in, a.ldwu);
    SADMM_TRY(f.run(s));
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
    d.db = a.dbg;
    d.dbu = a.dbu;
    d.rows = a.tokens;
    d.cols = a.n_hidden;
    d.act = a.act;
    SADMM_TRY(launch_dact(d, true, false, s));
    Filler f;
    if (a.dx) {
        f.add(p.wg, a.wg, a.n_hidden, a.n_in, a.ldwg);
        f.add(p.wu, a.wu, a.n_hidden, a.n_in, a.ldwu);
    }
    if (a.dwg) f.add(p.x, a.x, a.tokens, a.n_in, a.ldx);
    SADMM_TRY(f.run(s));
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
    return SADMM_OK;
}

}  // namespace sadmm
