// norm.cu -- layer norm over the rows of a matrix, forward and backward, with
// the gradients of its weight and bias.
//
//   y = gamma xhat + beta,  xhat = (x - mean) rstd,  rstd = (var + eps)^-1/2
//   d = gamma dy,  dx = rstd (d - avg(d) - xhat avg(d xhat)) [+ dres]
//   dgamma = sum over rows of dy xhat,  dbeta = sum over rows of dy
//
// Bound by memory: a row is read once and kept in registers by the threads that
// share it (a warp, or a block for long rows), in fp32; mean and variance are
// taken one after the other from those registers, so the variance has no
// cancellation.  The backward's threads own fixed columns, add up their shares
// of dgamma and dbeta over the rows of their block in registers and leave one
// partial sum per block, which a second kernel adds up in block order.  Rows
// too long for registers are read again from cache instead.
#include <string.h>

#include "common.cuh"
#include "internal.h"

namespace sadmm {
namespace {

using bf16 = __nv_bfloat16;

SADMM_DEV float to_f32(float v) { return v; }
SADMM_DEV float to_f32(bf16 v) { return __bfloat162float(v); }
SADMM_DEV void put(float* p, float v) { *p = v; }
SADMM_DEV void put(bf16* p, float v) { *p = __float2bfloat16_rn(v); }

SADMM_DEV void load_vec(const bf16* p, float (&v)[8])
{
    const uint4 q = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        v[2 * j] = __uint_as_float(w[j] << 16);
        v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
    }
}
SADMM_DEV void load_vec(const float* p, float (&v)[8])
{
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
SADMM_DEV void store_vec(bf16* p, const float (&v)[8])
{
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
        w[j] = *reinterpret_cast<const uint32_t*>(&h);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
SADMM_DEV void store_vec(float* p, const float (&v)[8])
{
    reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}

// A row over G threads, E times 8 elements each.  VEC: the matrices' rows start
// on 16-byte boundaries and thread t's k-th eight are the neighbours from
// column (k G + t) 8; otherwise element j of them is column (8 k + j) G + t, so
// that a warp's loads are neighbours.
template <bool VEC>
struct Cols {
    int g, t, cols;
    SADMM_DEV int at(int k, int j) const { return VEC ? (k * g + t) * 8 + j : (8 * k + j) * g + t; }
    SADMM_DEV bool whole(int k) const { return VEC && at(k, 0) + 8 <= cols; }
};

template <bool VEC, typename T>
SADMM_DEV void load_row(const T* p, const Cols<VEC>& c, int k, float fill, float (&v)[8])
{
    if (c.whole(k)) {
        load_vec(p + c.at(k, 0), v);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = c.at(k, j) < c.cols ? to_f32(p[c.at(k, j)]) : fill;
    }
}

template <bool VEC, typename T>
SADMM_DEV void store_row(T* p, const Cols<VEC>& c, int k, const float (&v)[8])
{
    if (c.whole(k)) {
        store_vec(p + c.at(k, 0), v);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (c.at(k, j) < c.cols) put(p + c.at(k, j), v[j]);
    }
}

// Sums over the threads of a row: a warp, or the whole block (`slot` alternates
// between calls so that one barrier a call is enough).
SADMM_DEV float2 warp_sum(float2 v)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
        v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
    }
    return v;
}

template <bool BLOCK>
SADMM_DEV float2 row_sum(float2 v, float2 (*red)[32], int slot)
{
    v = warp_sum(v);
    if (BLOCK) {
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = blockDim.x >> 5;
        if (lane == 0) red[slot][warp] = v;
        __syncthreads();
        v = warp_sum(lane < n ? red[slot][lane] : make_float2(0.0f, 0.0f));
    }
    return v;
}

struct FwdArgs {
    const void* x;
    void* y;
    const float* gamma;
    const float* beta;
    float* mean;
    float* rstd;
    long long rows, ldx, ldy;
    int cols;
    float eps;
    float n;  // cols: sums are divided by it, so that a constant row's mean is that constant
};

template <typename X, typename Y, bool VEC, bool BLOCK, int E>
__global__ void __launch_bounds__(BLOCK ? 1024 : 256) k_ln_fwd(const FwdArgs a)
{
    __shared__ float2 red[2][32];
    pdl_wait();
    pdl_trigger();
    const int G = BLOCK ? blockDim.x : 32, R = BLOCK ? 1 : blockDim.x / 32;
    const Cols<VEC> c = {G, BLOCK ? (int)threadIdx.x : (int)(threadIdx.x & 31), a.cols};
    const long long r = (long long)blockIdx.x * R + (BLOCK ? 0 : threadIdx.x >> 5);
    if (r >= a.rows) return;
    const X* x = static_cast<const X*>(a.x) + r * a.ldx;
    float v[E][8];
    float2 s = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int k = 0; k < E; ++k) {
        load_row<VEC>(x, c, k, 0.0f, v[k]);
#pragma unroll
        for (int j = 0; j < 8; ++j) s.x += v[k][j];
    }
    const float mean = row_sum<BLOCK>(s, red, 0).x / a.n;
    s = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int k = 0; k < E; ++k)
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (c.at(k, j) < a.cols) {
                const float d = v[k][j] - mean;
                s.x += d * d;
            }
    const float rstd = rsqrtf(row_sum<BLOCK>(s, red, 1).x / a.n + a.eps);
    if (c.t == 0) {
        if (a.mean) a.mean[r] = mean;
        if (a.rstd) a.rstd[r] = rstd;
    }
    Y* y = static_cast<Y*>(a.y) + r * a.ldy;
#pragma unroll
    for (int k = 0; k < E; ++k) {
        float g[8], b[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] = 1.0f, b[j] = 0.0f;
        if (a.gamma) load_row<VEC>(a.gamma, c, k, 0.0f, g);
        if (a.beta) load_row<VEC>(a.beta, c, k, 0.0f, b);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[k][j] = (v[k][j] - mean) * rstd * g[j] + b[j];
        store_row<VEC>(y, c, k, v[k]);
    }
}

// Rows of any length: a block a row, read three times (from cache after the first).
template <typename X, typename Y>
__global__ void __launch_bounds__(1024) k_ln_fwd_long(const FwdArgs a)
{
    __shared__ float2 red[2][32];
    pdl_wait();
    pdl_trigger();
    const long long r = blockIdx.x;
    const X* x = static_cast<const X*>(a.x) + r * a.ldx;
    float2 s = make_float2(0.0f, 0.0f);
    for (int c = threadIdx.x; c < a.cols; c += 1024) s.x += to_f32(x[c]);
    const float mean = row_sum<true>(s, red, 0).x / a.n;
    s = make_float2(0.0f, 0.0f);
    for (int c = threadIdx.x; c < a.cols; c += 1024) {
        const float d = to_f32(x[c]) - mean;
        s.x += d * d;
    }
    const float rstd = rsqrtf(row_sum<true>(s, red, 1).x / a.n + a.eps);
    if (threadIdx.x == 0) {
        if (a.mean) a.mean[r] = mean;
        if (a.rstd) a.rstd[r] = rstd;
    }
    Y* y = static_cast<Y*>(a.y) + r * a.ldy;
    for (int c = threadIdx.x; c < a.cols; c += 1024)
        put(y + c, (to_f32(x[c]) - mean) * rstd * (a.gamma ? a.gamma[c] : 1.0f) + (a.beta ? a.beta[c] : 0.0f));
}

struct BwdArgs {
    const void* x;
    const void* dy;
    const void* dres;
    void* dx;
    const float* gamma;
    const float* mean;
    const float* rstd;
    float* part_g;  // [blocks][cols] partial dgamma, dbeta; NULL: not wanted
    float* part_b;
    long long rows, ldx, lddy, lddres, lddx;
    int cols;
    float n;
};

template <typename X, typename Y, bool VEC, bool BLOCK, int E>
__global__ void __launch_bounds__(BLOCK ? 1024 / E : 256) k_ln_bwd(const BwdArgs a)
{
    __shared__ float2 red[2][32];
    __shared__ float comb[BLOCK ? 1 : 8][BLOCK ? 1 : 256];
    pdl_wait();
    pdl_trigger();
    const int G = BLOCK ? blockDim.x : 32, R = BLOCK ? 1 : blockDim.x / 32;
    const int warp = threadIdx.x >> 5;
    const Cols<VEC> c = {G, BLOCK ? (int)threadIdx.x : (int)(threadIdx.x & 31), a.cols};
    float g[E][8], dg[E][8], db[E][8];
#pragma unroll
    for (int k = 0; k < E; ++k) {
#pragma unroll
        for (int j = 0; j < 8; ++j) g[k][j] = 1.0f, dg[k][j] = db[k][j] = 0.0f;
        if (a.gamma) load_row<VEC>(a.gamma, c, k, 0.0f, g[k]);
    }
    int slot = 0;
    for (long long r = (long long)blockIdx.x * R + (BLOCK ? 0 : warp); r < a.rows; r += (long long)gridDim.x * R) {
        const X* x = static_cast<const X*>(a.x) + r * a.ldx;
        const Y* dy = static_cast<const Y*>(a.dy) + r * a.lddy;
        const float mean = a.mean[r], rstd = a.rstd[r];
        float xh[E][8], d[E][8];
        float2 s = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int k = 0; k < E; ++k) {
            load_row<VEC>(x, c, k, mean, xh[k]);  // past the row's end: xhat = dy = 0
            load_row<VEC>(dy, c, k, 0.0f, d[k]);
        }
#pragma unroll
        for (int k = 0; k < E; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                xh[k][j] = (xh[k][j] - mean) * rstd;
                dg[k][j] += d[k][j] * xh[k][j];
                db[k][j] += d[k][j];
                d[k][j] *= g[k][j];
                s.x += d[k][j];
                s.y += d[k][j] * xh[k][j];
            }
        if (!a.dx) continue;
        s = row_sum<BLOCK>(s, red, slot);
        slot ^= 1;
        const float c1 = s.x / a.n, c2 = s.y / a.n;
        X* dx = static_cast<X*>(a.dx) + r * a.lddx;
#pragma unroll
        for (int k = 0; k < E; ++k) {
            float o[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = rstd * (d[k][j] - c1 - xh[k][j] * c2);
            if (a.dres) {
                float e[8];
                load_row<VEC>(static_cast<const X*>(a.dres) + r * a.lddres, c, k, 0.0f, e);
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] += e[j];
            }
            store_row<VEC>(dx, c, k, o);
        }
    }
    if (!a.part_g) return;
    float* pg = a.part_g + (long long)blockIdx.x * a.cols;
    float* pb = a.part_b + (long long)blockIdx.x * a.cols;
    if (BLOCK) {
#pragma unroll
        for (int k = 0; k < E; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (c.at(k, j) < a.cols) {
                    pg[c.at(k, j)] = dg[k][j];
                    pb[c.at(k, j)] = db[k][j];
                }
    } else {
        // the warps' sums added up in warp order, thread (j, lane) for element j of lane's eight
#pragma unroll
        for (int k = 0; k < E; ++k)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                __syncthreads();
#pragma unroll
                for (int j = 0; j < 8; ++j) comb[BLOCK ? 0 : warp][BLOCK ? 0 : j * 32 + c.t] = half ? db[k][j] : dg[k][j];
                __syncthreads();
                float v = 0.0f;
                for (int w = 0; w < R; ++w) v += comb[BLOCK ? 0 : w][BLOCK ? 0 : threadIdx.x];
                const int col = c.at(k, warp);
                if (col < a.cols) (half ? pb : pg)[col] = v;
            }
    }
}

// Rows of any length: dx, a block a row, read twice.
template <typename X, typename Y>
__global__ void __launch_bounds__(1024) k_ln_bwd_long(const BwdArgs a)
{
    __shared__ float2 red[2][32];
    pdl_wait();
    pdl_trigger();
    const long long r = blockIdx.x;
    const X* x = static_cast<const X*>(a.x) + r * a.ldx;
    const Y* dy = static_cast<const Y*>(a.dy) + r * a.lddy;
    const float mean = a.mean[r], rstd = a.rstd[r];
    float2 s = make_float2(0.0f, 0.0f);
    for (int c = threadIdx.x; c < a.cols; c += 1024) {
        const float d = to_f32(dy[c]) * (a.gamma ? a.gamma[c] : 1.0f);
        s.x += d;
        s.y += d * (to_f32(x[c]) - mean) * rstd;
    }
    s = row_sum<true>(s, red, 0);
    const float c1 = s.x / a.n, c2 = s.y / a.n;
    const X* dres = a.dres ? static_cast<const X*>(a.dres) + r * a.lddres : nullptr;
    X* dx = static_cast<X*>(a.dx) + r * a.lddx;
    for (int c = threadIdx.x; c < a.cols; c += 1024) {
        const float d = to_f32(dy[c]) * (a.gamma ? a.gamma[c] : 1.0f);
        const float o = rstd * (d - c1 - (to_f32(x[c]) - mean) * rstd * c2);
        put(dx + c, o + (dres ? to_f32(dres[c]) : 0.0f));
    }
}

// Rows of any length: partial dgamma and dbeta of 256 columns over the rows
// blockIdx.y, blockIdx.y + gridDim.y, ...
template <typename X, typename Y>
__global__ void __launch_bounds__(256) k_ln_cols_long(const BwdArgs a)
{
    pdl_wait();
    pdl_trigger();
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= a.cols) return;
    float g = 0.0f, b = 0.0f;
    for (long long r = blockIdx.y; r < a.rows; r += gridDim.y) {
        const float dy = to_f32(static_cast<const Y*>(a.dy)[r * a.lddy + c]);
        g += dy * (to_f32(static_cast<const X*>(a.x)[r * a.ldx + c]) - a.mean[r]) * a.rstd[r];
        b += dy;
    }
    a.part_g[(long long)blockIdx.y * a.cols + c] = g;
    a.part_b[(long long)blockIdx.y * a.cols + c] = b;
}

// -------------------------------------------------------------------- host --

constexpr int kWarpCols = 1024;       // a warp takes a row up to this length,
constexpr int kFwdBlockCols = 32768;  // a block up to these (1024 threads x 32, 1024 x 8)
constexpr int kBwdBlockCols = 8192;

// Threads of a block that share a row of `cols`, at e times 8 elements each.
int block_threads(int cols, int e) { return (int)round_up((cols + 8 * e - 1) / (8 * e), 32); }

// Blocks of the backward: each leaves a partial sum.
int bwd_blocks(long long rows, int cols)
{
    const int per = cols <= kWarpCols ? 8 : 1;
    const long long want = (rows + per - 1) / per, most = 2ll * device_sm_count();
    return (int)(want < most ? want : most);
}

bool rows16(const void* p, long long ld, int dt)
{
    return !p || ((reinterpret_cast<uintptr_t>(p) | (uintptr_t)(ld * (dt == SADMM_BF16 ? 2 : 4))) & 15) == 0;
}

template <typename X, typename Y, bool VEC>
sadmm_status fwd(const FwdArgs& a, cudaStream_t s)
{
    cudaError_t e;
    if (a.cols <= kWarpCols) {
        const dim3 grid((unsigned)((a.rows + 7) / 8)), block(256);
        if (a.cols <= 256)
            e = launch_pdl(k_ln_fwd<X, Y, VEC, false, 1>, grid, block, 0, s, a);
        else if (a.cols <= 512)
            e = launch_pdl(k_ln_fwd<X, Y, VEC, false, 2>, grid, block, 0, s, a);
        else
            e = launch_pdl(k_ln_fwd<X, Y, VEC, false, 4>, grid, block, 0, s, a);
    } else {
        const dim3 grid((unsigned)a.rows);
        if (a.cols <= 8192)
            e = launch_pdl(k_ln_fwd<X, Y, VEC, true, 1>, grid, dim3(block_threads(a.cols, 1)), 0, s, a);
        else if (a.cols <= 16384)
            e = launch_pdl(k_ln_fwd<X, Y, VEC, true, 2>, grid, dim3(block_threads(a.cols, 2)), 0, s, a);
        else if (a.cols <= kFwdBlockCols)
            e = launch_pdl(k_ln_fwd<X, Y, VEC, true, 4>, grid, dim3(block_threads(a.cols, 4)), 0, s, a);
        else
            e = launch_pdl(k_ln_fwd_long<X, Y>, grid, dim3(1024), 0, s, a);
    }
    return e == cudaSuccess ? SADMM_OK : SADMM_ECUDA;
}

template <typename X, typename Y, bool VEC>
sadmm_status bwd(const BwdArgs& a, cudaStream_t s)
{
    cudaError_t e;
    const dim3 grid((unsigned)bwd_blocks(a.rows, a.cols));
    if (a.cols <= 256)
        e = launch_pdl(k_ln_bwd<X, Y, VEC, false, 1>, grid, dim3(256), 0, s, a);
    else if (a.cols <= 512)
        e = launch_pdl(k_ln_bwd<X, Y, VEC, false, 2>, grid, dim3(256), 0, s, a);
    else if (a.cols <= kWarpCols)
        e = launch_pdl(k_ln_bwd<X, Y, VEC, false, 4>, grid, dim3(256), 0, s, a);
    else if (a.cols <= kBwdBlockCols)
        e = launch_pdl(k_ln_bwd<X, Y, VEC, true, 1>, grid, dim3(block_threads(a.cols, 1)), 0, s, a);
    else {
        e = cudaSuccess;
        if (a.dx) e = launch_pdl(k_ln_bwd_long<X, Y>, dim3((unsigned)a.rows), dim3(1024), 0, s, a);
        if (e == cudaSuccess && a.part_g)
            e = launch_pdl(k_ln_cols_long<X, Y>, dim3((unsigned)((a.cols + 255) / 256), grid.x), dim3(256), 0, s, a);
    }
    return e == cudaSuccess ? SADMM_OK : SADMM_ECUDA;
}

}  // namespace

size_t layernorm_bwd_bytes(const sadmm_layernorm_bwd_args& a)
{
    if (!a.dgamma && !a.dbeta) return 0;
    return 2 * (size_t)bwd_blocks(a.rows, a.cols) * (size_t)round_up(a.cols, 64) * 4;
}

sadmm_status launch_layernorm_fwd(const sadmm_layernorm_fwd_args& a, cudaStream_t s)
{
    if (a.rows == 0) return SADMM_OK;
    const FwdArgs f = {a.x, a.y, a.gamma, a.beta, a.mean, a.rstd, a.rows, a.ldx, a.ldy, a.cols, a.eps,
                       (float)a.cols};
    const bool vec = rows16(a.x, a.ldx, a.xdt) && rows16(a.y, a.ldy, a.ydt) && rows16(a.gamma, 0, SADMM_FP32) &&
                     rows16(a.beta, 0, SADMM_FP32);
    if (a.xdt == SADMM_BF16) {
        if (a.ydt == SADMM_BF16) return vec ? fwd<bf16, bf16, true>(f, s) : fwd<bf16, bf16, false>(f, s);
        return vec ? fwd<bf16, float, true>(f, s) : fwd<bf16, float, false>(f, s);
    }
    if (a.ydt == SADMM_BF16) return vec ? fwd<float, bf16, true>(f, s) : fwd<float, bf16, false>(f, s);
    return vec ? fwd<float, float, true>(f, s) : fwd<float, float, false>(f, s);
}

sadmm_status launch_layernorm_bwd(const sadmm_layernorm_bwd_args& a, void* ws, cudaStream_t s)
{
    const bool cols = a.dgamma || a.dbeta;
    if (a.rows == 0) {
        if (a.dgamma && cudaMemsetAsync(a.dgamma, 0, (size_t)a.cols * 4, s) != cudaSuccess) return SADMM_ECUDA;
        if (a.dbeta && cudaMemsetAsync(a.dbeta, 0, (size_t)a.cols * 4, s) != cudaSuccess) return SADMM_ECUDA;
        return SADMM_OK;
    }
    const int blocks = bwd_blocks(a.rows, a.cols);
    float* pg = cols ? static_cast<float*>(ws) : nullptr;
    float* pb = cols ? pg + (size_t)blocks * (size_t)round_up(a.cols, 64) : nullptr;
    const BwdArgs b = {a.x, a.dy, a.dres, a.dx, a.gamma, a.mean, a.rstd, pg, pb, a.rows, a.ldx, a.lddy, a.lddres,
                       a.lddx, a.cols, (float)a.cols};
    const bool vec = rows16(a.x, a.ldx, a.xdt) && rows16(a.dy, a.lddy, a.dydt) && rows16(a.dres, a.lddres, a.xdt) &&
                     rows16(a.dx, a.lddx, a.xdt) && rows16(a.gamma, 0, SADMM_FP32);
    sadmm_status st;
    if (a.xdt == SADMM_BF16) {
        if (a.dydt == SADMM_BF16)
            st = vec ? bwd<bf16, bf16, true>(b, s) : bwd<bf16, bf16, false>(b, s);
        else
            st = vec ? bwd<bf16, float, true>(b, s) : bwd<bf16, float, false>(b, s);
    } else if (a.dydt == SADMM_BF16) {
        st = vec ? bwd<float, bf16, true>(b, s) : bwd<float, bf16, false>(b, s);
    } else {
        st = vec ? bwd<float, float, true>(b, s) : bwd<float, float, false>(b, s);
    }
    if (st != SADMM_OK || !cols) return st;
    return launch_colsum(pg, pb, a.dgamma, a.dbeta, a.cols, blocks, s);
}

}  // namespace sadmm
