// rms.cu -- root-mean-square norm of rows, with the residual's addition before
// it and its output in 8 bits where wanted (the backward pass: norm.cu).
//
//   h = x + residual (rounded to the residual's type),  y = gamma h rstd,
//   rstd = (avg h^2 + eps)^-1/2
//
// Bound by memory.  A group of threads (a warp, or a block for long rows) takes a row at a
// time and keeps it in registers; sixteen lanes hold a block of 128 columns, so that its
// scale is a matter of four shuffles.  Measured: 16384 x 4096 bf16 with an fp32 residual into e4m3,
// sum and 1/rms kept, 116 us (109 of its 740 MB at the copy's 6.79 TB/s); 4 x 4096 6.9 us, a launch,
// a row's loads and its sum one after the other.  Both from fp32 into bf16, 161 us (138); 4096 x 16384
// of them 179: past 8192 columns a thread's 32 values of two fp32 matrices do not fit 64 registers (260 bytes spilled).
#include "q8.cuh"

namespace sadmm {
namespace {

SADMM_DEV float warp_sum(float v)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// The sum over a row's threads: a warp, or the block, whose warps' sums every
// thread adds up in the same order.  `slot` alternates between calls.
struct __align__(16) RowSums {
    float v[2][32];
};
template <bool BLOCK>
SADMM_DEV float row_sum(float v, RowSums& red, int slot)
{
    v = warp_sum(v);
    if (BLOCK) {
        const int n = blockDim.x >> 5;
        if ((threadIdx.x & 31) == 0) red.v[slot][threadIdx.x >> 5] = v;
        __syncthreads();
        v = 0.0f;
        for (int w = 0; w < n; w += 4) {  // the places past the last warp hold zeros
            const float4 q = *reinterpret_cast<const float4*>(&red.v[slot][w]);
            v += (q.x + q.y) + (q.z + q.w);
        }
    }
    return v;
}
SADMM_DEV void clear(RowSums& red)
{
    for (int i = threadIdx.x; i < 64; i += blockDim.x) (&red.v[0][0])[i] = 0.0f;
}

// The rounded root and quotient: rsqrtf may be two units off, once a row for every value of it
// (4 x 4096 and 16384 x 4096 take the same time with either).
SADMM_DEV float rstd_of(float sum, float n, float eps) { return 1.0f / sqrtf(sum / n + eps); }

SADMM_DEV float round_to(float v, int dt) { return dt == SADMM_BF16 ? __bfloat162float(__float2bfloat16_rn(v)) : v; }

// Row r of a matrix of bf16 or fp32 elements.
struct Rows {
    const void* p;
    long long ld, rows;
    int dt, cols;
    int aligned;  // rows start on 16-byte boundaries
    template <int ES>
    SADMM_DEV const uint8_t* at(long long r, int c) const
    {
        return static_cast<const uint8_t*>(p) + (r * ld + c) * ES;
    }
    // Columns c .. c+7 of row r, in two steps.
    template <int ES, bool AL>
    SADMM_DEV void ask(long long r, int c, const Span& m, Raw8<ES, AL>& raw, int* status) const
    {
        const bool in = r < rows && c < cols && dbg_in(r, rows, status) && dbg_in(c, cols, status);
        ask8(at<ES>(in ? r : 0, in ? c : 0), in, aligned, m, raw);
    }
    template <int ES, bool AL>
    SADMM_DEV void take(long long r, int c, const Span& m, const Raw8<ES, AL>& raw, float (&v)[8]) const
    {
        take8(at<ES>(r, c), cols - c, aligned, m, raw, v);
    }
    SADMM_DEV int size() const { return dt == SADMM_BF16 ? 2 : 4; }
    SADMM_DEV Span span() const
    {
        const uint8_t* b = static_cast<const uint8_t*>(p);
        return {b, b + ((rows - 1) * ld + cols) * size()};
    }
    SADMM_DEV void load(long long r, int c, const Span& m, float (&v)[8], int* status) const
    {
        const int n = min(8, cols - c);
        if (n <= 0 || !dbg_in(r, rows, status) || !dbg_run(c, n, cols, status)) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = 0.0f;
            return;
        }
        load8(static_cast<const uint8_t*>(p) + (r * ld + c) * size(), dt, n, m, v);
    }
    SADMM_DEV void store(long long r, int c, const float (&v)[8], int* status) const
    {
        const int n = min(8, cols - c);
        if (n <= 0 || !dbg_in(r, rows, status) || !dbg_run(c, n, cols, status)) return;
        store8(const_cast<uint8_t*>(static_cast<const uint8_t*>(p)) + (r * ld + c) * size(), dt, n, v);
    }
};

struct FwdArgs {
    Rows x, res, h, y;    // p NULL: not there
    sadmm_q8_out y8;
    const float* gamma;
    float* rstd;
    long long rows;
    int cols;
    float eps, n;
    int* status;
};

// Columns c .. c+7 of row r: the value of h that the norm reads.
SADMM_DEV void load_h(const FwdArgs& a, long long r, int c, const Span& mx, const Span& mr, float (&v)[8])
{
    a.x.load(r, c, mx, v, a.status);
    if (a.res.p) {
        float e[8];
        a.res.load(r, c, mr, e, a.status);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = round_to(v[j] + e[j], a.res.dt);
    }
}

// Columns c .. c+7 of y; in 8 bits the 16 lanes of a block share its scale (all
// 32 lanes of the warp call it).
SADMM_DEV void finish8(const FwdArgs& a, long long r, int c, float rstd, float (&v)[8])
{
    if (a.gamma) {
        const int n = min(8, a.cols - c);
        const bool whole = n == 8 && (reinterpret_cast<uintptr_t>(a.gamma) & 15) == 0;
        if (whole && dbg_run(c, 8, a.cols, a.status)) {
            const float4 p = *reinterpret_cast<const float4*>(a.gamma + c), q = *reinterpret_cast<const float4*>(a.gamma + c + 4);
            const float g[8] = {p.x, p.y, p.z, p.w, q.x, q.y, q.z, q.w};
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = v[j] * rstd * g[j];
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = j < n ? v[j] * rstd * a.gamma[c + j] : 0.0f;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] *= rstd;
    }
    if (!a.y8.q) {
        a.y.store(r, c, v, a.status);
        return;
    }
    const Q8Scale k = q8_scale(max16(q8_top(v)));
    if (c >= a.cols || !dbg_in(c, a.cols, a.status) || !dbg_in(r, a.rows, a.status)) return;
    if ((threadIdx.x & 15) == 0) a.y8.s[r * a.y8.s_row + c / kQBlock * a.y8.s_block] = k.s;
    store_bytes8(static_cast<uint8_t*>(a.y8.q) + r * a.y8.ld + c, a.cols - c, q8_four(v[0], v[1], v[2], v[3], k),
                 q8_four(v[4], v[5], v[6], v[7], k));
}

// A row over a group of threads, a warp or a block, E times 8 neighbours each, kept in
// registers between the sum and the output; the next row's words are asked for
// before this one's are added up.  XS, RS: bytes of an element of x and of the
// residual (RS 0: none); AL: rows start on 16-byte boundaries.
template <int XS, int RS, bool BLOCK, int E, bool AL>
__global__ void __launch_bounds__(!BLOCK ? 256 : E == 4 ? 1024 : 512, !BLOCK ? 3 : E == 4 ? 1 : 2) k_rms_fwd(const FwdArgs a)
{
    constexpr int RW = RS ? RS : 2;
    constexpr bool AHEAD = E < 4;  // (four times eight: no registers for the next row)
    __shared__ RowSums red;
    const int G = BLOCK ? blockDim.x : 32, t = BLOCK ? threadIdx.x : threadIdx.x & 31;
    const long long step = (long long)gridDim.x * (BLOCK ? 1 : 8);
    long long r = BLOCK ? (long long)blockIdx.x : (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (BLOCK) {
        clear(red);
        __syncthreads();
    }
    pdl_wait();
    pdl_trigger();
    const Span mx = a.x.span(), mr = RS ? a.res.span() : mx;
    Raw8<XS, AL> nx[E];
    Raw8<RW, AL> nr[RS ? E : 1];
    auto ask = [&](long long row) {
#pragma unroll
        for (int k = 0; k < E; ++k) {
            a.x.ask(row, (k * G + t) * 8, mx, nx[k], a.status);
            if (RS) a.res.ask(row, (k * G + t) * 8, mr, nr[RS ? k : 0], a.status);
        }
    };
    if (AHEAD) ask(r);
    int slot = 0;
    for (; r < a.rows; r += step) {
        if (!AHEAD) ask(r);
        float v[E][8], sum = 0.0f;
#pragma unroll
        for (int k = 0; k < E; ++k) {
            const int c = (k * G + t) * 8;
            a.x.take(r, c, mx, nx[k], v[k]);
            if (RS) {
                float e[8];
                a.res.take(r, c, mr, nr[RS ? k : 0], e);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[k][j] = RS == 2 ? round_to(v[k][j] + e[j], SADMM_BF16) : v[k][j] + e[j];
            }
        }
        if (AHEAD) ask(r + step);
#pragma unroll
        for (int k = 0; k < E; ++k) {
            if (RS && a.h.p) a.h.store(r, (k * G + t) * 8, v[k], a.status);
            float p = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) p += v[k][j] * v[k][j];
            sum += p;
        }
        const float rstd = rstd_of(row_sum<BLOCK>(sum, red, slot), a.n, a.eps);
        slot ^= 1;
        if (t == 0 && a.rstd) a.rstd[r] = rstd;
#pragma unroll
        for (int k = 0; k < E; ++k) finish8(a, r, (k * G + t) * 8, rstd, v[k]);
    }
}

// Rows of any length: a block a row, read twice (the sum from h where it is written,
// which may be the residual's own place).
__global__ void __launch_bounds__(1024) k_rms_fwd_long(const FwdArgs a)
{
    __shared__ RowSums red;
    clear(red);
    __syncthreads();
    pdl_wait();
    pdl_trigger();
    const long long r = blockIdx.x;
    const Span mx = a.x.span(), mr = a.res.p ? a.res.span() : mx, mh = a.h.p ? a.h.span() : mx;
    float sum = 0.0f;
    for (int c = threadIdx.x * 8; c < a.cols; c += 8192) {
        float v[8];
        load_h(a, r, c, mx, mr, v);
        if (a.h.p) a.h.store(r, c, v, a.status);
        float p = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) p += v[j] * v[j];
        sum += p;
    }
    const float rstd = rstd_of(row_sum<true>(sum, red, 0), a.n, a.eps);
    if (threadIdx.x == 0 && a.rstd) a.rstd[r] = rstd;
    const int end = (a.cols + 255) & ~255;  // a whole warp's columns
    for (int c = threadIdx.x * 8; c < end; c += 8192) {
        float v[8];
        if (a.h.p)
            a.h.load(r, c, mh, v, a.status);
        else
            load_h(a, r, c, mx, mr, v);
        finish8(a, r, c, rstd, v);
    }
}

// -------------------------------------------------------------------- host --

constexpr int kWarpCols = 512;          // up to here a warp takes a row
constexpr int kFwdCols = 32768;         // up to here a row stays in registers (1024 threads of 32)

int row_threads(int cols, int e) { return (int)round_up((cols + 8 * e - 1) / (8 * e), 32); }

// Blocks of n threads of 64 registers an SM holds.
int per_sm(int n) { return n > 512 ? 1 : 1024 / n < 8 ? 1024 / n : 8; }

Rows rows_of(const void* p, long long ld, int dt, long long rows, int cols)
{
    const long long es = dt == SADMM_BF16 ? 2 : 4;
    return {p, ld, rows, dt, cols, ((reinterpret_cast<uintptr_t>(p) | (uintptr_t)(ld * es)) & 15) == 0};
}

template <int XS, int RS, bool AL, bool BLOCK, int E>
cudaError_t fwd(const FwdArgs& a, cudaStream_t s)
{
    const int threads = BLOCK ? row_threads(a.cols, E) : 256;
    const long long want = BLOCK ? a.rows : (a.rows + 7) / 8, most = (long long)per_sm(threads) * device_sm_count();
    return launch_pdl(k_rms_fwd<XS, RS, BLOCK, E, AL>, dim3((unsigned)(want < most ? want : most)), dim3(threads), 0, s, a);
}

template <int XS, int RS, bool AL>
cudaError_t fwd(const FwdArgs& a, cudaStream_t s)
{
    if (a.cols <= 256) return fwd<XS, RS, AL, false, 1>(a, s);
    if (a.cols <= kWarpCols) return fwd<XS, RS, AL, false, 2>(a, s);
    if (a.cols <= 8192) return fwd<XS, RS, AL, true, 2>(a, s);
    return fwd<XS, RS, AL, true, 4>(a, s);
}

template <int XS, int RS>
cudaError_t fwd(const FwdArgs& a, cudaStream_t s)
{
    return a.x.aligned && (!RS || a.res.aligned) ? fwd<XS, RS, true>(a, s) : fwd<XS, RS, false>(a, s);
}

}  // namespace

sadmm_status launch_rmsnorm_fwd(const sadmm_rmsnorm_fwd_args& a, cudaStream_t s)
{
    if (a.rows == 0) return SADMM_OK;
    FwdArgs f = {};
    f.x = rows_of(a.x, a.ldx, a.xdt, a.rows, a.cols);
    f.res = rows_of(a.residual, a.ldr, a.rdt, a.rows, a.cols);
    f.h = rows_of(a.h, a.ldh, a.rdt, a.rows, a.cols);
    f.y = rows_of(a.y, a.ldy, a.ydt, a.rows, a.cols);
    if (a.ydt == SADMM_E4M3) f.y8 = a.y8;
    f.gamma = a.gamma;
    f.rstd = a.rstd;
    f.rows = a.rows;
    f.cols = a.cols;
    f.eps = a.eps;
    f.n = (float)a.cols;
    f.status = device_status_ptr();
    const int xs = a.xdt == SADMM_BF16 ? 2 : 4, rs = !a.residual ? 0 : a.rdt == SADMM_BF16 ? 2 : 4;
    cudaError_t err;
    if (a.cols > kFwdCols)
        err = launch_pdl(k_rms_fwd_long, dim3((unsigned)a.rows), dim3(1024), 0, s, f);
    else if (xs == 2)
        err = rs == 0 ? fwd<2, 0>(f, s) : rs == 2 ? fwd<2, 2>(f, s) : fwd<2, 4>(f, s);
    else
        err = rs == 0 ? fwd<4, 0>(f, s) : rs == 2 ? fwd<4, 2>(f, s) : fwd<4, 4>(f, s);
    return err == cudaSuccess ? SADMM_OK : SADMM_ECUDA;
}

}  // namespace sadmm
