// few.cu -- the feed-forward products of one to sixteen tokens (of small weights
// to 32): y = act(x W^T + b) + residual and h = act(x Wg^T + bg) * (x Wu^T + bu).
//
// Bound by the weights, which are read once, and on small layers by latency: the
// tile kernels start and join pipelines, these have none.  In k_few a warp
// multiplies 16 weight rows (gated: 16 of either) by all tokens with the
// warp-level MMA, whose operands come straight from global memory: lane (g, t) =
// (lane / 4, lane % 4) reads 16 bytes of rows g and g + 8 and of token g, elements
// 8t .. 8t+7 of 32.  The MMA wants other elements in that lane's place, but the
// same for both operands, and a sum does not mind the order of its terms.
// Nothing is staged.  Warps that share rows join their sums in shared memory in
// warp order.  Rows that do not start on 16-byte boundaries are read as the
// aligned words around them, shifted into place.  k_one is for one token of
// ragged rows.
//
// Measured against the tile kernels (us, the same call repeated in a graph, so that
// weights below the L2's size stay there): 1 token 5120 -> 2048 4.7 (9.1), 8192 ->
// 8192 17 to 20 (26.6); 8 tokens 5.1 (9.7), 18.9 (27.0), the gated pair 2048 -> 2
// x 5464 8.0 (10.6); 16 tokens 5.9 (9.8), 23.7 (27.3), 9.7 (10.9); 17 tokens 7.9 (9.7),
// 30.4 (26.6), 13.9 (11.1).
#include <string.h>

#include "act.cuh"
#include "common.cuh"
#include "internal.h"
#include "output.cuh"

namespace sadmm {
namespace {

using bf16 = __nv_bfloat16;

constexpr int kFewWarps = 8;
constexpr int kLongRuns = 64;  // pieces of 32 elements until two accumulators have 1024 terms each

struct FewArgs {
    const bf16* x;
    const bf16* w[2];
    long long ldx, ldw[2];
    const float* bias[2];
    Out y, res, z, u;
    int tokens, n_in, n_out;
    int share;  // warps that share a group's rows: 1, 2, 4 or 8
    int act;
    int* status;
};

SADMM_DEV uint4 ld_stream(const uint4* p)
{
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "l"(p));
    return v;
}

// Elements c .. c+7 of a row of n, c a multiple of 8: `off` is the row's place in its
// first 16-byte word.  Whole words of the row that hold them all, or not `inside`.
SADMM_DEV int place(const bf16* row) { return (int)((reinterpret_cast<uintptr_t>(row) & 15) >> 1); }
SADMM_DEV bool inside(int off, int c, int n) { return c >= off && c + (off ? 16 : 8) <= n; }

SADMM_DEV uint4 ld_if(const bf16* p, bool on)  // zeros and no access where it is off
{
    uint4 v;
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.s32 p, %5, 0;\n\tmov.b32 %0, 0;\n\tmov.b32 %1, 0;\n\tmov.b32 %2, 0;\n\t"
        "mov.b32 %3, 0;\n\t@p ld.global.nc.v4.u32 {%0, %1, %2, %3}, [%4];\n\t}"
        : "=&r"(v.x), "=&r"(v.y), "=&r"(v.z), "=&r"(v.w)
        : "l"(p), "r"((int)on));
    return v;
}

struct Words {
    uint4 lo, hi;
};

template <bool ALIGNED>
SADMM_DEV void fetch(Words& v, const bf16* row, int c, int n, int* status)
{
    const int off = ALIGNED ? 0 : place(row);
    const bool in = inside(off, c, n) && dbg_run(c - off, off ? 16 : 8, n, status);
    v.lo = ld_if(row + c - off, in);
    if constexpr (!ALIGNED) v.hi = ld_if(row + c - off + 8, in && off);
}

// The fetched elements in place; those at the row's two ends one by one, zeros past it.
template <bool ALIGNED>
SADMM_DEV uint4 settle(const Words& v, const bf16* row, int c, int n)
{
    const int off = ALIGNED ? 0 : place(row);
    if (!inside(off, c, n)) {
        const unsigned short* e = reinterpret_cast<const unsigned short*>(row) + c;
        uint32_t x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = c + j < n ? __ldg(e + j) : 0u;
        return make_uint4(x[0] | x[1] << 16, x[2] | x[3] << 16, x[4] | x[5] << 16, x[6] | x[7] << 16);
    }
    if constexpr (ALIGNED) return v.lo;
    const bool two = off & 4, one = off & 2;
    const int sh = (off & 1) * 16;
    const uint32_t a0 = two ? v.lo.z : v.lo.x, a1 = two ? v.lo.w : v.lo.y, a2 = two ? v.hi.x : v.lo.z;
    const uint32_t a3 = two ? v.hi.y : v.lo.w, a4 = two ? v.hi.z : v.hi.x, a5 = two ? v.hi.w : v.hi.y;
    const uint32_t b0 = one ? a1 : a0, b1 = one ? a2 : a1, b2 = one ? a3 : a2, b3 = one ? a4 : a3, b4 = one ? a5 : a4;
    return make_uint4(__funnelshift_r(b0, b1, sh), __funnelshift_r(b1, b2, sh), __funnelshift_r(b2, b3, sh),
                      __funnelshift_r(b3, b4, sh));
}

// One output of one token: bias, activation, gate, residual.
template <bool GATED>
SADMM_DEV void finish(const FewArgs& a, int t, int n, float g, float u)
{
    if (a.bias[0]) g += a.bias[0][n];
    if (GATED) {
        if (a.bias[1]) u += a.bias[1][n];
        if (a.u.p) store1(a.u, t, n, u, a.status);
    }
    if (a.z.p) store1(a.z, t, n, g, a.status);
    with_act(a.act, [&](auto tag) { g = act_f32<decltype(tag)::value>(g); });
    if (GATED) g *= u;
    if (a.res.p) g += load1(a.res, t, n, a.status);
    store1(a.y, t, n, g, a.status);
}

// Two fp32 values in one 64-bit register, from two bf16.
SADMM_DEV unsigned long long pair_of(uint32_t w)
{
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(w << 16), "r"(w & 0xffff0000u));
    return r;
}
SADMM_DEV void fma2(unsigned long long& d, unsigned long long a, unsigned long long b)
{
    asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(d) : "l"(a), "l"(b));
}
SADMM_DEV float sum_of(unsigned long long v)
{
    uint32_t a, b;
    asm("mov.b64 {%0, %1}, %2;" : "=r"(a), "=r"(b) : "l"(v));
    return __uint_as_float(a) + __uint_as_float(b);
}

// Joins the lanes' N values: after the exchange over distance O a lane holds half
// as many, those its bit O selects (`index` is their first one's number).
template <int O, int N, int V>
SADMM_DEV void join(float (&v)[V], int lane, int& index)
{
    if constexpr (O > 0) {
        if constexpr (N > 1) {
            const bool hi = (lane & O) != 0;
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                const float keep = hi ? v[i + N / 2] : v[i], give = hi ? v[i] : v[i + N / 2];
                v[i] = keep + __shfl_xor_sync(0xffffffffu, give, O);
            }
            if (hi) index += N / 2;
            join<O / 2, N / 2>(v, lane, index);
        } else {
            v[0] += __shfl_xor_sync(0xffffffffu, v[0], O);
            join<O / 2, 1>(v, lane, index);
        }
    }
}

// One token on the CUDA cores, where rows are ragged or (not the gated pair's) off
// 16-byte boundaries.  A group of warps takes U outputs (gated: of two weight rows
// each); a lane multiplies its 16-byte pieces in pairs (fma.f32x2, fp32 sums).  Here
// and by k_few, over weights from DRAM: 1001 -> 1001 3.4 and 3.7 us, 5119 -> 2047 10.1
// and 12.0; the gated pair of 5000 -> 2 x 1500, aligned, 7.2 and 12.0; off 16-byte
// boundaries, where k_few serves it, 333 -> 2 x 777 5.7 and 3.7, 1023 -> 2 x 2731 8.1
// and 6.5, 2047 -> 2 x 5461 20.5 and 20.8.
template <int U, bool GATED, bool ALIGNED>
__global__ void __launch_bounds__(kFewWarps * 32, 2) k_one(const __grid_constant__ FewArgs a)
{
    constexpr int R = GATED ? 2 * U : U;  // weight rows
    __shared__ float red[kFewWarps][R];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int part = warp % a.share, group = warp / a.share;
    const int n0 = (blockIdx.x * (kFewWarps / a.share) + group) * U;
    const int first = (part * 32 + lane) * 8, step = a.share * 256;
    const bf16* row[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int n = min(n0 + r % U, a.n_out - 1);  // past the end: the last row again, not stored
        row[r] = a.w[r / U] + (long long)n * a.ldw[r / U];
    }
    // the weights on their way to L2 (where every write lands) while the kernel before still runs
    for (int c = first * 8; c < a.n_in; c += step * 8) {
#pragma unroll
        for (int r = 0; r < R; ++r) asm volatile("prefetch.global.L2 [%0];" ::"l"(row[r] + c));
    }
    pdl_wait();
    pdl_trigger();
    unsigned long long acc[R];
#pragma unroll
    for (int r = 0; r < R; ++r) acc[r] = 0;
    auto multiply = [&](const uint4 (&w)[R], const uint4& x) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const unsigned long long xp = pair_of(j == 0 ? x.x : j == 1 ? x.y : j == 2 ? x.z : x.w);
#pragma unroll
            for (int r = 0; r < R; ++r)
                fma2(acc[r], pair_of(j == 0 ? w[r].x : j == 1 ? w[r].y : j == 2 ? w[r].z : w[r].w), xp);
        }
    };
    int c = first;
    if constexpr (ALIGNED) {
#pragma unroll 2
        for (; c + 8 <= a.n_in; c += step) {
            uint4 w[R];
            if (!dbg_run(c, 8, a.n_in, a.status)) break;
#pragma unroll
            for (int r = 0; r < R; ++r) w[r] = ld_stream(reinterpret_cast<const uint4*>(row[r] + c));
            multiply(w, __ldg(reinterpret_cast<const uint4*>(a.x + c)));
        }
    }
#pragma unroll 1
    for (; c < a.n_in; c += step) {
        Words w[R], x;
#pragma unroll
        for (int r = 0; r < R; ++r) fetch<ALIGNED>(w[r], row[r], c, a.n_in, a.status);
        fetch<ALIGNED>(x, a.x, c, a.n_in, a.status);
        uint4 v[R];
#pragma unroll
        for (int r = 0; r < R; ++r) v[r] = settle<ALIGNED>(w[r], row[r], c, a.n_in);
        multiply(v, settle<ALIGNED>(x, a.x, c, a.n_in));
    }
    float v[R];
#pragma unroll
    for (int r = 0; r < R; ++r) v[r] = sum_of(acc[r]);
    int index = 0;
    join<16, R>(v, lane, index);
    if ((lane & (32 / R - 1)) == 0) red[warp][index] = v[0];
    __syncthreads();
    const int who = threadIdx.x / U, o = threadIdx.x % U;  // group and output of the CTA
    const int n = (blockIdx.x * (kFewWarps / a.share) + who) * U + o;
    if (who < kFewWarps / a.share && n < a.n_out) {
        float g = 0.0f, u = 0.0f;
        for (int p = who * a.share; p < (who + 1) * a.share; ++p) {
            g += red[p][o];
            if (GATED) u += red[p][R - U + o];
        }
        finish<GATED>(a, 0, n, g, u);
    }
}

// D (+)= A B, 16 rows x 8 tokens x 16 contraction elements, one warp.
SADMM_DEV void mma_16x8(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// NT times 8 tokens at most.  fp32 sums alternate between two accumulators.  LONG:
// these join the warp's sum in shared memory after 1024 terms each, because a sum
// inside the MMAs loses about 1e-9 of itself per term.  For long fp32 outputs alone:
// a bf16 one does not show it, and the loop is some 5 % slower with the joins in it.
template <int NT, bool GATED, bool ALIGNED, bool LONG>
__global__ void __launch_bounds__(kFewWarps * 32, 2) k_few(const __grid_constant__ FewArgs a)
{
    constexpr int M = GATED ? 2 : 1;  // weight matrices
    // pieces of 32 elements in flight (8 tokens of 8192 -> 8192: 18.8 us with 8, 24.0 with 4; the gated pair, more
    // tokens and rows off 16-byte boundaries have no registers for as many: 16 tokens 23.6 with 4, 24.4 with 8; with 8,
    // 4 and 2 unaligned, over weights from DRAM, 2 tokens of 333 -> 777 5.9, 3.6, 2.9, of 1001 -> 1001 6.3, 3.7, 4.2, of
    // 5119 -> 2047 15.8, 12.1, 13.5, of 8191 -> 8191 58, 50, 48)
    constexpr int kAhead = NT == 4 || GATED ? 2 : NT == 2 || !ALIGNED ? 4 : 8;
    __shared__ float red[kFewWarps][M][16][8 * NT + 1];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int part = warp % a.share, group = warp / a.share, groups = kFewWarps / a.share;
    const int n0 = (blockIdx.x * groups + group) * 16;
    const bf16* row[M][2];
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
        for (int h = 0; h < 2; ++h)  // past the end: the last row again, not stored
            row[m][h] = a.w[m] + (long long)min(n0 + g + 8 * h, a.n_out - 1) * a.ldw[m];
    // the weights on their way to L2 while the kernel before still runs
    for (int c = (part * 4 + t) * 64; c < a.n_in; c += a.share * 256) {
#pragma unroll
        for (int m = 0; m < M; ++m) {
            asm volatile("prefetch.global.L2 [%0];" ::"l"(row[m][0] + c));
            asm volatile("prefetch.global.L2 [%0];" ::"l"(row[m][1] + c));
        }
    }
    pdl_wait();
    pdl_trigger();
    const bf16* xr[NT];
#pragma unroll
    for (int q = 0; q < NT; ++q) xr[q] = a.x + min(g + 8 * q, a.tokens - 1) * a.ldx;
    float d[2][M][NT][4];
#pragma unroll
    for (int i = 0; i < 2 * M * NT * 4; ++i) (&d[0][0][0][0])[i] = 0.0f;
    auto multiply = [&](int which, const uint4 (&w)[M][2], const uint4 (&x)[NT]) {
#pragma unroll
        for (int m = 0; m < M; ++m)
#pragma unroll
            for (int q = 0; q < NT; ++q) {
                mma_16x8(d[which][m][q], w[m][0].x, w[m][1].x, w[m][0].y, w[m][1].y, x[q].x, x[q].y);
                mma_16x8(d[which][m][q], w[m][0].z, w[m][1].z, w[m][0].w, w[m][1].w, x[q].z, x[q].w);
            }
    };
    // lane (g, t) holds rows g, g + 8 and tokens 2t, 2t + 1 (of each eight)
    bool begun = false;  // whether the warp's sum has
    auto join_sums = [&]() {
#pragma unroll
        for (int m = 0; m < M; ++m)
#pragma unroll
            for (int q = 0; q < NT; ++q)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float& sum = red[warp][m][g + (j >> 1) * 8][8 * q + 2 * t + (j & 1)];
                    const float v = d[0][m][q][j] + d[1][m][q][j];
                    sum = LONG && begun ? sum + v : v;
                    d[0][m][q][j] = d[1][m][q][j] = 0.0f;
                }
        begun = true;
    };
    int runs = 0;  // since they were joined
    auto count_run = [&]() {
        if (!LONG || runs++ < kLongRuns / kAhead) return;
        join_sums();
        runs = 1;
    };
    // a warp takes runs of 32 kAhead elements, `share` warps in turn
    const int step = a.share * 32 * kAhead;
    int c = part * 32 * kAhead;
    if constexpr (ALIGNED) {
#pragma unroll (LONG ? 1 : 2)
        for (; c + 32 * kAhead <= a.n_in; c += step) {
            count_run();
            uint4 w[kAhead][M][2], x[kAhead][NT];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                int k = c + 32 * i + 8 * t;
                if (!dbg_run(k, 8, a.n_in, a.status)) k = 0;  // the row's start instead
#pragma unroll
                for (int m = 0; m < M; ++m) {
                    w[i][m][0] = ld_stream(reinterpret_cast<const uint4*>(row[m][0] + k));
                    w[i][m][1] = ld_stream(reinterpret_cast<const uint4*>(row[m][1] + k));
                }
#pragma unroll
                for (int q = 0; q < NT; ++q) x[i][q] = __ldg(reinterpret_cast<const uint4*>(xr[q] + k));
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) multiply(i & 1, w[i], x[i]);
        }
    }
    // the ragged end, and rows off 16-byte boundaries: again all loads before their products (the inner loop has one
    // turn; without it the compiler lays the same code out worse: the gated pair of 333 -> 2 x 777 3.7 us, 4.8)
#pragma unroll 1
    for (; c < a.n_in; c += step) {
        count_run();
#pragma unroll 1
        for (int i0 = 0; i0 < kAhead && c + 32 * i0 < a.n_in; i0 += kAhead) {
            Words w[kAhead][M][2], x[kAhead][NT];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int k = c + 32 * (i0 + i) + 8 * t;
#pragma unroll
                for (int m = 0; m < M; ++m) {
                    fetch<ALIGNED>(w[i][m][0], row[m][0], k, a.n_in, a.status);
                    fetch<ALIGNED>(w[i][m][1], row[m][1], k, a.n_in, a.status);
                }
#pragma unroll
                for (int q = 0; q < NT; ++q) fetch<ALIGNED>(x[i][q], xr[q], k, a.n_in, a.status);
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int k = c + 32 * (i0 + i) + 8 * t;
                if (c + 32 * (i0 + i) >= a.n_in) break;  // the whole warp
                uint4 v[M][2], u[NT];
#pragma unroll
                for (int m = 0; m < M; ++m) {
                    v[m][0] = settle<ALIGNED>(w[i][m][0], row[m][0], k, a.n_in);
                    v[m][1] = settle<ALIGNED>(w[i][m][1], row[m][1], k, a.n_in);
                }
#pragma unroll
                for (int q = 0; q < NT; ++q) u[q] = settle<ALIGNED>(x[i][q], xr[q], k, a.n_in);
                __syncwarp();
                multiply(i & 1, v, u);
            }
        }
    }
    join_sums();
    __syncthreads();
    // consecutive threads take consecutive outputs of a token
    for (int i = threadIdx.x; i < groups * 16 * a.tokens; i += kFewWarps * 32) {
        const int o = i % (groups * 16), tok = i / (groups * 16), who = o >> 4;
        const int n = blockIdx.x * groups * 16 + o;
        if (n >= a.n_out) continue;
        float v = 0.0f, u = 0.0f;
        for (int p = who * a.share; p < (who + 1) * a.share; ++p) {
            v += red[p][0][o & 15][tok];
            if (GATED) u += red[p][M - 1][o & 15][tok];
        }
        finish<GATED>(a, tok, n, v, u);
    }
}

template <int U, bool GATED>
sadmm_status run_one(FewArgs& a, bool aligned, cudaStream_t s)
{
    // as many warps a group as have four pieces of its rows each (K 8192, N 8192, one token: 18.8 us with eight warps
    // a group, 25.2 with two; the gated pair of K 2048, N 5464: 9.4 with eight, 6.6 with one), more where the groups
    // are too few to give an SM 16 warps
    const long long groups = (a.n_out + U - 1) / U;
    a.share = 1;
    while (a.share < kFewWarps && (a.n_in >= 2048 * a.share || groups * a.share < 16ll * device_sm_count())) a.share *= 2;
    const int per = kFewWarps / a.share;
    void (*kernel)(FewArgs) = k_one<U, GATED, true>;
    if constexpr (!GATED) {
        if (!aligned) kernel = k_one<U, GATED, false>;
    }
    return launch_pdl(kernel, dim3((unsigned)((groups + per - 1) / per)), dim3(kFewWarps * 32), 0, s, a) == cudaSuccess
               ? SADMM_OK
               : SADMM_ECUDA;
}

template <int NT, bool GATED>
sadmm_status run(FewArgs& a, bool aligned, cudaStream_t s)
{
    // as few warps a group as give the device 8 an SM (8 tokens of 2048 -> 2 x 5464: 8.1 us, 10.1 with 16, 10.9 with 4)
    const long long groups = (a.n_out + 15) / 16;
    a.share = 1;
    while (a.share < kFewWarps && groups * a.share < 8ll * device_sm_count()) a.share *= 2;
    const int per = kFewWarps / a.share;
    void (*kernel)(FewArgs) = k_few<NT, GATED, true, false>;
    if constexpr (NT == 1) {
        if (!aligned) kernel = k_few<NT, GATED, false, false>;
    }
    if constexpr (!GATED) {
        if (!a.y.bf16 && a.n_in > 32 * kLongRuns * a.share) {
            kernel = k_few<NT, GATED, true, true>;
            if constexpr (NT == 1) {
                if (!aligned) kernel = k_few<NT, GATED, false, true>;
            }
        }
    }
    return launch_pdl(kernel, dim3((unsigned)((groups + per - 1) / per)), dim3(kFewWarps * 32), 0, s, a) == cudaSuccess
               ? SADMM_OK
               : SADMM_ECUDA;
}

}  // namespace

static bool few_aligned(const sadmm_linear_fwd_args& a) { return tg_aligned(a.x, a.ldx) && tg_aligned(a.w, a.ldw); }
static bool few_aligned(const sadmm_gated_fwd_args& a)
{
    return tg_aligned(a.x, a.ldx) && tg_aligned(a.wg, a.ldwg) && tg_aligned(a.wu, a.ldwu);
}

// Up to 16 tokens, of small weights 32; where rows are off 16-byte boundaries 8 (the
// gated pair 2047 -> 2 x 5461: 8 tokens 17.9 us here, 26.2 by tiles after copying; 16
// tokens 39.1 and 26.5).
bool few_linear(const sadmm_linear_fwd_args& a)
{
    const bool small = (long long)a.n_in * a.n_out <= 1ll << 24;
    return a.tokens <= 8 || (a.tokens <= (small ? 32 : 16) && few_aligned(a));
}
bool few_gated(const sadmm_gated_fwd_args& a) { return a.tokens <= 8 || (a.tokens <= 16 && few_aligned(a)); }

sadmm_status launch_few_linear(const sadmm_linear_fwd_args& f, cudaStream_t s)
{
    FewArgs a;
    memset(&a, 0, sizeof(a));
    a.x = static_cast<const bf16*>(f.x);
    a.w[0] = static_cast<const bf16*>(f.w);
    a.ldx = f.ldx;
    a.ldw[0] = f.ldw;
    a.bias[0] = f.bias;
    a.y = make_out({f.y, f.ldy, f.ydt}, f.tokens, f.n_out);
    if (f.residual) a.res = make_out({const_cast<void*>(f.residual), f.ldr, f.ydt}, f.tokens, f.n_out);
    if (f.z) a.z = make_out({f.z, f.ldz, SADMM_BF16}, f.tokens, f.n_out);
    a.tokens = (int)f.tokens;
    a.n_in = f.n_in;
    a.n_out = f.n_out;
    a.act = f.act;
    a.status = device_status_ptr();
    const bool aligned = few_aligned(f);
    if (f.tokens == 1 && (!aligned || f.n_in % 256)) return run_one<4, false>(a, aligned, s);
    return f.tokens <= 8 ? run<1, false>(a, aligned, s) : f.tokens <= 16 ? run<2, false>(a, aligned, s) : run<4, false>(a, aligned, s);
}

sadmm_status launch_few_gated(const sadmm_gated_fwd_args& f, cudaStream_t s)
{
    FewArgs a;
    memset(&a, 0, sizeof(a));
    a.x = static_cast<const bf16*>(f.x);
    a.w[0] = static_cast<const bf16*>(f.wg);
    a.w[1] = static_cast<const bf16*>(f.wu);
    a.ldx = f.ldx;
    a.ldw[0] = f.ldwg;
    a.ldw[1] = f.ldwu;
    a.bias[0] = f.bg;
    a.bias[1] = f.bu;
    a.y = make_out({f.h, f.ldh, SADMM_BF16}, f.tokens, f.n_hidden);
    if (f.g) a.z = make_out({f.g, f.ldg, SADMM_BF16}, f.tokens, f.n_hidden);
    if (f.u) a.u = make_out({f.u, f.ldu, SADMM_BF16}, f.tokens, f.n_hidden);
    a.tokens = (int)f.tokens;
    a.n_in = f.n_in;
    a.n_out = f.n_hidden;
    a.act = f.act;
    a.status = device_status_ptr();
    const bool aligned = few_aligned(f);
    // one token of short rows goes to k_few where its groups of 16 units are more than the SMs (333 -> 2 x 5461 4.4 us and
    // by k_one 5.4, 1023 -> 2 x 2731 4.7 and 5.3; below 2432 units or from 2000 columns on k_one is the faster or level:
    // 2047 -> 2 x 2300 5.3 and 7.4, -> 2 x 4001 8.0 and 7.7, 5000 -> 2 x 5461 23.7 and 28.3)
    const bool one = f.n_hidden <= 16 * device_sm_count() || f.n_in >= 2000;
    if (f.tokens == 1 && aligned && f.n_in % 256 && one) return run_one<2, true>(a, aligned, s);
    return f.tokens <= 8 ? run<1, true>(a, aligned, s) : run<2, true>(a, aligned, s);
}

}  // namespace sadmm
