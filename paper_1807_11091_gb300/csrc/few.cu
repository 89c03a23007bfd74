// few.cu -- the feed-forward products of one to four tokens: y = act(x W^T + b)
// + residual and h = act(x Wg^T + bg) * (x Wu^T + bu), on the CUDA cores.
//
// Bound by the weights, which are read once, and on small layers by latency: the
// tensor-core kernels spend 5 us on their pipeline's start and join, so this
// one has none.  A CTA takes a few outputs (rows of the weights); each of its
// eight warps reads every eighth 512-byte piece of those rows, a lane 16 bytes,
// with the tokens' matching pieces of x from L1, and multiplies them in pairs
// (fma.f32x2, fp32 sums).  The lanes' sums are joined by a butterfly that halves
// the values with each exchange, the warps' in shared memory in warp order.
// Rows that do not start on 16-byte boundaries are read as the aligned words
// around them, shifted into place.
#include <string.h>

#include "act.cuh"
#include "common.cuh"
#include "internal.h"
#include "output.cuh"

namespace sadmm {
namespace {

using bf16 = __nv_bfloat16;

constexpr int kFewWarps = 8;

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

// Elements c .. c+7 of a row of n (zeros past its end), c a multiple of 8.
SADMM_DEV uint4 piece(const bf16* row, int c, int n)
{
    const int off = (int)((reinterpret_cast<uintptr_t>(row) & 15) >> 1);  // the row's place in its first 16-byte word
    if (off == 0 && c + 8 <= n) return __ldg(reinterpret_cast<const uint4*>(row + c));
    if (off && c >= off && c + 16 <= n) {
        const uint4* p = reinterpret_cast<const uint4*>(row + c - off);
        const uint4 lo = __ldg(p), hi = __ldg(p + 1);
        const int sh = (off & 1) * 16;
        uint32_t v0, v1, v2, v3, v4;
        switch (off >> 1) {
        case 0: v0 = lo.x; v1 = lo.y; v2 = lo.z; v3 = lo.w; v4 = hi.x; break;
        case 1: v0 = lo.y; v1 = lo.z; v2 = lo.w; v3 = hi.x; v4 = hi.y; break;
        case 2: v0 = lo.z; v1 = lo.w; v2 = hi.x; v3 = hi.y; v4 = hi.z; break;
        default: v0 = lo.w; v1 = hi.x; v2 = hi.y; v3 = hi.z; v4 = hi.w; break;
        }
        return make_uint4(__funnelshift_r(v0, v1, sh), __funnelshift_r(v1, v2, sh), __funnelshift_r(v2, v3, sh),
                          __funnelshift_r(v3, v4, sh));
    }
    const unsigned short* e = reinterpret_cast<const unsigned short*>(row) + c;
    uint32_t v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = c + j < n ? __ldg(e + j) : 0u;
    return make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
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

// U outputs a CTA (gated: of two weight rows each), T tokens at most.
template <int T, int U, bool GATED, bool ALIGNED>
__global__ void __launch_bounds__(kFewWarps * 32, 2) k_few(const __grid_constant__ FewArgs a)
{
    constexpr int R = GATED ? 2 * U : U;  // weight rows
    constexpr int V = R * T;              // sums of a lane, a power of two up to 32
    __shared__ float red[kFewWarps][V];
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
    unsigned long long acc[R][T];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int t = 0; t < T; ++t) acc[r][t] = 0;
    auto multiply = [&](const uint4 (&w)[R], const uint4 (&x)[T]) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            unsigned long long wp[R];
#pragma unroll
            for (int r = 0; r < R; ++r) wp[r] = pair_of(j == 0 ? w[r].x : j == 1 ? w[r].y : j == 2 ? w[r].z : w[r].w);
#pragma unroll
            for (int t = 0; t < T; ++t) {
                const unsigned long long xp = pair_of(j == 0 ? x[t].x : j == 1 ? x[t].y : j == 2 ? x[t].z : x[t].w);
#pragma unroll
                for (int r = 0; r < R; ++r) fma2(acc[r][t], wp[r], xp);
            }
        }
    };
    int c = first;
    if constexpr (ALIGNED) {
        const bf16* xr[T];
#pragma unroll
        for (int t = 0; t < T; ++t) xr[t] = a.x + min(t, a.tokens - 1) * a.ldx;  // past the end: the last again, not stored
#pragma unroll(R * T <= 8 ? 2 : 1)
        for (; c + 8 <= a.n_in; c += step) {
            uint4 w[R], x[T];
#pragma unroll
            for (int r = 0; r < R; ++r) w[r] = ld_stream(reinterpret_cast<const uint4*>(row[r] + c));
#pragma unroll
            for (int t = 0; t < T; ++t) x[t] = __ldg(reinterpret_cast<const uint4*>(xr[t] + c));
            multiply(w, x);
        }
    }
#pragma unroll 1
    for (; c < a.n_in; c += step) {
        uint4 w[R], x[T];
#pragma unroll
        for (int r = 0; r < R; ++r) w[r] = piece(row[r], c, a.n_in);
#pragma unroll
        for (int t = 0; t < T; ++t) x[t] = piece(a.x + min(t, a.tokens - 1) * a.ldx, c, a.n_in);
        multiply(w, x);
    }
    float v[V];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int t = 0; t < T; ++t) v[r * T + t] = sum_of(acc[r][t]);
    int index = 0;
    join<16, V>(v, lane, index);
    if ((lane & (32 / V - 1)) == 0) red[warp][index] = v[0];
    __syncthreads();
    const int who = threadIdx.x / (U * T), i = threadIdx.x % (U * T);  // group and output of the CTA
    if (who < kFewWarps / a.share) {
        const int t = i / U, o = i % U, n = (blockIdx.x * (kFewWarps / a.share) + who) * U + o;
        float g = 0.0f, u = 0.0f;
        for (int p = who * a.share; p < (who + 1) * a.share; ++p) {
            g += red[p][o * T + t];
            if (GATED) u += red[p][(U + o) * T + t];
        }
        if (t < a.tokens && n < a.n_out) {
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
    }
}

template <int T, int U, bool GATED>
sadmm_status run(FewArgs& a, cudaStream_t s)
{
    const bool aligned = tg_aligned(a.x, a.ldx) && tg_aligned(a.w[0], a.ldw[0]) && (!GATED || tg_aligned(a.w[1], a.ldw[1]));
    // as many warps a group as have four pieces of its rows each (K 8192, N 8192, one token: 18.8 us with eight warps
    // a group, 25.2 with two; the gated pair of K 2048, N 5464: 9.4 with eight, 6.6 with one), more where the groups
    // are too few to give an SM 16 warps
    const long long groups = (a.n_out + U - 1) / U;
    a.share = 1;
    while (a.share < kFewWarps && (a.n_in >= 2048 * a.share || groups * a.share < 16ll * device_sm_count())) a.share *= 2;
    const int per = kFewWarps / a.share;
    return launch_pdl(aligned ? k_few<T, U, GATED, true> : k_few<T, U, GATED, false>,
                      dim3((unsigned)((groups + per - 1) / per)), dim3(kFewWarps * 32), 0, s, a) == cudaSuccess
               ? SADMM_OK
               : SADMM_ECUDA;
}

}  // namespace

// One token, or up to four on weights of at most 2^24 elements: 2 and 4 tokens of
// 5120 -> 2048 take 5.6 and 6.5 us here and 8.0 on the tensor cores, of 8192 ->
// 8192 25.5 and 29.2 and 23.4 there (one token 19.1 and 23.0).
bool few(long long tokens, long long weights) { return tokens == 1 || (tokens <= 4 && weights <= 1ll << 24); }
bool few_linear(const sadmm_linear_fwd_args& a) { return few(a.tokens, (long long)a.n_in * a.n_out); }
bool few_gated(const sadmm_gated_fwd_args& a) { return few(a.tokens, 2ll * a.n_in * a.n_hidden); }

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
    if (f.tokens == 1) return run<1, 4, false>(a, s);
    if (f.tokens == 2) return run<2, 4, false>(a, s);
    return run<4, 4, false>(a, s);
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
    if (f.tokens == 1) return run<1, 2, true>(a, s);
    if (f.tokens == 2) return run<2, 2, true>(a, s);
    return run<4, 2, true>(a, s);
}

}  // namespace sadmm
