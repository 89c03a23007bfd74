// q8.cuh -- 8-bit matrices (e4m3 values, an fp32 scale for each block of 128):
// what their kernels share, and the host interface of the products.
#pragma once

#include <cuda_fp8.h>

#include "common.cuh"
#include "internal.h"
#include "output.cuh"
#include "tgemm.cuh"

namespace sadmm {

constexpr int kQBlock = 128;

// ------------------------------------------------------------------- host --

// One 8-bit operand of a product: `rows` rows of the output's row (or column)
// index, each `k` long; aligned for the tensor-memory accelerator.
struct Q8Operand {
    const void* p;
    long long rows, k, ld;
    const float* s;
    long long s_row, s_block;
    int shift;             // rows of a scale: 1 << shift
};

// C = A B^T in one of tgemm.cuh's modes.  kTgGated with y8.q: y in 8 bits.
struct Q8Problem {
    int mode;
    Q8Operand a[2], b[2];
    long long m, n;
    const float* bias;
    const float* bias2;
    int act;
    TgMatrix y, residual, z, u;
    sadmm_q8_out y8;
};

inline bool q8_aligned(const void* p, long long ld)
{
    return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && (ld & 15) == 0;
}

// One tile a CTA (q8gemm.cu), or one or two products by CTA pairs (q8pair.cu), and the times
// they are expected to take.
sadmm_status launch_q8_product(const Q8Problem& t, cudaStream_t s);
long long time_q8_product(const Q8Problem& t);
sadmm_status launch_q8_pair(const Q8Problem* t, int count, cudaStream_t s);
long long time_q8_pair(const Q8Problem& t);
// The most rows (of all columns), and the most columns (of all rows), that the pairs have done one round of
// tiles earlier, in whole tiles; 0: there is but one round.
void q8_pair_less(const Q8Problem& t, long long& rows, long long& cols);

// Matrices in 8 bits (quant.cu).  What is made 8-bit: x; dy act'(z) (z given); or
// the gated pair's dg and du (u given), whose outputs are [0] and [1].  sums: column
// sums of the values, or NULL.
struct Q8Source {
    const void* x;
    long long ldx;
    int xdt;
    const void* z;
    long long ldz;
    const void* u;
    long long ldu;
    int act;
    long long rows, cols;
    int tile;
    sadmm_q8_out out[2], out_t[2];
    float* sums[2];
};
size_t q8_source_bytes(const Q8Source& a);  // scratch of the column sums
sadmm_status launch_q8_source(const Q8Source& a, void* ws, cudaStream_t s);

// ----------------------------------------------------------------- device --

#ifdef __CUDACC__

// A block's scale s from its largest magnitude, and the quotients x / s of the block
// as fp32 divisions round them, zeros with their signs.  With s = d 2^e, 1 <= d < 2, and
// y = -x 2^-e: q = y (-r) with r = 1 / d and one correction, q + (q d + y)(-r), which gives the
// nearest number where r is the nearest to 1 / d (Markstein, 1990, theorem 8) and the rest
// q d + y is exact, as it is here for every q from 2^-80 on (without 2^-e its last digits are lost
// below s = 2^-92).  A zero's rest is +0, whatever its sign, and (+0)(-r) leaves either
// zero as it is.  An infinite x gives NaN.  A tenth of a division's time a value (1 / d is
// taken once a block).
struct Q8Scale {
    float s, d, m, r;  // the scale; d, -2^-e and -1 / d
};
constexpr float kE4m3Max = 448.0f;
SADMM_DEV Q8Scale q8_scale_of(float s, float r)
{
    const uint32_t bits = __float_as_uint(s);
    return {s, __uint_as_float((bits & 0x007fffffu) | 0x3f800000u),
            __uint_as_float((0x7f000000u - (bits & 0x7f800000u)) | 0x80000000u), r};
}
SADMM_DEV Q8Scale q8_scale(float top)
{
    constexpr float r = 1.0f / kE4m3Max;
    top = fmaxf(top, 1.2621774483536189e-29f /* 2^-96 */);
    const float q = __fmul_rn(top, r), s = __fmaf_rn(__fmaf_rn(-q, kE4m3Max, top), r, q);
    Q8Scale k = q8_scale_of(s, 0.0f);
    k.r = -__frcp_rn(k.d);
    return k;
}
// Two at a time, in half the instructions.
SADMM_DEV void q8_quotients(float& a, float& b, const Q8Scale& k)
{
    asm("{\n\t"
        ".reg .b64 y, q, e, d, m, r;\n\t"
        "mov.b64 y, {%0, %1};\n\t"
        "mov.b64 d, {%2, %2};\n\t"
        "mov.b64 m, {%3, %3};\n\t"
        "mov.b64 r, {%4, %4};\n\t"
        "mul.rn.f32x2 y, y, m;\n\t"
        "mul.rn.f32x2 q, y, r;\n\t"
        "fma.rn.f32x2 e, q, d, y;\n\t"
        "fma.rn.f32x2 q, e, r, q;\n\t"
        "mov.b64 {%0, %1}, q;\n\t"
        "}"
        : "+f"(a), "+f"(b)
        : "f"(k.d), "f"(k.m), "f"(k.r));
}
// The largest finite magnitude of N values (0: none), of which infinities become NaN, as
// which they end anyway: the largest passes over a NaN by itself.
template <int N>
SADMM_DEV float q8_top(float (&v)[N])
{
    float t = 0.0f;
#pragma unroll
    for (int j = 0; j < N; ++j) t = fmaxf(t, fabsf(v[j]));
    if (t == __int_as_float(0x7f800000)) {
        t = 0.0f;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            if (fabsf(v[j]) == __int_as_float(0x7f800000)) v[j] = __int_as_float(0x7fffffff);
            t = fmaxf(t, fabsf(v[j]));
        }
    }
    return t;
}
SADMM_DEV uint32_t q8_two(float lo, float hi)
{
    return __nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3);
}
SADMM_DEV uint32_t q8_four(float a, float b, float c, float d) { return q8_two(a, b) | q8_two(c, d) << 16; }
// The same of four quotients.
SADMM_DEV uint32_t q8_four(float a, float b, float c, float d, const Q8Scale& k)
{
    q8_quotients(a, b, k);
    q8_quotients(c, d, k);
    return q8_four(a, b, c, d);
}

// The largest of v over groups of 16 lanes.
SADMM_DEV float max16(float v)
{
#pragma unroll
    for (int o = 8; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}

// The scales of N rows (2 or 4) from their lanes' largest, over groups of 16 lanes: a lane goes on with
// one of the rows, so that a scale's arithmetic is done once.
template <int N>
SADMM_DEV void scales16(const float (&top)[N], Q8Scale (&k)[N])
{
    static_assert(N == 2 || N == 4, "rows of a group");
    const bool a = threadIdx.x & 8, b = threadIdx.x & 4;
    float v[N / 2];
#pragma unroll
    for (int j = 0; j < N / 2; ++j)
        v[j] = fmaxf(a ? top[2 * j + 1] : top[2 * j], __shfl_xor_sync(0xffffffffu, a ? top[2 * j] : top[2 * j + 1], 8));
    float t = v[0];
    if (N == 4)
        t = fmaxf(b ? v[N / 2 - 1] : v[0], __shfl_xor_sync(0xffffffffu, b ? v[0] : v[N / 2 - 1], 4));
    else
        t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 4));
#pragma unroll
    for (int o = 2; o; o >>= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, o));
    const Q8Scale own = q8_scale(t);
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int from = (j & 1) * 8 + (j >> 1) * 4;
        k[j] = q8_scale_of(__shfl_sync(0xffffffffu, own.s, from, 16), __shfl_sync(0xffffffffu, own.r, from, 16));
    }
}

// A matrix as bytes: it starts at lo and ends at hi.
struct Span {
    const uint8_t *lo, *hi;
};

// The 16 bytes at p.  Off a 16-byte boundary they come from the two aligned words that
// hold them, where these lie inside the matrix; else the `n` wanted ones one by
// one, zeros after them.
SADMM_DEV uint4 load16(const uint8_t* p, int n, const Span& m)
{
    const int off = (int)(reinterpret_cast<uintptr_t>(p) & 15);
    const uint8_t* w = p - off;
    if (off == 0 && p >= m.lo && p + 16 <= m.hi) return *reinterpret_cast<const uint4*>(p);
    if (w >= m.lo && w + 32 <= m.hi) {
        const uint4 a = *reinterpret_cast<const uint4*>(w), b = *reinterpret_cast<const uint4*>(w + 16);
        uint32_t v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
        if (off & 4) {
#pragma unroll
            for (int i = 0; i < 6; ++i) v[i] = v[i + 1];
            v[6] = b.w;
        }
        if (off & 8) {
#pragma unroll
            for (int i = 0; i < 5; ++i) v[i] = v[i + 2];
        }
        const int sh = (off & 3) * 8;
        return make_uint4(__funnelshift_r(v[0], v[1], sh), __funnelshift_r(v[1], v[2], sh),
                          __funnelshift_r(v[2], v[3], sh), __funnelshift_r(v[3], v[4], sh));
    }
    uint32_t v[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (i < n && p + i >= m.lo && p + i < m.hi) v[i >> 2] |= (uint32_t)p[i] << (8 * (i & 3));
    return make_uint4(v[0], v[1], v[2], v[3]);
}

// The 16-byte words that hold eight neighbours of ES bytes each: all of a group's are
// asked for before the first is used.
// AL: the matrix's rows start on 16-byte boundaries; else whether they do is said at run time.
template <int ES, bool AL = false>
struct Raw8 {
    static constexpr int n = ES / 2 + !AL;
    uint4 w[n];           // the last one off 16-byte boundaries only
    bool apart;           // not inside the matrix: to be read one by one
};
// `in`: at least one of the eight at p is wanted; aligned: p is on a 16-byte boundary (the same for the whole matrix).
template <int ES, bool AL>
SADMM_DEV void ask8(const uint8_t* p, bool in, bool aligned, const Span& m, Raw8<ES, AL>& r)
{
    aligned = AL || aligned;
    const uint8_t* b = AL ? p : p - (reinterpret_cast<uintptr_t>(p) & 15);
    const bool ok = in && (AL || b >= m.lo) && b + (ES / 2 + !aligned) * 16 <= m.hi;
    r.apart = in && !ok;
#pragma unroll
    for (int k = 0; k < r.n; ++k) {
        r.w[k] = make_uint4(0, 0, 0, 0);
        if (ok && (k < ES / 2 || !aligned)) r.w[k] = *reinterpret_cast<const uint4*>(b + 16 * k);
    }
}
SADMM_DEV void load8(const void* p, int dt, int n, const Span& m, float (&v)[8]);
// Their values, zeros after the n-th.
template <int ES, bool AL>
SADMM_DEV void take8(const uint8_t* p, int n, bool aligned, const Span& m, const Raw8<ES, AL>& r, float (&v)[8])
{
    if (r.apart) {
        load8(p, ES == 2 ? SADMM_BF16 : SADMM_FP32, n, m, v);
        return;
    }
    constexpr int W = 2 * ES;  // 32-bit words of the eight
    uint32_t w[W + 4];
#pragma unroll
    for (int k = 0; k < r.n; ++k) w[4 * k] = r.w[k].x, w[4 * k + 1] = r.w[k].y, w[4 * k + 2] = r.w[k].z, w[4 * k + 3] = r.w[k].w;
    if (!AL && !aligned) {
        const int off = (int)(reinterpret_cast<uintptr_t>(p) & 15);
        if (off & 4) {
#pragma unroll
            for (int i = 0; i < W + 3; ++i) w[i] = w[i + 1];
        }
        if (off & 8) {
#pragma unroll
            for (int i = 0; i < W + 2; ++i) w[i] = w[i + 2];
        }
        if (ES == 2 && (off & 2)) {
#pragma unroll
            for (int i = 0; i < W; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 16);
        }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float x = ES == 4 ? __uint_as_float(w[ES == 4 ? j : 0])
                                : __uint_as_float((j & 1) ? w[j / 2] & 0xffff0000u : w[j / 2] << 16);
        v[j] = x;
    }
    if (n < 8) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j >= n) v[j] = 0.0f;
    }
}

// Eight neighbours of a bf16 (dt SADMM_BF16) or fp32 matrix at element p, `n` of
// them wanted (at least one); zeros after those.
SADMM_DEV void load8(const void* p, int dt, int n, const Span& m, float (&v)[8])
{
    const uint8_t* b = static_cast<const uint8_t*>(p);
    if (dt == SADMM_BF16) {
        const uint4 q = load16(b, 2 * n, m);
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[2 * j] = __uint_as_float(w[j] << 16);
            v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
        }
    } else {
        const uint4 lo = load16(b, 4 * n, m);
        const uint4 hi = n > 4 ? load16(b + 16, 4 * n - 16, m) : make_uint4(0, 0, 0, 0);
        v[0] = __uint_as_float(lo.x); v[1] = __uint_as_float(lo.y);
        v[2] = __uint_as_float(lo.z); v[3] = __uint_as_float(lo.w);
        v[4] = __uint_as_float(hi.x); v[5] = __uint_as_float(hi.y);
        v[6] = __uint_as_float(hi.z); v[7] = __uint_as_float(hi.w);
    }
    if (n < 8) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j >= n) v[j] = 0.0f;
    }
}

// Eight neighbours to element p, of which n are inside the row.
SADMM_DEV void store8(void* p, int dt, int n, const float (&v)[8])
{
    if (dt == SADMM_BF16) {
        __nv_bfloat16* o = static_cast<__nv_bfloat16*>(p);
        if (n >= 8 && (reinterpret_cast<uintptr_t>(p) & 15) == 0) {
            uint32_t w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
                w[j] = *reinterpret_cast<const uint32_t*>(&h);
            }
            *reinterpret_cast<uint4*>(o) = make_uint4(w[0], w[1], w[2], w[3]);
            return;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) o[j] = __float2bfloat16_rn(v[j]);
    } else {
        float* o = static_cast<float*>(p);
        if (n >= 8 && (reinterpret_cast<uintptr_t>(p) & 15) == 0) {
            reinterpret_cast<float4*>(o)[0] = make_float4(v[0], v[1], v[2], v[3]);
            reinterpret_cast<float4*>(o)[1] = make_float4(v[4], v[5], v[6], v[7]);
            return;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) o[j] = v[j];
    }
}

// Eight bytes to p, of which n are inside the row.
SADMM_DEV void store_bytes8(uint8_t* p, int n, uint32_t lo, uint32_t hi)
{
    if (n >= 8 && (reinterpret_cast<uintptr_t>(p) & 7) == 0) {
        *reinterpret_cast<uint2*>(p) = make_uint2(lo, hi);
        return;
    }
    if (n >= 8 && (reinterpret_cast<uintptr_t>(p) & 3) == 0) {
        reinterpret_cast<uint32_t*>(p)[0] = lo;
        reinterpret_cast<uint32_t*>(p)[1] = hi;
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < n) p[j] = (uint8_t)((j < 4 ? lo : hi) >> (8 * (j & 3)));
}

#endif

}  // namespace sadmm
