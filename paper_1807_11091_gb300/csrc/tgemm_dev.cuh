// tgemm_dev.cuh -- device parts shared by the feed-forward products' kernels
// (tgemm.cu, tgemm_pair.cu): operand loads and descriptors, the cluster
// primitives, and the epilogue that finishes an operator's output.
#pragma once

#include <cuda.h>
#include <cudaTypedefs.h>
#include <string.h>

#include "act.cuh"
#include "common.cuh"
#include "output.cuh"
#include "internal.h"
#include "tgemm.cuh"

namespace sadmm {

PFN_cuTensorMapEncodeTiled_v12000 get_encode_fn();  // pack.cu

namespace {

constexpr int kBox = 8192;        // one 64 x 64 bf16 box
constexpr int kPTile = 2 * kBox;  // 128 rows x 64
constexpr int kTgProducts = 3;    // products of a launch, at most
// and their tensor maps: a gated pair's gradients have four for the sum of dx, and two for either weights' gradient,
// which share x's only where x is the Q side (tiles not swapped)
constexpr int kTgMaps = 8;

// fp32 outputs of long contractions (LONG) are added up over accumulators of
// kLongSteps steps each, in registers, because a sum inside the tensor cores loses
// digits as it grows longer (relative error of weight gradients: 0.24e-6 over 256
// terms, 0.48e-6 over 512, 1.0e-6 over 1024, 2.1e-6 over 2048).
constexpr int kLongSteps = 12;  // 768 contraction elements

// One product of a launch.  The P side is the tile's 128-row side: the output's
// rows, or its columns where the tiles are swapped.
struct TgProduct {
    Out y;
    long long m, n;            // output rows, columns
    int first;                 // its first tile
    int p_tiles, q_tiles;
    int nk0, nk;               // 64-element contraction steps: of the first summand, of all
    int steps;                 // steps of each CTA of a cluster (tgemm.cu)
    int acc_steps;             // steps that an accumulator holds before it is added to the sums in registers
    int pm, qm;                // maps; the second summand's (gated: the second weights') follow
    int p_kmajor, q_kmajor;
    uint32_t idesc;
};

struct TgMaps {
    CUtensorMap map[kTgMaps];
};

struct TgArgs {
    TgProduct prod[kTgProducts];
    int products;
    int tiles;                 // of all products
    Out res, z, u;             // epilogue of a single product
    const float* bias;
    const float* bias2;
    int act;
    int bn;                    // rows of the Q side per tile (tgemm.cu: per half when gated)
    int splits;                // CTAs per cluster (tgemm.cu)
    int stages;
    uint32_t stage_bytes, q_off;
    uint32_t acc_cols, tmem_cols;
    int long_tiles, catch_up, shift;  // the pairs' schedule (tgemm_pair.cu)
    int* status;
};

// ------------------------------------------------------------- device PTX --

// Shared-memory matrix descriptor of a row-contiguous (MN-major) operand held
// as 64-row boxes of 64 contraction elements with the 128-byte swizzle: within
// a box one contraction element is a 128-byte line of 64 rows, groups of 8
// lines are 1024 bytes apart (stride offset), boxes of the next 64 rows follow
// 8192 bytes on (leading offset).  16 contraction elements are 2048 bytes.
SADMM_DEV uint64_t sdesc_mnmajor_sw128(uint32_t saddr)
{
    uint64_t d = 0;
    d |= (uint64_t)((saddr & 0x3FFFFu) >> 4);
    d |= (uint64_t)(8192u >> 4) << 16;
    d |= (uint64_t)(1024u >> 4) << 32;
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}

SADMM_DEV uint64_t sdesc(uint32_t saddr, int kmajor)
{
    return kmajor ? sdesc_kmajor_sw128(saddr) : sdesc_mnmajor_sw128(saddr);
}

// ---------------------------------------------------------------- epilogue --

SADMM_DEV void st_v8(void* p, const uint32_t (&w)[8])
{
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]),
                 "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                 : "memory");
}

SADMM_DEV uint32_t pack_bf16(float lo, float hi)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// v[0..15] to row r, columns c .. c+15 of o; columns at or past n are skipped.
SADMM_DEV void store16(const Out& o, long long r, long long c, long long n, const float (&v)[16], int* status)
{
    const long long at = r * o.ld + c;
    if (c + 16 <= n && o.vec && dbg_in(at, o.total, status) && dbg_in(at + 15, o.total, status)) {
        if (o.bf16) {
            __nv_bfloat16* p = static_cast<__nv_bfloat16*>(o.p) + at;
            uint32_t w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = pack_bf16(v[2 * j], v[2 * j + 1]);
            if (o.vec == 2) {
                st_v8(p, w);
            } else {
                reinterpret_cast<uint4*>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
                reinterpret_cast<uint4*>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
            }
        } else {
            float* p = static_cast<float*>(o.p) + at;
            if (o.vec == 2) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t w[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) w[j] = __float_as_uint(v[8 * h + j]);
                    st_v8(p + 8 * h, w);
                }
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    reinterpret_cast<float4*>(p)[j] = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
            }
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        if (c + j >= n || !dbg_in(at + j, o.total, status)) continue;
        if (o.bf16)
            static_cast<__nv_bfloat16*>(o.p)[at + j] = __float2bfloat16_rn(v[j]);
        else
            static_cast<float*>(o.p)[at + j] = v[j];
    }
}

// v += row r, columns c .. c+15 of o.
SADMM_DEV void add16(const Out& o, long long r, long long c, long long n, float (&v)[16], int* status)
{
    const long long at = r * o.ld + c;
    if (c + 16 <= n && o.vec && dbg_in(at, o.total, status) && dbg_in(at + 15, o.total, status)) {
        if (o.bf16) {
            const uint4* p = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(o.p) + at);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint4 q = p[h];
                const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    v[8 * h + 2 * j] += __uint_as_float(w[j] << 16);
                    v[8 * h + 2 * j + 1] += __uint_as_float(w[j] & 0xffff0000u);
                }
            }
        } else {
            const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(o.p) + at);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float4 q = p[j];
                v[4 * j] += q.x; v[4 * j + 1] += q.y; v[4 * j + 2] += q.z; v[4 * j + 3] += q.w;
            }
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        if (c + j >= n || !dbg_in(at + j, o.total, status)) continue;
        v[j] += o.bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(o.p)[at + j])
                       : static_cast<const float*>(o.p)[at + j];
    }
}

// The same for N neighbouring columns, 2 or 4 (c a multiple of N).
template <int N>
SADMM_DEV void store_n(const Out& o, long long r, long long c, long long n, const float (&v)[N], int* status)
{
    const long long at = r * o.ld + c;
    if (c + N <= n && o.vec && dbg_in(at, o.total, status) && dbg_in(at + N - 1, o.total, status)) {
        if (o.bf16) {
            uint32_t w[N / 2];
#pragma unroll
            for (int j = 0; j < N / 2; ++j) w[j] = pack_bf16(v[2 * j], v[2 * j + 1]);
            __nv_bfloat16* p = static_cast<__nv_bfloat16*>(o.p) + at;
            if constexpr (N == 4)
                *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
            else
                *reinterpret_cast<uint32_t*>(p) = w[0];
        } else {
            float* p = static_cast<float*>(o.p) + at;
            if constexpr (N == 4)
                *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
            else
                *reinterpret_cast<float2*>(p) = make_float2(v[0], v[1]);
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
        if (c + j >= n || !dbg_in(at + j, o.total, status)) continue;
        if (o.bf16)
            static_cast<__nv_bfloat16*>(o.p)[at + j] = __float2bfloat16_rn(v[j]);
        else
            static_cast<float*>(o.p)[at + j] = v[j];
    }
}

// N neighbouring columns of o, zero at or past n.
template <int N>
SADMM_DEV void load_n(const Out& o, long long r, long long c, long long n, float (&v)[N], int* status)
{
    const long long at = r * o.ld + c;
    if (c + N <= n && o.vec && dbg_in(at, o.total, status) && dbg_in(at + N - 1, o.total, status)) {
        if (o.bf16) {
            const __nv_bfloat162* p = reinterpret_cast<const __nv_bfloat162*>(static_cast<const __nv_bfloat16*>(o.p) + at);
            uint32_t w[N / 2];
            if constexpr (N == 4) {
                const uint2 q = *reinterpret_cast<const uint2*>(p);
                w[0] = q.x;
                w[N / 2 - 1] = q.y;
            } else {
                w[0] = *reinterpret_cast<const uint32_t*>(p);
            }
#pragma unroll
            for (int j = 0; j < N / 2; ++j) {
                v[2 * j] = __uint_as_float(w[j] << 16);
                v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
            }
        } else {
            const float* p = static_cast<const float*>(o.p) + at;
            if constexpr (N == 4) {
                const float4 q = *reinterpret_cast<const float4*>(p);
                v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
            } else {
                const float2 q = *reinterpret_cast<const float2*>(p);
                v[0] = q.x; v[1] = q.y;
            }
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
        v[j] = 0.0f;
        if (c + j >= n || !dbg_in(at + j, o.total, status)) continue;
        v[j] = o.bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(o.p)[at + j])
                      : static_cast<const float*>(o.p)[at + j];
    }
}

// Sixteen columns of one output row: sb / sb2 are their biases in shared memory.
template <bool GATED>
SADMM_DEV void finish16(const TgArgs& a, const TgProduct& p, long long r, long long c, float (&v)[16], float (&w)[16],
                        const float* sb, const float* sb2)
{
    if (a.bias) {
#pragma unroll
        for (int j = 0; j < 16; j += 4) {
            const float4 b = *reinterpret_cast<const float4*>(sb + j);
            v[j] += b.x; v[j + 1] += b.y; v[j + 2] += b.z; v[j + 3] += b.w;
        }
    }
    if (GATED) {
        if (a.bias2) {
#pragma unroll
            for (int j = 0; j < 16; j += 4) {
                const float4 b = *reinterpret_cast<const float4*>(sb2 + j);
                w[j] += b.x; w[j + 1] += b.y; w[j + 2] += b.z; w[j + 3] += b.w;
            }
        }
        if (a.u.p) store16(a.u, r, c, p.n, w, a.status);
    }
    if (a.z.p) store16(a.z, r, c, p.n, v, a.status);
    with_act(a.act, [&](auto tag) {
        constexpr int A = decltype(tag)::value;
#pragma unroll
        for (int j = 0; j < 16; ++j) v[j] = act_f32<A>(v[j]);
    });
    if (GATED) {
#pragma unroll
        for (int j = 0; j < 16; ++j) v[j] *= w[j];
    }
    if (a.res.p) add16(a.res, r, c, p.n, v, a.status);
    store16(p.y, r, c, p.n, v, a.status);
}

// N neighbouring columns; b and b2 are their biases, e their residual.
template <bool GATED, int N>
SADMM_DEV void finish_n(const TgArgs& a, const TgProduct& p, long long r, long long c, float (&v)[N], float (&w)[N],
                        const float (&b)[N], const float (&b2)[N], const float (&e)[N])
{
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] += b[j];
    if (GATED) {
#pragma unroll
        for (int j = 0; j < N; ++j) w[j] += b2[j];
        if (a.u.p) store_n<N>(a.u, r, c, p.n, w, a.status);
    }
    if (a.z.p) store_n<N>(a.z, r, c, p.n, v, a.status);
    with_act(a.act, [&](auto tag) {
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = act_f32<decltype(tag)::value>(v[j]);
    });
#pragma unroll
    for (int j = 0; j < N; ++j) {
        if (GATED) v[j] *= w[j];
        if (a.res.p) v[j] += e[j];
    }
    store_n<N>(p.y, r, c, p.n, v, a.status);
}

// One operand's part of a stage: `rows` rows from row0, 64 contraction elements from k0.
SADMM_DEV void load_part(uint8_t* dst, const CUtensorMap* map, uint64_t* bar, int kmajor, int rows, int row0, int k0)
{
    if (kmajor) {
        tma_load_2d(dst, map, bar, k0, row0);
    } else {
        for (int j = 0; j * 64 < rows; ++j) tma_load_2d(dst + j * kBox, map, bar, row0 + 64 * j, k0);
    }
}

// -------------------------------------------------------------------- host --

// Steps of 64 contraction elements.
long long steps_of(const TgProblem& t) { return (t.a[0].k + 63) / 64 * (t.mode == kTgSum ? 2 : 1); }

bool encode(CUtensorMap* map, const TgOperand& o, int rows_per_tile)
{
    PFN_cuTensorMapEncodeTiled_v12000 enc = get_encode_fn();
    if (!enc) return false;
    memset(map, 0, sizeof(*map));
    const cuuint64_t gdim[2] = {(cuuint64_t)(o.kmajor ? o.k : o.rows), (cuuint64_t)(o.kmajor ? o.rows : o.k)};
    const cuuint64_t gstride[1] = {(cuuint64_t)o.ld * 2};
    const cuuint32_t box[2] = {64u, o.kmajor ? (cuuint32_t)rows_per_tile : 64u};
    const cuuint32_t estride[2] = {1u, 1u};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(o.p), gdim, gstride, box, estride,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// What the kernels' arguments have in common: the products' outputs, and the
// epilogue of the first (the others have none).
void fill_common(TgArgs& a, const TgProblem* t, int count)
{
    memset(&a, 0, sizeof(a));
    a.products = count;
    for (int i = 0; i < count; ++i) {
        a.prod[i].m = t[i].m;
        a.prod[i].n = t[i].n;
        a.prod[i].y = make_out(t[i].y, t[i].m, t[i].n);
        a.prod[i].nk0 = (int)((t[i].a[0].k + 63) / 64);
        a.prod[i].nk = (int)steps_of(t[i]);
    }
    a.bias = t->bias;
    a.bias2 = t->bias2;
    a.act = act_for(t->act, t->y.dt == SADMM_BF16);
    if (t->residual.p) a.res = make_out(t->residual, t->m, t->n);
    if (t->z.p) a.z = make_out(t->z, t->m, t->n);
    if (t->u.p) a.u = make_out(t->u, t->m, t->n);
    a.status = device_status_ptr();
}

// Encodes a product's operands from map `next` on, with boxes of p_rows and
// q_rows; an operand that the product before it has too is not encoded again.
bool encode_product(TgMaps& maps, int& next, TgProduct& p, const TgProblem& t, bool swap, int p_rows, int q_rows,
                    const TgProduct* last, const TgProblem* last_t)
{
    const TgOperand* P = swap ? t.b : t.a;
    const TgOperand* Q = swap ? t.a : t.b;
    const bool p_two = t.mode == kTgSum || (t.mode == kTgGated && swap);
    const bool q_two = t.mode == kTgSum || (t.mode == kTgGated && !swap);
    p.p_kmajor = P[0].kmajor;
    p.q_kmajor = Q[0].kmajor;
    p.pm = next;
    for (int i = 0; i < (p_two ? 2 : 1); ++i)
        if (next >= kTgMaps || !encode(&maps.map[next++], P[i], p_rows)) return false;
    const TgOperand* lq = !last_t ? nullptr : swap ? last_t->a : last_t->b;
    if (lq && !q_two && lq->p == Q->p && lq->ld == Q->ld && lq->rows == Q->rows && lq->k == Q->k &&
        lq->kmajor == Q->kmajor) {
        p.qm = last->qm;
        return true;
    }
    p.qm = next;
    for (int i = 0; i < (q_two ? 2 : 1); ++i)
        if (next >= kTgMaps || !encode(&maps.map[next++], Q[i], q_rows)) return false;
    return true;
}

}  // namespace
}  // namespace sadmm
