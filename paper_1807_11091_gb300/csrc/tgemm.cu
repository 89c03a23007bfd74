// tgemm.cu -- the tensor-core products of the feed-forward operators
// (linear.cu): C = A B^T with bf16 operands, fp32 sums in TMEM and an epilogue
// that adds the bias, applies the activation, multiplies the gated pair and
// adds the residual in registers, so that nothing but the operator's own
// outputs is written.
//
// One CTA per 128 x bn tile, six warps:
//   warp 0      TMA producer: boxes of 64 contraction elements (K-major
//               operand: 64 x rows; row-contiguous operand: 64 rows x 64) with
//               the 128-byte swizzle
//   warp 1      TMEM allocator and issuer of tcgen05.mma (M 128, N bn, K 16)
//   warps 2-5   epilogue: tcgen05.ld, one lane per tile row
// The tile's 128 rows are the product's rows ("plain"), or, where there are few
// of those, its columns ("swapped": weights on the 128-row side, tokens on the
// bn side, so that a handful of tokens costs a handful of MMA columns).  Few
// tiles: the contraction is cut over the CTAs of a cluster, which leave their
// sums in shared memory and add each other's up in rank order, so that results
// do not depend on timing and no scratch memory is needed.
#include <cuda.h>
#include <cudaTypedefs.h>
#include <string.h>

#include "act.cuh"
#include "common.cuh"
#include "internal.h"
#include "tgemm.cuh"

namespace sadmm {

PFN_cuTensorMapEncodeTiled_v12000 get_encode_fn();  // pack.cu

namespace {

constexpr int kThreads = 192;
constexpr int kBox = 8192;        // one 64 x 64 bf16 box
constexpr int kPTile = 2 * kBox;  // 128 rows x 64
constexpr int kMaxStages = 8;
constexpr int kMaxAccCols = 128;  // accumulator columns of a CTA (fp32 sums: 64 KB when cut over a cluster)

// An output matrix as the epilogue stores it.  vec: 2 / 1 / 0 for rows on
// 32-byte / 16-byte / other boundaries.
struct Out {
    void* p;
    long long ld;
    long long total;  // elements from p to the end of the last row
    int bf16;
    int vec;
};

struct TgArgs {
    Out y, y2, res, z, u;
    const float* bias;
    const float* bias2;
    long long m, n;        // output rows, columns
    int act;
    int mode;
    int p_tiles;           // 128-row tiles of one product
    int q_tiles;
    int bn;                // rows of the Q side per tile (per half when gated)
    int nk0, nk;           // 64-element contraction steps: of the first summand, of all
    int splits, steps;     // CTAs per cluster, contraction steps of each
    int stages;
    int p_kmajor, q_kmajor;
    uint32_t stage_bytes, q_off;
    uint32_t acc_cols, tmem_cols;
    uint32_t idesc;
    int* status;
};

// ------------------------------------------------------------- device PTX --

SADMM_DEV uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}

// Every thread of every CTA of the cluster calls it.
SADMM_DEV void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}

SADMM_DEV uint32_t map_rank(uint32_t saddr, uint32_t rank)
{
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(saddr), "r"(rank));
    return a;
}

SADMM_DEV float ld_cluster_f32(uint32_t a)
{
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
    return v;
}

// Waits for the 128 epilogue threads.
SADMM_DEV void epi_sync() { asm volatile("bar.sync 1, 128;" ::: "memory"); }

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

SADMM_DEV void store1(const Out& o, long long r, long long c, float v, int* status)
{
    const long long at = r * o.ld + c;
    if (!dbg_in(at, o.total, status)) return;
    if (o.bf16)
        static_cast<__nv_bfloat16*>(o.p)[at] = __float2bfloat16_rn(v);
    else
        static_cast<float*>(o.p)[at] = v;
}

SADMM_DEV float load1(const Out& o, long long r, long long c, int* status)
{
    const long long at = r * o.ld + c;
    if (!dbg_in(at, o.total, status)) return 0.0f;
    return o.bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(o.p)[at]) : static_cast<const float*>(o.p)[at];
}

// Sixteen columns of one output row: sb / sb2 are the tile's biases in shared memory.
template <bool GATED>
SADMM_DEV void finish16(const TgArgs& a, const Out& y, long long r, long long c, float (&v)[16], float (&w)[16],
                        const float* sb, const float* sb2)
{
#pragma unroll
    for (int j = 0; j < 16; ++j) v[j] += sb[j];
    if (GATED) {
#pragma unroll
        for (int j = 0; j < 16; ++j) w[j] += sb2[j];
        if (a.u.p) store16(a.u, r, c, a.n, w, a.status);
    }
    if (a.z.p) store16(a.z, r, c, a.n, v, a.status);
    with_act(a.act, [&](auto tag) {
        constexpr int A = decltype(tag)::value;
#pragma unroll
        for (int j = 0; j < 16; ++j) v[j] = act_f32<A>(v[j]);
    });
    if (GATED) {
#pragma unroll
        for (int j = 0; j < 16; ++j) v[j] *= w[j];
    }
    if (a.res.p) add16(a.res, r, c, a.n, v, a.status);
    store16(y, r, c, a.n, v, a.status);
}

// One element.
template <bool GATED>
SADMM_DEV void finish1(const TgArgs& a, const Out& y, long long r, long long c, float v, float w, float b, float b2)
{
    v += b;
    if (GATED) {
        w += b2;
        if (a.u.p) store1(a.u, r, c, w, a.status);
    }
    if (a.z.p) store1(a.z, r, c, v, a.status);
    with_act(a.act, [&](auto tag) { v = act_f32<decltype(tag)::value>(v); });
    if (GATED) v *= w;
    if (a.res.p) v += load1(a.res, r, c, a.status);
    store1(y, r, c, v, a.status);
}

// ------------------------------------------------------------------ kernel --

// One operand's part of a stage: `rows` rows from row0, 64 contraction elements from k0.
SADMM_DEV void load_part(uint8_t* dst, const CUtensorMap* map, uint64_t* bar, int kmajor, int rows, int row0, int k0)
{
    if (kmajor) {
        tma_load_2d(dst, map, bar, k0, row0);
    } else {
        for (int j = 0; j * 64 < rows; ++j) tma_load_2d(dst + j * kBox, map, bar, row0 + 64 * j, k0);
    }
}

template <bool SWAP, bool GATED>
__global__ void __launch_bounds__(kThreads)
    k_tgemm(const __grid_constant__ CUtensorMap p0, const __grid_constant__ CUtensorMap p1,
            const __grid_constant__ CUtensorMap q0, const __grid_constant__ CUtensorMap q1,
            const __grid_constant__ TgArgs a)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    __shared__ uint64_t full[kMaxStages], empty[kMaxStages], acc_full, drain;
    __shared__ uint32_t tmem_holder;
    __shared__ volatile int abort_flag;
    __shared__ float s_bias[2 * kMaxAccCols];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    const uint32_t rank = a.splits > 1 ? cluster_rank() : 0;
    long long tile = blockIdx.x / a.splits;
    const int pt = (int)(tile % a.p_tiles);
    tile /= a.p_tiles;
    const int qt = (int)(tile % a.q_tiles);
    const int prob = (int)(tile / a.q_tiles);  // kTgPair: which product
    const int row0 = pt * 128, col0 = qt * a.bn;
    const int k_begin = min((int)rank * a.steps, a.nk), k_end = min(k_begin + a.steps, a.nk);
    const int nk = k_end - k_begin;

    if (threadIdx.x == 0) {
        for (int s = 0; s < a.stages; ++s) {
            mbar_init(&full[s], 1);
            mbar_init(&empty[s], 1);
        }
        mbar_init(&acc_full, 1);
        mbar_init(&drain, 1);
        abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == 1) {
        tmem_alloc(&tmem_holder, a.tmem_cols);
        tmem_relinquish();
    }
    pdl_wait();  // nothing above reads global memory
    pdl_trigger();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_holder;

    if (warp == 0) {
        if (lane == 0) {
            const CUtensorMap* pa = (a.mode == kTgPair && prob) ? &p1 : &p0;
            int issued = 0, s = 0;
            uint32_t phase = 0;
            for (int i = 0; i < nk; ++i) {
                if (!mbar_wait(&empty[s], phase ^ 1u, &abort_flag, a.status)) break;
                uint8_t* st = smem + (size_t)s * a.stage_bytes;
                mbar_arrive_expect_tx(&full[s], a.stage_bytes);
                int k = k_begin + i;
                const bool second = a.mode == kTgSum && k >= a.nk0;
                if (second) k -= a.nk0;
                load_part(st, second ? &p1 : pa, &full[s], a.p_kmajor, 128, row0, k * 64);
                if (GATED && SWAP) load_part(st + kPTile, &p1, &full[s], a.p_kmajor, 128, row0, k * 64);
                uint8_t* sq = st + a.q_off;
                load_part(sq, second ? &q1 : &q0, &full[s], a.q_kmajor, a.bn, col0, k * 64);
                if (GATED && !SWAP) load_part(sq + a.bn * 128, &q1, &full[s], a.q_kmajor, a.bn, col0, k * 64);
                ++issued;
                if (++s == a.stages) { s = 0; phase ^= 1u; }
            }
            // the loads issued have landed before the CTA retires
            for (int q = (issued > a.stages ? issued - a.stages : 0); q < issued; ++q) {
                const unsigned long long t0 = globaltimer();
                while (!mbar_try_wait(&full[q % a.stages], (uint32_t)(q / a.stages) & 1u) &&
                       globaltimer() - t0 < kWaitLimitNs) {}
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        const uint32_t pstep = a.p_kmajor ? 2u : 128u, qstep = a.q_kmajor ? 2u : 128u;  // 16 elements, in 16 bytes
        bool ok = true;
        int s = 0;
        uint32_t phase = 0;
        for (int i = 0; i < nk; ++i) {
            if (!mbar_wait_warp(&full[s], phase, &abort_flag, a.status)) { ok = false; break; }
            tc_fence_after();
            const uint32_t st = smem_u32(smem + (size_t)s * a.stage_bytes);
            const uint64_t pd = sdesc(st, a.p_kmajor), qd = sdesc(st + a.q_off, a.q_kmajor);
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
                mma_bf16_ss_elect(tmem, pd + kk * pstep, qd + kk * qstep, a.idesc, (i | kk) != 0);
                if (GATED && SWAP)
                    mma_bf16_ss_elect(tmem + a.bn, pd + (kPTile >> 4) + kk * pstep, qd + kk * qstep, a.idesc,
                                      (i | kk) != 0);
            }
            mma_commit_elect(&empty[s]);
            if (++s == a.stages) { s = 0; phase ^= 1u; }
        }
        if (ok) mma_commit_elect(&acc_full);
        mma_commit_elect(&drain);
        if (lane == 0) {
            const unsigned long long t0 = globaltimer();
            while (!mbar_try_wait(&drain, 0) && globaltimer() - t0 < kWaitLimitNs) {}
        }
        __syncwarp();
    }

    // ---- epilogue: TMEM lane = tile row
    const int q = warp & 3;
    const int trow = q * 32 + lane;
    const uint32_t taddr = tmem + ((uint32_t)(q * 32) << 16);
    float* part = reinterpret_cast<float*>(smem);  // [accumulator column][128 rows], when the contraction is cut
    bool ok = false;
    if (warp >= 2) {
        const int t = threadIdx.x - 64;
        if (!SWAP) {
            for (int j = t; j < a.bn; j += 128) {
                const long long c = col0 + j;
                s_bias[j] = a.bias && c < a.n ? a.bias[c] : 0.0f;
                if (GATED) s_bias[kMaxAccCols + j] = a.bias2 && c < a.n ? a.bias2[c] : 0.0f;
            }
            epi_sync();
        }
        ok = __all_sync(0xffffffffu, mbar_wait(&acc_full, 0, &abort_flag, a.status));
        tc_fence_after();
    }
    if (a.splits > 1) {
        if (warp >= 2 && ok) {
            for (uint32_t c = 0; c < a.acc_cols; c += 16) {
                uint32_t r[16];
                if (nk > 0) {
                    tmem_ld_32x32b_x16(taddr + c, r);
                    tmem_ld_wait();
                }
#pragma unroll
                for (int j = 0; j < 16; ++j) part[(c + j) * 128 + trow] = nk > 0 ? __uint_as_float(r[j]) : 0.0f;
            }
        }
        cluster_sync();
    }
    if (warp >= 2 && ok) {
        const Out& y = (a.mode == kTgPair && prob) ? a.y2 : a.y;
        const long long prow = (long long)row0 + trow;
        const uint32_t base = smem_u32(part) + 4u * (uint32_t)trow;
        if (SWAP) {
            const float b = a.bias && prow < a.n ? a.bias[prow] : 0.0f;
            const float b2 = GATED && a.bias2 && prow < a.n ? a.bias2[prow] : 0.0f;
            const int cols = (int)min((long long)a.bn, a.m - col0);
            if (a.splits > 1) {
                for (int c = (int)rank; c < cols; c += a.splits) {
                    float v = 0.0f, w = 0.0f;
                    for (int s = 0; s < a.splits; ++s) {
                        const uint32_t peer = map_rank(base, (uint32_t)s);
                        v += ld_cluster_f32(peer + (uint32_t)c * 512u);
                        if (GATED) w += ld_cluster_f32(peer + (uint32_t)(a.bn + c) * 512u);
                    }
                    if (prow < a.n) finish1<GATED>(a, y, col0 + c, prow, v, w, b, b2);
                }
            } else {
                for (int c0 = 0; c0 < cols; c0 += 16) {
                    uint32_t rv[16], rw[16];
                    if (nk > 0) {
                        tmem_ld_32x32b_x16(taddr + c0, rv);
                        if (GATED) tmem_ld_32x32b_x16(taddr + a.bn + c0, rw);
                        tmem_ld_wait();
                    }
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        if (c0 + j < cols && prow < a.n)
                            finish1<GATED>(a, y, col0 + c0 + j, prow, nk > 0 ? __uint_as_float(rv[j]) : 0.0f,
                                           GATED && nk > 0 ? __uint_as_float(rw[j]) : 0.0f, b, b2);
                }
            }
        } else {
            const int cols = (int)min((long long)a.bn, a.n - col0);
            const int first = a.splits > 1 ? 16 * (int)rank : 0, step = 16 * a.splits;
            for (int c = first; c < cols; c += step) {
                float v[16], w[16];
                if (a.splits > 1) {
#pragma unroll
                    for (int j = 0; j < 16; ++j) v[j] = w[j] = 0.0f;
                    for (int s = 0; s < a.splits; ++s) {
                        const uint32_t peer = map_rank(base, (uint32_t)s);
#pragma unroll
                        for (int j = 0; j < 16; ++j) v[j] += ld_cluster_f32(peer + (uint32_t)(c + j) * 512u);
                        if (GATED) {
#pragma unroll
                            for (int j = 0; j < 16; ++j) w[j] += ld_cluster_f32(peer + (uint32_t)(a.bn + c + j) * 512u);
                        }
                    }
                } else {
                    uint32_t rv[16], rw[16];
                    tmem_ld_32x32b_x16(taddr + c, rv);
                    if (GATED) tmem_ld_32x32b_x16(taddr + a.bn + c, rw);
                    tmem_ld_wait();
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        v[j] = __uint_as_float(rv[j]);
                        w[j] = GATED ? __uint_as_float(rw[j]) : 0.0f;
                    }
                }
                if (prow < a.m) finish16<GATED>(a, y, prow, col0 + c, v, w, s_bias + c, s_bias + kMaxAccCols + c);
            }
        }
    }
    if (a.splits > 1) cluster_sync();  // the others have read this CTA's sums
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, a.tmem_cols);
    }
}

// -------------------------------------------------------------------- host --

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

Out make_out(const TgMatrix& m, long long rows, long long cols)
{
    Out o;
    const long long es = m.dt == SADMM_BF16 ? 2 : 4;
    o.p = m.p;
    o.ld = m.ld;
    o.total = (rows - 1) * m.ld + cols;
    o.bf16 = m.dt == SADMM_BF16;
    const uintptr_t at = reinterpret_cast<uintptr_t>(m.p) | (uintptr_t)(m.ld * es);
    o.vec = at % 32 == 0 ? 2 : at % 16 == 0 ? 1 : 0;
    return o;
}

template <bool SWAP, bool GATED>
sadmm_status run(const CUtensorMap (&map)[4], const TgArgs& a, size_t smem, long long ctas, cudaStream_t s)
{
    static bool configured[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return SADMM_ECUDA;
    auto kern = k_tgemm<SWAP, GATED>;
    if (!configured[dev]) {
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, 220 * 1024) != cudaSuccess)
            return SADMM_ECUDA;
        configured[dev] = true;
    }
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)a.splits;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cfg.attrs = attr;
    cfg.numAttrs = a.splits > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kern, map[0], map[1], map[2], map[3], a) == cudaSuccess ? SADMM_OK : SADMM_ECUDA;
}

}  // namespace

sadmm_status launch_tgemm(const TgProblem& t, cudaStream_t s)
{
    const bool gated = t.mode == kTgGated;
    const bool swap = t.m <= 64 && t.b[0].rows > t.m && t.mode != kTgPair;
    const TgOperand* P = swap ? t.b : t.a;
    const TgOperand* Q = swap ? t.a : t.b;
    const long long p_rows = swap ? t.n : t.m, q_rows = swap ? t.m : t.n;
    TgArgs a;
    memset(&a, 0, sizeof(a));
    a.m = t.m;
    a.n = t.n;
    a.bias = t.bias;
    a.bias2 = t.bias2;
    a.act = t.act;
    a.mode = t.mode;
    a.y = make_out(t.y, t.m, t.n);
    if (t.mode == kTgPair) a.y2 = make_out(t.y2, t.m, t.n);
    if (t.residual.p) a.res = make_out(t.residual, t.m, t.n);
    if (t.z.p) a.z = make_out(t.z, t.m, t.n);
    if (t.u.p) a.u = make_out(t.u, t.m, t.n);
    a.p_kmajor = P[0].kmajor;
    a.q_kmajor = Q[0].kmajor;
    const int sm = device_sm_count();
    int bn = gated ? 64 : 128;
    if (swap) {
        bn = 16;
        while (bn < q_rows) bn <<= 1;
    }
    if (!a.q_kmajor && bn < 64) bn = 64;  // whole 64-row boxes
    a.bn = bn;
    a.p_tiles = (int)((p_rows + 127) / 128);
    a.q_tiles = (int)((q_rows + bn - 1) / bn);
    const long long products = t.mode == kTgPair ? 2 : 1;
    const long long tiles = (long long)a.p_tiles * a.q_tiles * products;
    a.nk0 = (int)((P[0].k + 63) / 64);
    a.nk = t.mode == kTgSum ? 2 * a.nk0 : a.nk0;
    // few tiles: each contraction is cut over 2, 4 or 8 CTAs (of at least four steps each)
    int splits = 1;
    while (splits < 8 && tiles * splits * 2 <= 2 * sm && a.nk >= 8 * splits) splits *= 2;
    a.splits = splits;
    a.steps = (a.nk + splits - 1) / splits;
    a.acc_cols = (uint32_t)(gated ? 2 * bn : bn);
    uint32_t cols = 32;
    while (cols < a.acc_cols) cols <<= 1;
    a.tmem_cols = cols;
    a.q_off = gated && swap ? 2 * kPTile : kPTile;
    a.stage_bytes = a.q_off + (uint32_t)(gated && !swap ? 2 * bn : bn) * 128u;
    // two CTAs an SM: one's epilogue beside the other's products
    a.stages = (int)(108 * 1024 / a.stage_bytes);
    if (a.stages > kMaxStages) a.stages = kMaxStages;
    if (a.stages > a.steps) a.stages = a.steps;
    size_t smem = (size_t)a.stages * a.stage_bytes;
    if (splits > 1 && smem < (size_t)a.acc_cols * 512) smem = (size_t)a.acc_cols * 512;
    smem += 1024;
    const int n_mma = gated && !swap ? 2 * bn : bn;
    a.idesc = idesc_bf16_f32(128, n_mma) | (a.p_kmajor ? 0u : 1u << 15) | (a.q_kmajor ? 0u : 1u << 16);
    a.status = device_status_ptr();
    if (tiles * splits > 0x7fffffffll) return SADMM_EUNSUPPORTED;
    alignas(64) CUtensorMap map[4];
    const bool p_two = t.mode == kTgSum || t.mode == kTgPair || (gated && swap);
    const bool q_two = t.mode == kTgSum || (gated && !swap);
    if (!encode(&map[0], P[0], 128) || !encode(&map[1], P[p_two ? 1 : 0], 128) || !encode(&map[2], Q[0], bn) ||
        !encode(&map[3], Q[q_two ? 1 : 0], bn))
        return SADMM_ECUDA;
    const long long ctas = tiles * splits;
    if (gated) return swap ? run<true, true>(map, a, smem, ctas, s) : run<false, true>(map, a, smem, ctas, s);
    return swap ? run<true, false>(map, a, smem, ctas, s) : run<false, false>(map, a, smem, ctas, s);
}

}  // namespace sadmm
