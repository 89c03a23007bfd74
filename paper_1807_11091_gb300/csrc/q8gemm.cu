// q8gemm.cu -- products of 8-bit matrices on the tensor cores, one tile a CTA:
//
//   C[m][n] = sum over blocks b of a_s[m][b] b_s[n][b] (sum over b of a_q b_q)
//
// A tile is 128 of the output's columns (P: the weights' rows, TMEM lanes) by
// up to 128 of its rows (Q: tokens).  The tensor cores (tcgen05.mma kind::f8f6f4)
// add up one block of 128, then the epilogue's warps multiply it by its scales and
// add it to fp32 sums in registers, while the next block's products run into
// another accumulator.  Few tiles share their contraction among the CTAs of
// a cluster, which exchange their sums through shared memory in rank order.
// Measured: one token, 5120 -> 4096, 6.9 us (3.1 of its 21 MB at 6.79 TB/s): bound by the latencies of
// a launch, of the loads and of the join; the gated pair of 16 tokens, 4096 -> 2 x 5461, 13.0
// (6.6 of its 45 MB), from 129 CTAs on 152 SMs; 777 dense rows, 2731 -> 1025, 20.4 with the copy of the
// unaligned operands (1.7).
// Per CTA, six warps:
//   warp 0     TMA producer
//   warp 1     TMEM allocator, issuer of the MMAs
//   warps 2-5  sums; then all six finish the output, a warp a row of 128
#include <string.h>

#include "q8.cuh"
#include "tgemm_dev.cuh"

namespace sadmm {
namespace {

constexpr int kThreads = 192;
constexpr int kStageSmem = 200 * 1024;
constexpr int kMostStages = 12;
constexpr int kPRows = 128;
constexpr int kPBytes = kPRows * kQBlock;

struct Scales {
    const float* s;
    long long s_row, s_block, rows;
    int shift;
    SADMM_DEV float at(long long r, int b) const { return r < rows ? s[(r >> shift) * s_row + b * s_block] : 0.0f; }
};

struct Maps {
    CUtensorMap p[2], q[2];
};

struct Args {
    Scales ps[2], qs[2];   // of both summands, or of the pair's weights and once of x
    int sum;               // the second half of the contraction is the second operands'
    int nk0, nk;           // blocks of the first summand, of all
    int splits, steps;     // CTAs of a cluster, blocks of each
    int stages, p_tiles;
    uint32_t stage_bytes, tmem_cols;
    uint32_t idesc;
    long long m, n;
    Out y, res, z, u;
    sadmm_q8_out y8;
    const float* bias;
    const float* bias2;
    int act;
    int* status;
};

SADMM_DEV void mma_f8_elect(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p, e;\n\t.reg .b32 l;\n\telect.sync l|e, 0xffffffff;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
        "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate));
}

// e4m3 A and B, K-major, fp32 accumulator.
constexpr uint32_t idesc_e4m3(int m, int n)
{
    return (1u << 4) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

// Four neighbouring 8-bit columns; a warp has the 128 of a block.
SADMM_DEV void put4(const Args& a, long long r, long long c, float (&v)[4])
{
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (c + j >= a.n) v[j] = 0.0f;
    float top = q8_top(v);
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const Q8Scale k = q8_scale(top);
    if (c >= a.n || !dbg_in(c, a.n, a.status) || !dbg_in(r, a.m, a.status)) return;
    if ((threadIdx.x & 31) == 0) a.y8.s[r * a.y8.s_row + c / kQBlock * a.y8.s_block] = k.s;
    const uint32_t q = q8_four(v[0], v[1], v[2], v[3], k);
    uint8_t* p = static_cast<uint8_t*>(a.y8.q) + r * a.y8.ld + c;
    if (c + 4 <= a.n && (reinterpret_cast<uintptr_t>(p) & 3) == 0) {
        *reinterpret_cast<uint32_t*>(p) = q;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (c + j < a.n) p[j] = (uint8_t)(q >> (8 * j));
    }
}

// Four neighbouring columns c .. c+3 of output row r; all lanes of a warp call it, a
// warp one row's 128 columns.  v (and w, the pair's u) are the sums.
template <bool GATED>
SADMM_DEV void finish4(const Args& a, long long r, long long c, float (&v)[4], float (&w)[4])
{
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (c + j < a.n) {
            if (a.bias) v[j] += a.bias[c + j];
            if (GATED && a.bias2) w[j] += a.bias2[c + j];
        }
    if (GATED && a.u.p) store_n<4>(a.u, r, c, a.n, w, a.status);
    if (a.z.p) store_n<4>(a.z, r, c, a.n, v, a.status);
    with_act(a.act, [&](auto tag) {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = act_f32<decltype(tag)::value>(v[j]);
    });
    if (GATED) {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] *= w[j];
    }
    if (a.res.p) {
        float e[4];
        load_n<4>(a.res, r, c, a.n, e, a.status);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] += e[j];
    }
    if (!GATED || !a.y8.q) {
        store_n<4>(a.y, r, c, a.n, v, a.status);
        return;
    }
    if constexpr (GATED) put4(a, r, c, v);
}

// PROWS: P's scales are single rows'; else one for the tile, which then goes into the other
// side's and saves a product an element.
template <bool GATED, int BN, bool PROWS>
__global__ void __launch_bounds__(kThreads, 1) k_q8_tiles(const __grid_constant__ Maps maps, const __grid_constant__ Args a)
{
    constexpr int H = GATED ? 2 : 1;
    constexpr int NB = 512 / (BN * H) < 4 ? 512 / (BN * H) : 4;  // accumulators
    constexpr int CH = BN < 32 ? BN : 32;                        // columns of a TMEM load
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    __shared__ uint64_t full[kMostStages], empty[kMostStages], acc_full[NB], acc_empty[NB];
    __shared__ uint32_t tmem_holder;
    __shared__ volatile int abort_flag;
    __shared__ __align__(16) float s_q[4][PROWS ? 1 : H][BN];  // a warp's own copy of the rows' scales
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const int rank = (int)(blockIdx.x % (unsigned)a.splits);
    const long long tile = blockIdx.x / (unsigned)a.splits;
    const long long qt = tile / a.p_tiles, pt = tile - qt * a.p_tiles;
    const long long p0 = pt * kPRows, q0 = qt * BN;
    const int k0 = min(rank * a.steps, a.nk), k1 = min(k0 + a.steps, a.nk);

    if (threadIdx.x == 0) {
        for (int s = 0; s < a.stages; ++s) {
            mbar_init(&full[s], 1);
            mbar_init(&empty[s], 1);
        }
        for (int b = 0; b < NB; ++b) {
            mbar_init(&acc_full[b], 1);
            mbar_init(&acc_empty[b], 4);
        }
        abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == 1) {
        tmem_alloc(&tmem_holder, a.tmem_cols);
        tmem_relinquish();
    }
    pdl_wait();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_holder;

    if (warp == 0) {
        if (lane == 0) {
            int s = 0;
            uint32_t phase = 0;
            bool ok = true;
            for (int k = k0; k < k1; ++k) {
                if (!mbar_wait(&empty[s], phase ^ 1u, &abort_flag, a.status)) { ok = false; break; }
                mbar_arrive_expect_tx(&full[s], (uint32_t)(H * kPBytes + BN * kQBlock));
                const int second = a.sum && k >= a.nk0;
                const int kc = (second ? k - a.nk0 : k) * kQBlock;
                uint8_t* sp = smem + (size_t)s * a.stage_bytes;
                tma_load_2d(sp, &maps.p[second], &full[s], kc, (int)p0);
                if (GATED) tma_load_2d(sp + kPBytes, &maps.p[1], &full[s], kc, (int)p0);
                tma_load_2d(sp + H * kPBytes, &maps.q[second], &full[s], kc, (int)q0);
                if (++s == a.stages) { s = 0; phase ^= 1u; }
            }
            if (!ok) {  // time for the copies in flight to land
                const unsigned long long t0 = globaltimer();
                while (globaltimer() - t0 < 10000000ull) {}
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        int s = 0, buf = 0;
        uint32_t phase = 0, bphase = 0;
        for (int k = k0; k < k1; ++k) {
            if (!mbar_wait_warp(&acc_empty[buf], bphase ^ 1u, &abort_flag, a.status)) break;
            if (!mbar_wait_warp(&full[s], phase, &abort_flag, a.status)) break;
            tc_fence_after();
            const uint32_t st = smem_u32(smem + (size_t)s * a.stage_bytes);
            const uint64_t qd = sdesc_kmajor_sw128(st + H * kPBytes);
#pragma unroll
            for (int h = 0; h < H; ++h) {
                const uint64_t pd = sdesc_kmajor_sw128(st + h * kPBytes);
                const uint32_t d = tmem + (uint32_t)((buf * H + h) * BN);
#pragma unroll
                for (int kk = 0; kk < 4; ++kk) mma_f8_elect(d, pd + kk * 2, qd + kk * 2, a.idesc, kk != 0);
            }
            mma_commit_elect(&empty[s]);
            mma_commit_elect(&acc_full[buf]);
            if (++s == a.stages) { s = 0; phase ^= 1u; }
            if (++buf == NB) { buf = 0; bphase ^= 1u; }
        }
        __syncwarp();
    } else {
        const int q = warp & 3;
        const uint32_t taddr = tmem + ((uint32_t)(q * 32) << 16);
        const long long prow = p0 + q * 32 + lane;
        float (&sq)[PROWS ? 1 : H][BN] = s_q[warp - 2];
        float acc[H][BN];
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
            for (int j = 0; j < BN; ++j) acc[h][j] = 0.0f;
        // the scales of the next blocks are on their way in registers, AHEAD of them (with one, each block waited for
        // its own: 1.2 us a block)
        constexpr int SQ = (BN + 31) / 32, AHEAD = 4;
        float nq[AHEAD][SQ], np[AHEAD][H];
        auto fetch = [&](int k, float (&q)[SQ], float (&p)[H]) {
            if (k >= k1) return;
            const int second = a.sum && k >= a.nk0;
            const int b = second ? k - a.nk0 : k;
#pragma unroll
            for (int i = 0; i < SQ; ++i) {
                const int j = i * 32 + lane;
                q[i] = j < BN ? a.qs[second].at(q0 + j, b) : 0.0f;
            }
#pragma unroll
            for (int h = 0; h < H; ++h) p[h] = a.ps[GATED ? h : second].at(PROWS ? prow : p0, b);
        };
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) fetch(k0 + i, nq[i], np[i]);
        int buf = 0;
        uint32_t bphase = 0;
        for (int k = k0; k < k1; ++k) {
            __syncwarp();  // the last block's scales have been read
#pragma unroll
            for (int i = 0; i < SQ; ++i)
                if (i * 32 + lane < BN) {
#pragma unroll
                    for (int h = 0; h < (PROWS ? 1 : H); ++h) sq[h][i * 32 + lane] = PROWS ? nq[0][i] : nq[0][i] * np[0][h];
                }
            float sp[H];
#pragma unroll
            for (int h = 0; h < H; ++h) sp[h] = np[0][h];
            __syncwarp();
#pragma unroll
            for (int d = 0; d + 1 < AHEAD; ++d) {
#pragma unroll
                for (int i = 0; i < SQ; ++i) nq[d][i] = nq[d + 1][i];
#pragma unroll
                for (int h = 0; h < H; ++h) np[d][h] = np[d + 1][h];
            }
            fetch(k + AHEAD, nq[AHEAD - 1], np[AHEAD - 1]);
            if (!mbar_wait_warp(&acc_full[buf], bphase, &abort_flag, a.status)) break;
            tc_fence_after();
#pragma unroll
            for (int h = 0; h < H; ++h) {
                const uint32_t from = taddr + (uint32_t)((buf * H + h) * BN);
#pragma unroll
                for (int c = 0; c < BN; c += CH) {
                    uint32_t r[CH];
                    if constexpr (CH == 32)
                        tmem_ld_32x32b_x32(from + c, r);
                    else
                        tmem_ld_32x32b_x16(from + c, r);
                    tmem_ld_wait();
#pragma unroll
                    for (int j = 0; j < CH; j += 4) {
                        float4 f = *reinterpret_cast<const float4*>(sq[PROWS ? 0 : h] + c + j);
                        if (PROWS) f.x *= sp[h], f.y *= sp[h], f.z *= sp[h], f.w *= sp[h];
                        acc[h][c + j] = fmaf(__uint_as_float(r[j]), f.x, acc[h][c + j]);
                        acc[h][c + j + 1] = fmaf(__uint_as_float(r[j + 1]), f.y, acc[h][c + j + 1]);
                        acc[h][c + j + 2] = fmaf(__uint_as_float(r[j + 2]), f.z, acc[h][c + j + 2]);
                        acc[h][c + j + 3] = fmaf(__uint_as_float(r[j + 3]), f.w, acc[h][c + j + 3]);
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&acc_empty[buf]);
            if (++buf == NB) { buf = 0; bphase ^= 1u; }
        }
        // the last accumulator is done, so the stages have been read; the sums take their place
        float* part = reinterpret_cast<float*>(smem);
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
            for (int j = 0; j < BN; ++j) part[(h * BN + j) * kPRows + q * 32 + lane] = acc[h][j];
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();
    // the cluster's CTAs finish the tile's rows in turn
    const int rows = (int)min((long long)BN, a.m - q0);
    for (int j = rank * (kThreads / 32) + warp; j < rows; j += a.splits * (kThreads / 32)) {
        float v[2][4], e[H][8][4];
        // all of them on their way before the first is added
#pragma unroll
        for (int h = 0; h < H; ++h) {
            const uint32_t at = smem_u32(smem) + (uint32_t)((h * BN + j) * kPRows + lane * 4) * 4u;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < a.splits) ld_cluster<4>(map_rank(at, (uint32_t)i), e[h][i]);
        }
#pragma unroll
        for (int h = 0; h < H; ++h) {
#pragma unroll
            for (int l = 0; l < 4; ++l) v[h][l] = e[h][0][l];
#pragma unroll
            for (int i = 1; i < 8; ++i)
                if (i < a.splits) {
#pragma unroll
                    for (int l = 0; l < 4; ++l) v[h][l] += e[h][i][l];
                }
        }
        finish4<GATED>(a, q0 + j, p0 + lane * 4, v[0], v[1]);
    }
    cluster_sync();  // the others have read this CTA's sums
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, a.tmem_cols);
    }
}

bool encode8(CUtensorMap* map, const Q8Operand& o, int box_rows)
{
    PFN_cuTensorMapEncodeTiled_v12000 enc = get_encode_fn();
    if (!enc) return false;
    memset(map, 0, sizeof(*map));
    const cuuint64_t gdim[2] = {(cuuint64_t)o.k, (cuuint64_t)o.rows};
    const cuuint64_t gstride[1] = {(cuuint64_t)o.ld};
    const cuuint32_t box[2] = {(cuuint32_t)kQBlock, (cuuint32_t)box_rows};
    const cuuint32_t estride[2] = {1u, 1u};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(o.p), gdim, gstride, box, estride,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

Scales scales_of(const Q8Operand& o) { return {o.s, o.s_row, o.s_block, o.rows, o.shift}; }

// Clusters of n CTAs of this kernel's kind that the device holds at once, one CTA an SM (a GPC's SMs
// are no multiple of eight: of 128 CTAs in clusters of eight the last ones waited, 11.7 us where
// clusters of four take 7.8).
int clusters_at_once(int n)
{
    static int known[64][9];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
    if (!known[dev][n]) {
        auto kern = k_q8_tiles<false, 128, false>;
        constexpr int smem = kStageSmem + 1024;
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) return 0;
        cudaLaunchAttribute attr;
        attr.id = cudaLaunchAttributeClusterDimension;
        attr.val.clusterDim.x = (unsigned)n;
        attr.val.clusterDim.y = 1;
        attr.val.clusterDim.z = 1;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)n);
        cfg.blockDim = dim3(kThreads);
        cfg.dynamicSmemBytes = smem;
        cfg.attrs = &attr;
        cfg.numAttrs = 1;
        int most = 0;
        if (cudaOccupancyMaxActiveClusters(&most, kern, &cfg) != cudaSuccess) {
            cudaGetLastError();
            most = device_sm_count() / (2 * n);
        }
        known[dev][n] = most > 0 ? most : 1;
    }
    return known[dev][n];
}

// CTAs that share a tile's contraction: as many as run at once (eight at most), none
// of them without a block.
int split_of(long long tiles, int nk)
{
    int n = nk < 8 ? nk : 8;
    while (n > 1 && tiles > clusters_at_once(n)) --n;
    const int steps = (nk + n - 1) / n;
    return (nk + steps - 1) / steps;
}

// Output rows of a tile.
int rows_of_tile(const Q8Problem& t)
{
    if (t.m <= 16) return 16;
    if (t.m <= 32) return 32;
    return t.m <= 64 || t.mode == kTgGated ? 64 : 128;
}

template <bool GATED, int BN, bool PROWS>
sadmm_status run(const Q8Problem& t, Args a, cudaStream_t s)
{
    constexpr int H = GATED ? 2 : 1;
    static bool configured[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return SADMM_ECUDA;
    constexpr int smem = kStageSmem + 1024;
    auto kern = k_q8_tiles<GATED, BN, PROWS>;
    if (!configured[dev]) {
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess)
            return SADMM_ECUDA;
        configured[dev] = true;
    }
    Maps maps;
    const bool two = t.mode != kTgSingle;
    for (int i = 0; i < 2; ++i) {
        const Q8Operand &p = t.b[two ? i : 0], &q = t.a[t.mode == kTgSum ? i : 0];
        if (!encode8(&maps.p[i], p, kPRows) || !encode8(&maps.q[i], q, BN)) return SADMM_ECUDA;
        a.ps[i] = scales_of(p);
        a.qs[i] = scales_of(q);
    }
    a.stage_bytes = H * kPBytes + BN * kQBlock;
    a.stages = kStageSmem / (int)a.stage_bytes;
    if (a.stages > kMostStages) a.stages = kMostStages;
    constexpr int cols = (512 / (BN * H) < 4 ? 512 / (BN * H) : 4) * BN * H;
    a.tmem_cols = cols;
    a.idesc = idesc_e4m3(kPRows, BN);
    a.p_tiles = (int)((t.n + kPRows - 1) / kPRows);
    const long long tiles = a.p_tiles * ((t.m + BN - 1) / BN);
    a.splits = split_of(tiles, a.nk);
    a.steps = (a.nk + a.splits - 1) / a.splits;
    if (tiles * a.splits > 0x7fffffffll) return SADMM_EUNSUPPORTED;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)a.splits;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(tiles * a.splits));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kern, maps, a) == cudaSuccess ? SADMM_OK : SADMM_ECUDA;
}

template <bool GATED, int BN>
sadmm_status run(const Q8Problem& t, const Args& a, cudaStream_t s)
{
    const bool rows = t.b[0].shift == 0 || (t.mode != kTgSingle && t.b[1].shift == 0);
    return rows ? run<GATED, BN, true>(t, a, s) : run<GATED, BN, false>(t, a, s);
}

}  // namespace

sadmm_status launch_q8_product(const Q8Problem& t, cudaStream_t s)
{
    Args a;
    memset(&a, 0, sizeof(a));
    a.sum = t.mode == kTgSum;
    a.nk0 = (int)((t.a[0].k + kQBlock - 1) / kQBlock);
    a.nk = a.nk0 + (a.sum ? (int)((t.a[1].k + kQBlock - 1) / kQBlock) : 0);
    a.m = t.m;
    a.n = t.n;
    a.y8 = t.y8;
    if (t.y.p) a.y = make_out(t.y, t.m, t.n);
    if (t.residual.p) a.res = make_out(t.residual, t.m, t.n);
    if (t.z.p) a.z = make_out(t.z, t.m, t.n);
    if (t.u.p) a.u = make_out(t.u, t.m, t.n);
    a.bias = t.bias;
    a.bias2 = t.bias2;
    a.act = act_for(t.act, t.y.p && t.y.dt == SADMM_BF16);
    a.status = device_status_ptr();
    const int bn = rows_of_tile(t);
    if (t.mode == kTgGated) {
        if (bn == 16) return run<true, 16>(t, a, s);
        return bn == 32 ? run<true, 32>(t, a, s) : run<true, 64>(t, a, s);
    }
    if (bn == 16) return run<false, 16>(t, a, s);
    if (bn == 32) return run<false, 32>(t, a, s);
    return bn == 64 ? run<false, 64>(t, a, s) : run<false, 128>(t, a, s);
}

// Expected time, ns.  Measured: a block takes 0.20 us on tiles of 16 rows, 0.25 on 32, 0.33 on
// 64, 0.56 on 128 (the gated pair's 0.27, 0.45, 0.70); a round of tiles 3.5 beside its blocks,
// a launch 4, the join of a split contraction 2.
long long time_q8_product(const Q8Problem& t)
{
    const bool gated = t.mode == kTgGated;
    const int bn = rows_of_tile(t);
    const int nk = (int)((t.a[0].k + kQBlock - 1) / kQBlock) + (t.mode == kTgSum ? (int)((t.a[1].k + kQBlock - 1) / kQBlock) : 0);
    const long long tiles = (t.n + kPRows - 1) / kPRows * ((t.m + bn - 1) / bn);
    const int splits = split_of(tiles, nk), steps = (nk + splits - 1) / splits;
    const long long rounds = (tiles * splits + device_sm_count() - 1) / device_sm_count();
    const long long block = bn == 16 ? (gated ? 270 : 200) : bn == 32 ? (gated ? 450 : 250) : bn == 64 ? (gated ? 700 : 330) : 560;
    return rounds * (steps * block + 3500) + 4000 + (splits > 1 ? 2000 : 0);
}

}  // namespace sadmm
