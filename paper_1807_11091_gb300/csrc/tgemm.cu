// tgemm.cu -- the tensor-core products of the feed-forward operators
// (linear.cu): C = A B^T with bf16 operands, fp32 sums in TMEM and an epilogue
// that adds the bias, applies the activation, multiplies the gated pair and
// adds the residual in registers, so that nothing but the operator's own
// outputs is written.
//
// One CTA per 128 x bn tile, eight warps:
//   warp 0      TMA producer: boxes of 64 contraction elements (K-major
//               operand: 64 x rows; row-contiguous operand: 64 rows x 64) with
//               the 128-byte swizzle
//   warp 1      TMEM allocator and issuer of tcgen05.mma (M 128, N bn, K 16)
//   warps 2-5   tcgen05.ld of the sums, one lane per tile row; then all eight
//               warps finish the output's rows
// The tile's 128 rows are the product's rows ("plain"), or, where there are few
// of those, its columns ("swapped": weights on the 128-row side, tokens on the
// bn side, so that a handful of tokens costs a handful of MMA columns).  Where
// tiles are few or uneven the contraction is cut over the CTAs of a cluster,
// which leave their sums in shared memory and add each other's up in rank
// order, so that results do not depend on timing and no scratch memory is
// needed.  Where eight CTAs are not enough to keep an fp32 output's sums inside the
// tensor cores to 1024 terms (LONG), these go to registers by kLongSteps steps,
// through two accumulators in turn (dW of 64 units over 65536 tokens in one sum of
// 8192 a CTA: off by 9.1e-6 in norm, so by 0.72e-6; 40 tokens of 16384 -> 5000: 50.1
// us and 52.7).
//
// Bound by latency at the sizes that come here: a launch takes 6 us beside its
// steps (first loads, joining, the last stores).  777 x 2736 -> 1024 takes 13.2 us,
// 1024^3 10, 17 tokens of 8192 -> 8192 26.6 (their weights alone 20), the gated
// pair of 17 tokens 2048 -> 2 x 5464 11.
#include "tgemm_dev.cuh"

namespace sadmm {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxStages = 8;
constexpr int kPrefetchSteps = 32;
constexpr int kSwapStride = 132;  // floats of a staged row of 128, so that neither way in or out has bank conflicts

template <bool SWAP, bool GATED, bool LONG>
__global__ void __launch_bounds__(kThreads, LONG ? 1 : 2)
    k_tgemm(const __grid_constant__ TgMaps maps, const __grid_constant__ TgArgs a)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    __shared__ uint64_t full[kMaxStages], empty[kMaxStages], acc_full[2], acc_empty[2], drain;
    __shared__ uint32_t tmem_holder;
    __shared__ volatile int abort_flag;
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;  // uniform

    const uint32_t rank = a.splits > 1 ? cluster_rank() : 0;
    int tile = (int)(blockIdx.x / (unsigned)a.splits), which = 0;
    while (which + 1 < a.products && tile >= a.prod[which + 1].first) ++which;
    const TgProduct& p = a.prod[which];
    tile -= p.first;
    const int qt = tile / p.p_tiles, pt = tile - qt * p.p_tiles;
    const int row0 = pt * 128, col0 = qt * a.bn;
    const int k_begin = min((int)rank * p.steps, p.nk), k_end = min(k_begin + p.steps, p.nk);
    const int nk = k_end - k_begin;

    if (threadIdx.x == 0) {
        for (int s = 0; s < a.stages; ++s) {
            mbar_init(&full[s], 1);
            mbar_init(&empty[s], 1);
        }
        for (int b = 0; b < (LONG ? 2 : 1); ++b) {
            mbar_init(&acc_full[b], 1);
            if (LONG) mbar_init(&acc_empty[b], 4);  // the warps that read the sums
        }
        mbar_init(&drain, 1);
        abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == 1) {
        tmem_alloc(&tmem_holder, a.tmem_cols);
        tmem_relinquish();
    }
    if (SWAP && warp == 0 && lane == 0) {
        // the weights are what a few tokens wait for: on their way to L2 while the kernel before still runs
        for (int i = 0; i < nk && i < kPrefetchSteps; ++i) {
            int k = k_begin + i;
            const int second = k >= p.nk0;
            if (second) k -= p.nk0;
            for (int half = 0; half < (GATED ? 2 : 1); ++half) {
                const CUtensorMap* map = &maps.map[p.pm + second + half];
                if (p.p_kmajor) {
                    tma_prefetch_2d(map, k * 64, row0);
                } else {
                    tma_prefetch_2d(map, row0, k * 64);
                    tma_prefetch_2d(map, row0 + 64, k * 64);
                }
            }
        }
    }
    pdl_wait();  // nothing above reads what an earlier kernel may write
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    // (clusters do not: see common.cuh; and not before this CTA has its TMEM, which the next kernel may want too)
    if (a.splits == 1) pdl_trigger();
    const uint32_t tmem = tmem_holder;

    if (warp == 0) {
        if (lane == 0) {
            const CUtensorMap *p0 = &maps.map[p.pm], *q0 = &maps.map[p.qm];
            int issued = 0, s = 0;
            uint32_t phase = 0;
            for (int i = 0; i < nk; ++i) {
                if (!mbar_wait(&empty[s], phase ^ 1u, &abort_flag, a.status)) break;
                uint8_t* st = smem + (size_t)s * a.stage_bytes;
                mbar_arrive_expect_tx(&full[s], a.stage_bytes);
                int k = k_begin + i;
                const int second = k >= p.nk0;  // of a sum
                if (second) k -= p.nk0;
                load_part(st, p0 + second, &full[s], p.p_kmajor, 128, row0, k * 64);
                if (GATED && SWAP) load_part(st + kPTile, p0 + 1, &full[s], p.p_kmajor, 128, row0, k * 64);
                uint8_t* sq = st + a.q_off;
                load_part(sq, q0 + second, &full[s], p.q_kmajor, a.bn, col0, k * 64);
                if (GATED && !SWAP) load_part(sq + a.bn * 128, q0 + 1, &full[s], p.q_kmajor, a.bn, col0, k * 64);
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
        const uint32_t pstep = p.p_kmajor ? 2u : 128u, qstep = p.q_kmajor ? 2u : 128u;  // 16 elements, in 16 bytes
        bool ok = true;
        int s = 0, buf = 0, held = 0;  // LONG: the accumulator and its steps
        uint32_t phase = 0, bphase = 0, d = tmem;
        for (int i = 0; i < nk; ++i) {
            if constexpr (LONG) {
                ok = held != 0 || mbar_wait_warp(&acc_empty[buf], bphase ^ 1u, &abort_flag, a.status);
                if (!ok) break;
                d = tmem + (uint32_t)buf * a.acc_cols;
            }
            if (!mbar_wait_warp(&full[s], phase, &abort_flag, a.status)) { ok = false; break; }
            tc_fence_after();
            const uint32_t st = smem_u32(smem + (size_t)s * a.stage_bytes);
            const uint64_t pd = sdesc(st, p.p_kmajor), qd = sdesc(st + a.q_off, p.q_kmajor);
            const int before = LONG ? held : i;
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
                mma_bf16_ss_elect(d, pd + kk * pstep, qd + kk * qstep, p.idesc, (before | kk) != 0);
                if (GATED && SWAP)
                    mma_bf16_ss_elect(d + a.bn, pd + (kPTile >> 4) + kk * pstep, qd + kk * qstep, p.idesc,
                                      (before | kk) != 0);
            }
            mma_commit_elect(&empty[s]);
            if (++s == a.stages) { s = 0; phase ^= 1u; }
            if constexpr (LONG) {
                if (++held == p.acc_steps || i + 1 == nk) {
                    mma_commit_elect(&acc_full[buf]);
                    held = 0;
                    if (++buf == 2) { buf = 0; bphase ^= 1u; }
                }
            }
        }
        if (!LONG && ok) mma_commit_elect(&acc_full[0]);
        mma_commit_elect(&drain);
        if (lane == 0) {
            const unsigned long long t0 = globaltimer();
            while (!mbar_try_wait(&drain, 0) && globaltimer() - t0 < kWaitLimitNs) {}
        }
        __syncwarp();
    }

    // ---- epilogue: the sums to shared memory as rows of the output, then every warp of the cluster's CTAs takes
    // rows of them in turn, a lane N neighbouring columns, so that loads and stores are neighbours whatever the
    // output's alignment
    constexpr int N = !SWAP && GATED ? 2 : 4;
    float* part = reinterpret_cast<float*>(smem);
    const int live = (int)min((long long)(SWAP ? a.bn : 128), p.m - (SWAP ? col0 : row0));  // rows
    const uint32_t stride = SWAP ? kSwapStride : a.acc_cols + 4;                             // floats of a staged row
    const uint32_t u_off = SWAP ? (uint32_t)a.bn * kSwapStride : (uint32_t)a.bn;             // gated: from g to u
    if constexpr (LONG) {  // (not the gated pair)
        if (warp >= 2 && warp < 6) {
            const int q = warp & 3, trow = q * 32 + lane, columns = SWAP ? live : (int)a.acc_cols;
            const uint32_t taddr = tmem + ((uint32_t)(q * 32) << 16);
            float sum[8][16];  // 128 columns at most
#pragma unroll
            for (int h = 0; h < 8; ++h)
#pragma unroll
                for (int j = 0; j < 16; ++j) sum[h][j] = 0.0f;
            bool ok = true;
            int buf = 0;
            uint32_t bphase = 0;
            for (int i = 0; i < nk; i += p.acc_steps) {
                ok = __all_sync(0xffffffffu, mbar_wait(&acc_full[buf], bphase, &abort_flag, a.status));
                if (!ok) break;
                tc_fence_after();
#pragma unroll
                for (int h = 0; h < 8; ++h) {
                    if (16 * h >= columns) continue;
                    uint32_t r[16];
                    tmem_ld_32x32b_x16(taddr + (uint32_t)buf * a.acc_cols + 16 * h, r);
                    tmem_ld_wait();
#pragma unroll
                    for (int j = 0; j < 16; ++j) sum[h][j] += __uint_as_float(r[j]);
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&acc_empty[buf]);
                if (++buf == 2) { buf = 0; bphase ^= 1u; }
            }
            if (ok) {  // the last accumulator is there, so the stages have been read
#pragma unroll
                for (int h = 0; h < 8; ++h) {
                    if (16 * h >= columns) continue;
                    if (SWAP) {
#pragma unroll
                        for (int j = 0; j < 16; ++j) part[(16 * h + j) * kSwapStride + trow] = sum[h][j];
                    } else {
#pragma unroll
                        for (int j = 0; j < 16; j += 4)
                            *reinterpret_cast<float4*>(part + trow * stride + 16 * h + j) =
                                make_float4(sum[h][j], sum[h][j + 1], sum[h][j + 2], sum[h][j + 3]);
                    }
                }
            }
        }
    }
    if (!LONG && warp >= 2 && warp < 6 && __all_sync(0xffffffffu, mbar_wait(&acc_full[0], 0, &abort_flag, a.status))) {
        const int q = warp & 3, trow = q * 32 + lane;
        const uint32_t taddr = tmem + ((uint32_t)(q * 32) << 16);
        tc_fence_after();
        for (uint32_t c = 0; c < a.acc_cols; c += 16) {
            if (SWAP && (int)(c >= (uint32_t)a.bn ? c - a.bn : c) >= live) continue;
            uint32_t r[16];
            if (nk > 0) {
                tmem_ld_32x32b_x16(taddr + c, r);
                tmem_ld_wait();
            } else {
#pragma unroll
                for (int j = 0; j < 16; ++j) r[j] = 0;
            }
            if (SWAP) {
#pragma unroll
                for (int j = 0; j < 16; ++j) part[(c + j) * kSwapStride + trow] = __uint_as_float(r[j]);
            } else {
#pragma unroll
                for (int j = 0; j < 16; j += 4)
                    *reinterpret_cast<uint4*>(part + trow * stride + c + j) = make_uint4(r[j], r[j + 1], r[j + 2], r[j + 3]);
            }
        }
    }
    if (a.splits > 1)
        cluster_sync();
    else
        __syncthreads();
    if (!abort_flag) {
        const long long col = (SWAP ? row0 : col0) + lane * N;
        const int first_row = SWAP ? col0 : row0;
        float b[N], b2[N];
#pragma unroll
        for (int j = 0; j < N; ++j) {
            b[j] = a.bias && col + j < p.n ? a.bias[col + j] : 0.0f;
            b2[j] = GATED && a.bias2 && col + j < p.n ? a.bias2[col + j] : 0.0f;
        }
        const uint32_t base = smem_u32(part) + 4u * (uint32_t)(lane * N);
        auto rows = [&](auto cut) {
            constexpr int S = decltype(cut)::value;
            constexpr int kStep = S * (kThreads / 32);
            auto load = [&](int i, float (&t)[S][N], float (&tw)[GATED ? S : 1][N], float (&e)[N]) {
                const uint32_t at = base + 4u * (uint32_t)i * stride;
#pragma unroll
                for (int s = 0; s < S; ++s) {
                    if constexpr (S == 1) {
                        ld_own<N>(at, t[s]);
                        if (GATED) ld_own<N>(at + 4u * u_off, tw[s]);
                    } else {
                        const uint32_t peer = map_rank(at, (uint32_t)s);
                        ld_cluster<N>(peer, t[s]);
                        if (GATED) ld_cluster<N>(peer + 4u * u_off, tw[GATED ? s : 0]);
                    }
                }
                if (a.res.p) load_n<N>(a.res, first_row + i, col, p.n, e, a.status);
            };
            // the next row's loads run beside this row's arithmetic; one copy of the code, which is what fits the
            // instruction cache
            float t[S][N], tw[GATED ? S : 1][N], e[N];
            int i = (int)rank + S * warp;
            if (i < live) load(i, t, tw, e);
#pragma unroll 1
            for (; i < live; i += kStep) {
                float v[N], w[N], r[N];
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    v[j] = t[0][j];
                    w[j] = GATED ? tw[0][j] : 0.0f;
                    r[j] = e[j];
#pragma unroll
                    for (int s = 1; s < S; ++s) {
                        v[j] += t[s][j];
                        if (GATED) w[j] += tw[GATED ? s : 0][j];
                    }
                }
                if (i + kStep < live) load(i + kStep, t, tw, e);
                if (col < p.n) finish_n<GATED, N>(a, p, first_row + i, col, v, w, b, b2, r);
            }
        };
        switch (a.splits) {
        case 1: rows(ActTag<1>()); break;
        case 2: rows(ActTag<2>()); break;
        case 4: rows(ActTag<4>()); break;
        default: rows(ActTag<8>()); break;
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

template <bool SWAP, bool GATED, bool LONG>
sadmm_status run(const TgMaps& maps, const TgArgs& a, size_t smem, cudaStream_t s)
{
    static bool configured[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return SADMM_ECUDA;
    auto kern = k_tgemm<SWAP, GATED, LONG>;
    if (!configured[dev]) {
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, 112 * 1024) != cudaSuccess)
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
    cfg.gridDim = dim3((unsigned)a.tiles * (unsigned)a.splits);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cfg.attrs = attr;
    cfg.numAttrs = a.splits > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kern, maps, a) == cudaSuccess ? SADMM_OK : SADMM_ECUDA;
}

// Weights on the 128-row side, tokens on the other: products of few rows.
bool swapped(const TgProblem& t) { return t.m <= 64 && t.n > t.m; }

// Rows of the Q side per tile (per half when gated).
int tile_width(const TgProblem* t, int count)
{
    if (!swapped(*t)) return t->mode == kTgGated ? 64 : 128;
    long long most = 0;
    bool boxes = false;
    for (int i = 0; i < count; ++i) {
        if (t[i].m > most) most = t[i].m;
        boxes = boxes || !t[i].a[0].kmajor;
    }
    int bn = boxes ? 64 : 16;  // row-contiguous operands come in whole 64-row boxes
    while (bn < most) bn <<= 1;
    return bn;
}

// CTAs that each contraction is cut over, 1, 2, 4 or 8 (of at least two steps
// each), and an estimate of the time in 10 ns.  Measured: a round of CTAs (two
// an SM) takes 6 us beside its steps and 8 us each one after the first, a step
// 0.3 us where a CTA has its SM to itself and 0.5 us where two share it, joining
// the parts 1 us (777 x 2736 -> 1024: 19.9 us whole, 14.1 / 13.5 / 21.5 cut in 2
// / 4 / 8; 512 x 4096 -> 4096: 27.3, 20.9, 29.2, 47.8).  An fp32 output's
// contraction is cut anyway, so that no sum inside the tensor cores passes 1024
// elements where 8 CTAs are enough for that (elsewhere: LONG).
struct Cut {
    int splits;
    long long time;
};
Cut choose_cut(const TgProblem* t, int count)
{
    const int bn = tile_width(t, count);
    const long long sm = device_sm_count();
    long long tiles = 0, work = 0, nk = 0, longest = 0;
    bool alike = true;
    for (int i = 0; i < count; ++i) {
        const long long steps = steps_of(t[i]);
        const bool swap = swapped(t[i]);
        const long long n = ((swap ? t[i].n : t[i].m) + 127) / 128 * (((swap ? t[i].m : t[i].n) + bn - 1) / bn);
        tiles += n;
        work += n * steps;
        alike = alike && (!i || steps == nk);
        if (steps > nk) nk = steps;
        if (t[i].y.dt == SADMM_FP32 && steps > longest) longest = steps;
    }
    Cut best = {1, 0};
    for (int s = 1; s <= 8; s *= 2) {
        if (s > 1 && nk < 2 * s) break;
        const long long ctas = tiles * s, steps = (nk + s - 1) / s;
        const long long rounds = (ctas + 2 * sm - 1) / (2 * sm);
        long long busiest = steps * (alike ? rounds : 1);  // steps of one place for a CTA
        if (!alike && busiest < work / (2 * sm)) busiest = work / (2 * sm);
        const long long time = 600 + 800 * (rounds - 1) + busiest * (ctas > sm ? 50 : 30) + (s > 1 ? 100 : 0) +
                               (s == 8 && ctas > sm ? 250 : 0);  // clusters of eight, two CTAs an SM
        if (s == 1 || time < best.time || longest > 16 * best.splits) best = {s, time};
    }
    return best;
}

sadmm_status launch_tiles(const TgProblem* t, int count, int splits, cudaStream_t s)
{
    const bool gated = t->mode == kTgGated, swap = swapped(*t);
    TgArgs a;
    TgMaps maps;
    fill_common(a, t, count);
    const int bn = tile_width(t, count);
    a.bn = bn;
    long long tiles = 0;
    int next = 0;
    const int n_mma = gated && !swap ? 2 * bn : bn;
    for (int i = 0; i < count; ++i) {
        TgProduct& p = a.prod[i];
        const long long p_rows = swap ? p.n : p.m, q_rows = swap ? p.m : p.n;
        p.p_tiles = (int)((p_rows + 127) / 128);
        p.q_tiles = (int)((q_rows + bn - 1) / bn);
        p.first = (int)tiles;
        tiles += (long long)p.p_tiles * p.q_tiles;
        if (tiles > 0x0fffffffll) return SADMM_EUNSUPPORTED;
        if (!encode_product(maps, next, p, t[i], swap, 128, bn, i ? &a.prod[i - 1] : nullptr, i ? &t[i - 1] : nullptr))
            return SADMM_ECUDA;
        p.idesc = idesc_bf16_f32(128, n_mma) | (p.p_kmajor ? 0u : 1u << 15) | (p.q_kmajor ? 0u : 1u << 16);
    }
    a.tiles = (int)tiles;
    a.splits = splits;
    int steps = 1;
    bool lng = false;
    for (int i = 0; i < count; ++i) {
        TgProduct& p = a.prod[i];
        p.steps = p.acc_steps = (p.nk + splits - 1) / splits;
        if (p.steps > steps) steps = p.steps;
        if (!gated && !p.y.bf16 && p.steps > 16) {
            p.acc_steps = kLongSteps;
            lng = true;
        }
    }
    a.acc_cols = (uint32_t)(gated ? 2 * bn : bn);
    uint32_t cols = 32;
    while (cols < (lng ? 2 : 1) * a.acc_cols) cols <<= 1;
    a.tmem_cols = cols;
    a.q_off = gated && swap ? 2 * kPTile : kPTile;
    a.stage_bytes = a.q_off + (uint32_t)n_mma * 128u;
    // two CTAs an SM: one's epilogue beside the other's products
    a.stages = (int)(108 * 1024 / a.stage_bytes);
    if (a.stages > kMaxStages) a.stages = kMaxStages;
    if (a.stages > steps) a.stages = steps;
    size_t smem = (size_t)a.stages * a.stage_bytes;
    const size_t staged = 4 * (size_t)(swap ? a.acc_cols * kSwapStride : 128 * (a.acc_cols + 4));
    if (smem < staged) smem = staged;
    smem += 1024;
    if (gated) return swap ? run<true, true, false>(maps, a, smem, s) : run<false, true, false>(maps, a, smem, s);
    if (lng) return swap ? run<true, false, true>(maps, a, smem, s) : run<false, false, true>(maps, a, smem, s);
    return swap ? run<true, false, false>(maps, a, smem, s) : run<false, false, false>(maps, a, smem, s);
}

}  // namespace

sadmm_status launch_tgemm(const TgProblem* all, int count, cudaStream_t s)
{
    for (int i = 1; i < count; ++i) {
        if (swapped(all[i]) == swapped(all[0])) continue;
        for (int j = 0; j < count; ++j) {
            const sadmm_status st = launch_tgemm(all + j, 1, s);
            if (st != SADMM_OK) return st;
        }
        return SADMM_OK;
    }
    TgProblem t[kTgProducts];
    int wanted = 0;
    for (int i = 0; i < count; ++i)
        if (!all[i].skip) t[wanted++] = all[i];
    if (!wanted) return SADMM_OK;
    const Cut cut = choose_cut(all, count);
    if (!swapped(all[0])) {
        if (choose_tgemm_pair(all, count).time < cut.time)
            return launch_tgemm_pair(t, wanted, choose_tgemm_pair(t, wanted).bn, s);
    }
    return launch_tiles(t, wanted, cut.splits, s);
}

}  // namespace sadmm
