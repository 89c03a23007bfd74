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
#include "tgemm_dev.cuh"

namespace sadmm {

namespace {

constexpr int kThreads = 192;
constexpr int kMaxStages = 8;
constexpr int kMaxAccCols = 128;  // accumulator columns of a CTA (fp32 sums: 64 KB when cut over a cluster)

template <bool SWAP, bool GATED>
__global__ void __launch_bounds__(kThreads, 2)
    k_tgemm(const __grid_constant__ TgMaps maps, const __grid_constant__ TgArgs a)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    __shared__ uint64_t full[kMaxStages], empty[kMaxStages], acc_full, drain;
    __shared__ uint32_t tmem_holder;
    __shared__ volatile int abort_flag;
    __shared__ float s_bias[2 * kMaxAccCols];
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
        int s = 0;
        uint32_t phase = 0;
        for (int i = 0; i < nk; ++i) {
            if (!mbar_wait_warp(&full[s], phase, &abort_flag, a.status)) { ok = false; break; }
            tc_fence_after();
            const uint32_t st = smem_u32(smem + (size_t)s * a.stage_bytes);
            const uint64_t pd = sdesc(st, p.p_kmajor), qd = sdesc(st + a.q_off, p.q_kmajor);
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
                mma_bf16_ss_elect(tmem, pd + kk * pstep, qd + kk * qstep, p.idesc, (i | kk) != 0);
                if (GATED && SWAP)
                    mma_bf16_ss_elect(tmem + a.bn, pd + (kPTile >> 4) + kk * pstep, qd + kk * qstep, p.idesc,
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
                s_bias[j] = a.bias && c < p.n ? a.bias[c] : 0.0f;
                if (GATED) s_bias[kMaxAccCols + j] = a.bias2 && c < p.n ? a.bias2[c] : 0.0f;
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
        const long long prow = (long long)row0 + trow;
        const uint32_t base = smem_u32(part) + 4u * (uint32_t)trow;
        if (SWAP) {
            const float b = a.bias && prow < p.n ? a.bias[prow] : 0.0f;
            const float b2 = GATED && a.bias2 && prow < p.n ? a.bias2[prow] : 0.0f;
            const int cols = (int)min((long long)a.bn, p.m - col0);
            if (a.splits > 1) {
                for (int c = (int)rank; c < cols; c += a.splits) {
                    float v = 0.0f, w = 0.0f;
                    for (int s = 0; s < a.splits; ++s) {
                        const uint32_t peer = map_rank(base, (uint32_t)s);
                        v += ld_cluster_f32(peer + (uint32_t)c * 512u);
                        if (GATED) w += ld_cluster_f32(peer + (uint32_t)(a.bn + c) * 512u);
                    }
                    if (prow < p.n) finish1<GATED>(a, p, col0 + c, prow, v, w, b, b2);
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
                        if (c0 + j < cols && prow < p.n)
                            finish1<GATED>(a, p, col0 + c0 + j, prow, nk > 0 ? __uint_as_float(rv[j]) : 0.0f,
                                           GATED && nk > 0 ? __uint_as_float(rw[j]) : 0.0f, b, b2);
                }
            }
        } else {
            const int cols = (int)min((long long)a.bn, p.n - col0);
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
                if (prow < p.m) finish16<GATED>(a, p, prow, col0 + c, v, w, s_bias + c, s_bias + kMaxAccCols + c);
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

template <bool SWAP, bool GATED>
sadmm_status run(const TgMaps& maps, const TgArgs& a, size_t smem, cudaStream_t s)
{
    static bool configured[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return SADMM_ECUDA;
    auto kern = k_tgemm<SWAP, GATED>;
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

// CTAs that each contraction is cut over.  Few tiles: 2, 4 or 8 (of at least
// four steps each); and an fp32 output's anyway, so that no sum inside the
// tensor cores passes 2048 elements where 8 CTAs are enough for that (over 8192
// elements one sum was 1.0e-6 off, four added up in fp32 0.25e-6).
int cuts(const TgProblem* t, int count)
{
    const int bn = tile_width(t, count), sm = device_sm_count();
    long long tiles = 0, nk = 0, longest = 0;
    for (int i = 0; i < count; ++i) {
        const long long steps = steps_of(t[i]);
        const bool swap = swapped(t[i]);
        tiles += ((swap ? t[i].n : t[i].m) + 127) / 128 * (((swap ? t[i].m : t[i].n) + bn - 1) / bn);
        if (steps > nk) nk = steps;
        if (t[i].y.dt == SADMM_FP32 && steps > longest) longest = steps;
    }
    int splits = 1;
    while (splits < 8 && ((tiles * splits * 2 <= 2 * sm && nk >= 8 * splits) || longest > 32 * splits)) splits *= 2;
    return splits;
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
    for (int i = 0; i < count; ++i) {
        a.prod[i].steps = (a.prod[i].nk + splits - 1) / splits;
        if (a.prod[i].steps > steps) steps = a.prod[i].steps;
    }
    a.acc_cols = (uint32_t)(gated ? 2 * bn : bn);
    uint32_t cols = 32;
    while (cols < a.acc_cols) cols <<= 1;
    a.tmem_cols = cols;
    a.q_off = gated && swap ? 2 * kPTile : kPTile;
    a.stage_bytes = a.q_off + (uint32_t)n_mma * 128u;
    // two CTAs an SM: one's epilogue beside the other's products
    a.stages = (int)(108 * 1024 / a.stage_bytes);
    if (a.stages > kMaxStages) a.stages = kMaxStages;
    if (a.stages > steps) a.stages = steps;
    size_t smem = (size_t)a.stages * a.stage_bytes;
    if (splits > 1 && smem < (size_t)a.acc_cols * 512) smem = (size_t)a.acc_cols * 512;
    smem += 1024;
    if (gated) return swap ? run<true, true>(maps, a, smem, s) : run<false, true>(maps, a, smem, s);
    return swap ? run<true, false>(maps, a, smem, s) : run<false, false>(maps, a, smem, s);
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
    if (!swapped(all[0])) {
        const bool gated = all->mode == kTgGated;
        const TgPairChoice c = choose_tgemm_pair(all, count);
        long long work = 0;  // steps of 128-row tiles
        for (int i = 0; i < count; ++i)
            work += (all[i].m + 127) / 128 * ((all[i].n + (gated ? 63 : 127)) / (gated ? 64 : 128)) * steps_of(all[i]);
        if (c.cycles < work * 560 / device_sm_count() + 6000)
            return launch_tgemm_pair(t, wanted, choose_tgemm_pair(t, wanted).bn, s);
    }
    return launch_tiles(t, wanted, cuts(all, count), s);
}

}  // namespace sadmm
