// tgemm_pair.cu -- the feed-forward products of large matrices: a persistent
// kernel of CTA pairs, one 256 x bn tile at a time (bn at most 256).
//
// The pair shares each MMA (tcgen05.mma.cta_group::2, M 256): a CTA holds 128
// of the tile's rows and half of its columns' operand, so that every byte in
// shared memory feeds twice the products of a single CTA's tile; the gated
// pair's second CTA holds the columns of Wu where the first has those of Wg.
// Per CTA, ten warps:
//   warp 0      TMA producer, 192 KB of stages of 64 contraction elements
//   warp 1      TMEM allocator; in the pair's first CTA, issuer of the MMAs
//   warps 2-9   epilogue: TMEM lane = tile row, each half of the warps takes
//               half of the columns
// Two accumulators in TMEM: a tile's epilogue runs beside the next tile's
// products.  fp32 outputs of long contractions (LONG) are added up in registers
// over accumulators of kLongSteps steps each (8192 x 5120 -> 2048's gradients take
// 238 us with sums of 2048 terms, 250 to 255 over boxes with these of 768, 254 with
// sums of 512).
//
// Bound by the tensor pipe: 8192 x 4096 -> 2 x 10240 (the gated pair, both
// pre-activations kept) in 770 to 893 us over boxes, 1780 to 1540 TFLOP/s, where
// the power limit sets the clock (a library product alone: 1946 for a moment,
// 1740 sustained).  Smaller products lose their last round of tiles: 4096^3 in
// 86 us (1600 TFLOP/s) with four rounds of 224 columns, 104 to 106 with GELU, z kept
// and inputs that change between calls.
#include "tgemm_dev.cuh"

namespace sadmm {
namespace {

constexpr int kPairThreads = 320;
constexpr int kPairStages = 10;          // at most
constexpr int kPairSmem = 192 * 1024;    // of stages

// ------------------------------------------------------------- device PTX --

SADMM_DEV void tmem_alloc2(uint32_t* dst, uint32_t ncols)
{
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(dst)), "r"(ncols)
                 : "memory");
}
SADMM_DEV void tmem_relinquish2() { asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory"); }
SADMM_DEV void tmem_dealloc2(uint32_t taddr, uint32_t ncols)
{
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(ncols) : "memory");
}

// One box into this CTA's shared memory; the bytes are counted on `bar`, a
// cluster address in either CTA of the pair.
SADMM_DEV void tma_load_pair(void* dst, const void* tmap, uint32_t bar, int c0, int c1)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2"
        " [%0], [%1, {%3, %4}], [%2];" ::"r"(smem_u32(dst)),
        "l"(tmap), "r"(bar), "r"(c0), "r"(c1)
        : "memory");
}

// As mma_bf16_ss_elect, over the pair's shared memory and TMEM.
SADMM_DEV void mma_pair_elect(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p, e;\n\t.reg .b32 l;\n\telect.sync l|e, 0xffffffff;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "@e tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
        "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate));
}

// Arrives on the barrier at this place in both CTAs once the MMAs so far are done.
SADMM_DEV void commit_pair_elect(uint64_t* bar)
{
    asm volatile(
        "{\n\t.reg .pred e;\n\t.reg .b32 l;\n\t.reg .b16 m;\n\telect.sync l|e, 0xffffffff;\n\tmov.b16 m, 3;\n\t"
        "@e tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], m;\n\t}" ::"r"(
            smem_u32(bar))
        : "memory");
}
SADMM_DEV void commit_own_elect(uint64_t* bar)
{
    asm volatile(
        "{\n\t.reg .pred e;\n\t.reg .b32 l;\n\telect.sync l|e, 0xffffffff;\n\t"
        "@e tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(smem_u32(bar))
        : "memory");
}

// Arrival on a barrier of either CTA.
SADMM_DEV void mbar_arrive_cluster(uint32_t bar)
{
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

// ------------------------------------------------------------------ kernel --

// The k-th tile of pair i of n: the tiles of the longest contraction (the first
// `long_tiles`) in turn; the pairs that have one less of those catch up with
// `catch_up` of the others first, which then also go in turn, from pair
// `shift` on.  -1: no more.
SADMM_DEV int tile_of(const TgArgs& a, int i, int n, int k)
{
    const int rem = a.long_tiles % n, mine = a.long_tiles / n + (i < rem);
    if (k < mine) return k * n + i;
    k -= mine;
    const int ahead = a.catch_up * (n - rem);
    int t;
    if (i >= rem && k < a.catch_up) {
        t = k * (n - rem) + i - rem;
    } else {
        if (i >= rem) k -= a.catch_up;
        int at = i - a.shift;
        if (at < 0) at += n;
        t = ahead + k * n + at;
    }
    t += a.long_tiles;
    return t < a.tiles ? t : -1;
}

// Product, row tile and column tile of tile t, eight row tiles at a time so
// that the tiles in flight share their operands in L2.
struct Place {
    int prod, mt, nt;
};
SADMM_DEV Place place(const TgArgs& a, int t)
{
    constexpr int kGroup = 8;
    Place p;
    p.prod = 0;
    while (p.prod + 1 < a.products && t >= a.prod[p.prod + 1].first) ++p.prod;
    const TgProduct& d = a.prod[p.prod];
    t -= d.first;
    const int g = t / (kGroup * d.q_tiles);
    const int rows = min(kGroup, d.p_tiles - g * kGroup);
    t -= g * kGroup * d.q_tiles;
    p.nt = t / rows;
    p.mt = g * kGroup + t - p.nt * rows;
    return p;
}

template <bool GATED, bool LONG>
__global__ void __launch_bounds__(kPairThreads, 1)
    k_tgemm_pair(const __grid_constant__ TgMaps maps, const __grid_constant__ TgArgs a)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    __shared__ uint64_t full[kPairStages], empty[kPairStages], acc_full[2], acc_empty[2], drain;
    __shared__ uint32_t tmem_holder;
    __shared__ volatile int abort_flag;
    // each epilogue warp's columns (gated: of g, then of u): its own copy, so that no warp waits for another, which
    // may have given up its wait for an accumulator and left the loop over tiles
    __shared__ __align__(16) float s_bias[8][128];
    // warp-uniform to the compiler, which keeps the issue loop's descriptors in uniform registers: an MMA and its
    // stage then cost less to issue than to run (4096^3: 86.5 -> 83.7 us)
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    const int me = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    const int half = a.bn >> 1;

    if (threadIdx.x == 0) {
        for (int s = 0; s < a.stages; ++s) {
            mbar_init(&full[s], 1);
            mbar_init(&empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&acc_full[b], 1);
            mbar_init(&acc_empty[b], 16);  // eight epilogue warps of either CTA
        }
        mbar_init(&drain, 1);
        abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == 1) {
        tmem_alloc2(&tmem_holder, 512);
        tmem_relinquish2();
    }
    pdl_wait();  // nothing above reads global memory
    tc_fence_before();
    __syncthreads();
    cluster_sync();  // barriers and TMEM of both CTAs are there
    tc_fence_after();
    const uint32_t tmem = tmem_holder;

    if (warp == 0) {
        if (lane == 0) {
            int s = 0;
            uint32_t phase = 0;
            bool ok = true;
            for (int i = 0, t; ok && (t = tile_of(a, me, pairs, i)) >= 0; ++i) {
                const Place pl = place(a, t);
                const TgProduct& p = a.prod[pl.prod];
                const uint32_t q_bytes = p.q_kmajor ? (uint32_t)half * 128u : (uint32_t)((half + 63) / 64) * kBox;
                const uint32_t bytes = 2u * (kPTile + q_bytes);
                const int row0 = pl.mt * 256 + (int)rank * 128;
                const int col0 = GATED ? pl.nt * half : pl.nt * a.bn + (int)rank * half;
                const CUtensorMap *p0 = &maps.map[p.pm], *q0 = &maps.map[p.qm + (GATED && rank)];
                for (int k = 0; k < p.nk; ++k) {
                    if (!mbar_wait(&empty[s], phase ^ 1u, &abort_flag, a.status)) { ok = false; break; }
                    if (rank == 0) mbar_arrive_expect_tx(&full[s], bytes);
                    const uint32_t bar = map_rank(smem_u32(&full[s]), 0);
                    const int second = k >= p.nk0;  // of a sum
                    const CUtensorMap *pm = p0 + second, *qm = q0 + second;
                    const int kc = (second ? k - p.nk0 : k) * 64;
                    uint8_t* sp = smem + (size_t)s * a.stage_bytes;
                    uint8_t* sq = sp + kPTile;
                    if (p.p_kmajor) {
                        tma_load_pair(sp, pm, bar, kc, row0);
                    } else {
                        tma_load_pair(sp, pm, bar, row0, kc);
                        tma_load_pair(sp + kBox, pm, bar, row0 + 64, kc);
                    }
                    if (p.q_kmajor) {
                        tma_load_pair(sq, qm, bar, kc, col0);
                    } else {
                        tma_load_pair(sq, qm, bar, col0, kc);
                        if (half > 64) tma_load_pair(sq + kBox, qm, bar, col0 + 64, kc);
                    }
                    if (++s == a.stages) { s = 0; phase ^= 1u; }
                }
            }
            // every stage filled has been read before the CTA retires; after a failure, time for the copies to land
            for (int i = 0; i < a.stages && ok; ++i) {
                ok = mbar_wait(&empty[s], phase ^ 1u, &abort_flag, a.status);
                if (++s == a.stages) { s = 0; phase ^= 1u; }
            }
            if (!ok) {
                const unsigned long long t0 = globaltimer();
                while (globaltimer() - t0 < 10000000ull) {}
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (rank == 0) {
            int s = 0, buf = 0;
            uint32_t phase = 0, bphase = 0;
            bool ok = true;
            for (int i = 0, t; ok && (t = tile_of(a, me, pairs, i)) >= 0; ++i) {
                const TgProduct& p = a.prod[place(a, t).prod];
                const uint32_t pstep = p.p_kmajor ? 2u : 128u, qstep = p.q_kmajor ? 2u : 128u;
                const int p_kmajor = p.p_kmajor, q_kmajor = p.q_kmajor, nk = p.nk;
                const uint32_t idesc = p.idesc;
                for (int k = 0; k < nk && ok;) {
                    const int k1 = LONG ? min(k + p.acc_steps, nk) : nk;
                    if (!mbar_wait_warp(&acc_empty[buf], bphase ^ 1u, &abort_flag, a.status)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t d = tmem + (uint32_t)buf * 256u;
                    for (bool more = false; k < k1; ++k) {
                        if (!mbar_wait_warp(&full[s], phase, &abort_flag, a.status)) { ok = false; break; }
                        tc_fence_after();
                        const uint32_t st = smem_u32(smem + (size_t)s * a.stage_bytes);
                        const uint64_t pd = sdesc(st, p_kmajor), qd = sdesc(st + kPTile, q_kmajor);
#pragma unroll
                        for (int kk = 0; kk < 4; ++kk) {
                            mma_pair_elect(d, pd + kk * pstep, qd + kk * qstep, idesc, more || kk != 0);
                        }
                        more = true;
                        commit_pair_elect(&empty[s]);
                        if (++s == a.stages) { s = 0; phase ^= 1u; }
                    }
                    if (ok) commit_pair_elect(&acc_full[buf]);
                    if (++buf == 2) { buf = 0; bphase ^= 1u; }
                }
            }
            commit_own_elect(&drain);
            if (lane == 0) {
                const unsigned long long t0 = globaltimer();
                while (!mbar_try_wait(&drain, 0) && globaltimer() - t0 < kWaitLimitNs) {}
            }
        }
        __syncwarp();
    } else {
        const int q = warp & 3, part = (warp - 2) >> 2;
        const uint32_t taddr = tmem + ((uint32_t)(q * 32) << 16);
        const int cols = GATED ? half : a.bn;        // output columns of a tile
        const int c_begin = part * (cols >> 1), c_end = c_begin + (cols >> 1);
        float* sb = s_bias[warp - 2];
        int buf = 0;
        uint32_t bphase = 0;
        bool ok = true;
        for (int i = 0, t; ok && (t = tile_of(a, me, pairs, i)) >= 0; ++i) {
            const Place pl = place(a, t);
            const TgProduct& p = a.prod[pl.prod];
            const long long row = (long long)pl.mt * 256 + rank * 128 + q * 32 + lane;
            const long long col0 = (long long)pl.nt * cols;
            const int live = (int)min((long long)cols, p.n - col0);  // columns inside the output
            if (a.bias || a.bias2) {
                __syncwarp();  // the last tile's have been read
#pragma unroll
                for (int j = lane; j < 128; j += 32) {
                    const int at = GATED ? j & 63 : j, c = c_begin + at;
                    const float* from = GATED && j >= 64 ? a.bias2 : a.bias;
                    sb[j] = from && c < c_end && c < live ? from[col0 + c] : 0.0f;
                }
                __syncwarp();
            }
            float sum[LONG ? 8 : 1][16];
            for (int k = 0; k < p.nk; k += LONG ? p.acc_steps : p.nk) {
                ok = __all_sync(0xffffffffu, mbar_wait(&acc_full[buf], bphase, &abort_flag, a.status));
                if (!ok) break;
                tc_fence_after();
                const uint32_t acc = taddr + (uint32_t)buf * 256u;
                if (LONG) {
                    const bool last = k + p.acc_steps >= p.nk;
#pragma unroll
                    for (int h = 0; h < 8; ++h) {
                        const int c = c_begin + 16 * h;
                        if (c < c_end) {
                            uint32_t r[16];
                            tmem_ld_32x32b_x16(acc + (uint32_t)c, r);
                            tmem_ld_wait();
#pragma unroll
                            for (int j = 0; j < 16; ++j)
                                sum[h][j] = k ? sum[h][j] + __uint_as_float(r[j]) : __uint_as_float(r[j]);
                            if (last && row < p.m && c < live) {
                                float w[16];
                                finish16<false>(a, p, row, col0 + c, sum[h], w, sb + 16 * h, sb);
                            }
                        }
                    }
                } else {
                    for (int c = c_begin; c < c_end && c < live; c += 16) {
                        uint32_t rv[16], rw[16];
                        tmem_ld_32x32b_x16(acc + (uint32_t)c, rv);
                        if (GATED) tmem_ld_32x32b_x16(acc + (uint32_t)(half + c), rw);
                        tmem_ld_wait();
                        float v[16], w[16];
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            v[j] = __uint_as_float(rv[j]);
                            w[j] = GATED ? __uint_as_float(rw[j]) : 0.0f;
                        }
                        const float* b = sb + c - c_begin;
                        if (row < p.m) finish16<GATED>(a, p, row, col0 + c, v, w, b, b + 64);
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(map_rank(smem_u32(&acc_empty[buf]), 0));
                if (++buf == 2) { buf = 0; bphase ^= 1u; }
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();  // neither CTA's barriers nor TMEM are in use any more
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc2(tmem, 512);
    }
}

template <bool GATED, bool LONG>
sadmm_status run(const TgMaps& maps, const TgArgs& a, int ctas, cudaStream_t s)
{
    static bool configured[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return SADMM_ECUDA;
    constexpr int smem = kPairSmem + 1024;
    auto kern = k_tgemm_pair<GATED, LONG>;
    if (!configured[dev]) {
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess)
            return SADMM_ECUDA;
        configured[dev] = true;
    }
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 2;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(kPairThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kern, maps, a) == cudaSuccess ? SADMM_OK : SADMM_ECUDA;
}

}  // namespace

namespace {

// The pairs' schedule of tiles of two costs: `a` tiles of ca steps, then `b` of
// cb.  Gives the number of the latter that pairs with one long tile less take
// to catch up, and the steps of the busiest pair.
struct Schedule {
    int catch_up, shift;
    long long steps;
};
Schedule schedule(long long a, long long ca, long long b, long long cb, long long pairs)
{
    const long long rem = a % pairs, base = a / pairs * ca;
    Schedule best = {0, 0, 0};
    if (!b) {
        best.steps = base + (rem ? ca : 0);
        return best;
    }
    const long long d0 = rem ? ca / cb : 0;
    for (long long d = d0; d <= d0 + (rem ? 1 : 0); ++d) {
        long long rest = b - d * (pairs - rem);
        if (rest < 0) rest = 0;
        const long long rounds = rest / pairs, left = rest - rounds * pairs;
        const long long heavy = rem ? base + ca : 0, light = base + d * cb;
        // the last round starts at the lighter group
        const bool light_first = !rem || light <= heavy;
        const long long first = light_first ? pairs - rem : rem;
        const long long l = light + (rounds + (light_first ? left > 0 : left > first)) * cb;
        const long long h = rem ? heavy + (rounds + (light_first ? left > first : left > 0)) * cb : 0;
        const long long most = l > h ? l : h;
        if (!best.steps || most < best.steps) best = {(int)d, light_first ? (int)rem : 0, most};
    }
    return best;
}

long long tiles_of(const TgProblem& t, int bn)
{
    const int cols = t.mode == kTgGated ? bn / 2 : bn;
    return (t.m + 255) / 256 * ((t.n + cols - 1) / cols);
}

// Products of the longest contraction first (stable); those after it are of
// one length here (the two weight gradients of a gated pair), or are taken as
// the longest of theirs.
Schedule schedule_of(const TgProblem* const* t, int count, int bn, long long pairs)
{
    long long b = 0, cb = 0;
    int i = 1;
    long long a = tiles_of(*t[0], bn);
    for (; i < count && steps_of(*t[i]) == steps_of(*t[0]); ++i) a += tiles_of(*t[i], bn);
    for (; i < count; ++i) {
        b += tiles_of(*t[i], bn);
        if (steps_of(*t[i]) > cb) cb = steps_of(*t[i]);
    }
    return schedule(a, steps_of(*t[0]), b, cb, pairs);
}

void by_length(const TgProblem* t, int count, const TgProblem** order)
{
    for (int i = 0; i < count; ++i) {
        int j = i;
        for (; j > 0 && steps_of(*order[j - 1]) < steps_of(t[i]); --j) order[j] = order[j - 1];
        order[j] = &t[i];
    }
}

}  // namespace

// The tile width whose busiest pair costs least.  Measured: a step of 64
// contraction elements takes 0.34 us at 256 columns (0.27 us of MMAs) and hardly
// less below, because issuing a stage takes about 470 cycles; beside its steps a
// launch takes 5.4 us at 256 columns and 4.6 at 64, most of it the last
// epilogue (1024^3: 10.8 us at 256, 10.0 at 128, 9.5 at 64).  Widths are
// multiples of 64, or of 32 where the columns' operand is contiguous along the
// contraction (no whole 64-row boxes) and not a gated pair's.
TgPairChoice choose_tgemm_pair(const TgProblem* t, int count)
{
    const TgProblem* order[kTgProducts];
    by_length(t, count, order);
    int grain = t->mode == kTgGated ? 64 : 32;
    for (int i = 0; i < count; ++i)
        if (!t[i].b[0].kmajor) grain = 64;
    TgPairChoice best = {0, 0};
    for (int bn = 256; bn >= 64; bn -= grain) {
        const Schedule w = schedule_of(order, count, bn, device_sm_count() / 2);
        const long long time = w.steps * (28 + bn / 48 + (bn == 256)) + 430 + bn * 2 / 5;
        if (!best.bn || time < best.time) best = {bn, time};
    }
    return best;
}

sadmm_status launch_tgemm_pair(const TgProblem* problems, int count, int bn, cudaStream_t s)
{
    const TgProblem* order[kTgProducts];
    by_length(problems, count, order);
    TgProblem t[kTgProducts];
    for (int i = 0; i < count; ++i) t[i] = *order[i];
    const bool gated = t->mode == kTgGated;
    TgArgs a;
    TgMaps maps;
    fill_common(a, t, count);
    a.bn = bn;
    const long long pairs = device_sm_count() / 2;
    long long tiles = 0;
    bool lng = false, boxes = false;
    int next = 0;
    for (int i = 0; i < count; ++i) {
        TgProduct& p = a.prod[i];
        const int cols = gated ? bn / 2 : bn;
        p.p_tiles = (int)((p.m + 255) / 256);
        p.q_tiles = (int)((p.n + cols - 1) / cols);
        p.first = (int)tiles;
        tiles += (long long)p.p_tiles * p.q_tiles;
        if (tiles > 0x0fffffffll) return SADMM_EUNSUPPORTED;
        if (p.nk == a.prod[0].nk) a.long_tiles = (int)tiles;
        if (!encode_product(maps, next, p, t[i], false, 128, bn / 2, i ? &a.prod[i - 1] : nullptr,
                            i ? &t[i - 1] : nullptr))
            return SADMM_ECUDA;
        p.idesc = idesc_bf16_f32(256, bn) | (p.p_kmajor ? 0u : 1u << 15) | (p.q_kmajor ? 0u : 1u << 16);
        p.acc_steps = p.nk;
        if (!gated && !p.y.bf16 && p.nk > kLongSteps) {
            p.acc_steps = kLongSteps;
            lng = true;
        }
        boxes = boxes || !p.q_kmajor;
    }
    a.tiles = (int)tiles;
    const Schedule w = schedule_of(order, count, bn, pairs);
    a.catch_up = w.catch_up;
    a.shift = w.shift;
    a.stage_bytes = kPTile + (uint32_t)(boxes ? (bn / 2 + 63) / 64 * kBox : bn / 2 * 128);
    a.stages = kPairSmem / (int)a.stage_bytes;
    if (a.stages > kPairStages) a.stages = kPairStages;
    const int ctas = 2 * (int)(tiles < pairs ? tiles : pairs);
    if (gated) return run<true, false>(maps, a, ctas, s);
    return lng ? run<false, true>(maps, a, ctas, s) : run<false, false>(maps, a, ctas, s);
}

}  // namespace sadmm
