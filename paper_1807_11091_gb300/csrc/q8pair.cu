// q8pair.cu -- products of large 8-bit matrices: a persistent kernel of CTA pairs,
// one tile of 256 rows by 256 columns at a time (gated: 128 of either weight's; where
// the columns' scales are single rows', as a weight gradient's, 512 by 128).
//
// The pair shares each MMA (tcgen05.mma.cta_group::2, M 256): a CTA holds 128 of
// the tile's rows and half of its columns' operand (gated: the second CTA Wu's
// columns where the first has Wg's).  A block of 128 of the contraction is one stage
// of shared memory and one accumulator in TMEM, of which there are two; the
// epilogue's warps multiply it by its scales and add it to fp32 sums in registers
// while the next block's products run.  Per CTA, twelve warps:
//   warp 0      TMA producer
//   warp 1      TMEM allocator; in the pair's first CTA, issuer of the MMAs
//   warps 2, 3  the rows' and the columns' scales, by cp.async into a ring of blocks (in
//               the sums' warps the addresses alone took 720 cycles a block, of 512)
//   warps 4-11  sums and output: TMEM lane = tile row, each half of the warps
//               takes half of the columns, 128 sums a thread
//
// Measured (us, of the operations at twice the 1859 TFLOP/s of bf16): 8192 x 4096 -> 4096 with
// GELU 160 (74), the gated pair 8192 x 4096 -> 2 x 10240 with g and u kept 667 (370), gradients of
// 8192 x 5120 -> 2048 with the quantiser 252 (92).  Bound by the accumulators' way to the sums and
// back: a block takes 0.41 us where its MMAs take 0.27, with single rows' scales 0.75; beside it
// a tile's output is not hidden, some 4 us and with GELU 8.
#include <string.h>

#include <initializer_list>

#include "q8.cuh"
#include "tgemm_dev.cuh"

namespace sadmm {
namespace {

constexpr int kThreads = 384;
// Registers of a thread: 168 at launch (384 of them fill an SM), then these.
template <bool VEC>
struct Regs {
    static constexpr int few = VEC ? 56 : 40, many = VEC ? 224 : 232;
    static_assert(128 * few + 256 * many <= 384 * 168, "more registers than the block was launched with");
};
constexpr int kStages = 4;
constexpr uint32_t kHalfBytes = 128 * kQBlock;        // 128 rows of one block
// A tile is 256 rows by 256 columns; with VEC (the columns' scales are single rows') 512 by 128, so
// that a thread has two rows and a column's scale is read half as often.
template <bool VEC>
struct Tile {
    static constexpr int rows = VEC ? 512 : 256, cols = VEC ? 128 : 256;
    static constexpr uint32_t p_bytes = (VEC ? 2 : 1) * kHalfBytes;            // a CTA's part of a stage: of the rows,
    static constexpr uint32_t bytes = p_bytes + (VEC ? kHalfBytes / 2 : kHalfBytes);  // and of the columns too
    static constexpr int boxes = VEC ? 1 : 2;                                  // of a warp
    // the ring of scales: [block][row of the CTA], then [block][column], or where 128 columns have one [half][block]
    static constexpr int own = VEC ? 256 : 128, columns = 4 * own;
};
constexpr int kProducts = 2, kOperands = 4;            // of a launch, and maps of its operands
constexpr int kBoxBytes = 4096;                       // 32 output rows of 128 bytes on their way out
constexpr int kSlots = 3;                             // places of the ring of scales, four blocks each
constexpr int kSlotFloats = 4 * 384;

struct Scales {
    const float* s;
    long long s_row, s_block, rows;
    int shift;
};

struct Product {
    TgProduct t;           // y, m, n, first, p_tiles, q_tiles, nk0, nk are used
    Scales ps[2], qs[2];   // of both summands; gated: qs of Wg and Wu
    int sum;
    int pm, qm;            // maps; the second summand's (gated: Wu's) follow
    int ym;                // map of y, -1: its rows do not start on 16-byte boundaries
};

struct Maps {
    CUtensorMap map[kOperands + kProducts + 2];
};

struct Args {
    Product prod[kProducts];
    TgArgs t;              // products, tiles, res, z, u, bias, bias2, act, status are used
    sadmm_q8_out y8;
    int zm, um;            // maps of z and u, as ym
    uint32_t idesc;
};

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
SADMM_DEV void tma_load_pair(void* dst, const void* tmap, uint32_t bar, int c0, int c1)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2"
        " [%0], [%1, {%3, %4}], [%2];" ::"r"(smem_u32(dst)),
        "l"(tmap), "r"(bar), "r"(c0), "r"(c1)
        : "memory");
}
SADMM_DEV void mma_f8_pair_elect(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p, e;\n\t.reg .b32 l;\n\telect.sync l|e, 0xffffffff;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "@e tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
        "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate));
}
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
// Arrival on a barrier of either CTA.  Its order is that of the CTA: what it hands over
// is TMEM that has been read, and a release to the cluster waits for every copy in
// flight (2500 cycles a block of the contraction, where its products take 512).
SADMM_DEV void mbar_arrive_either(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

// Four bytes into shared memory, zero where `in` is false.
SADMM_DEV void cp_async4(float* dst, const float* src, bool in)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(in ? 4 : 0) : "memory");
}
// 16 bytes, of which `bytes` are there and the others zero.
SADMM_DEV void cp_async16(float* dst, const float* src, int bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(bytes) : "memory");
}
// Arrives on the barrier once this thread's copies so far have landed.
SADMM_DEV void cp_async_arrive(uint64_t* bar)
{
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
SADMM_DEV void cp_async_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// ------------------------------------------------------------------ kernel --

// Product, row tile and column tile of tile t, eight row tiles at a time so
// that the tiles in flight share their operands in L2.
struct Place {
    int prod, mt, nt;
};
SADMM_DEV Place place(const Args& a, int t)
{
    constexpr int kGroup = 8;
    Place p;
    p.prod = 0;
    while (p.prod + 1 < a.t.products && t >= a.prod[p.prod + 1].t.first) ++p.prod;
    const TgProduct& d = a.prod[p.prod].t;
    t -= d.first;
    const int g = t / (kGroup * d.q_tiles);
    const int rows = min(kGroup, d.p_tiles - g * kGroup);
    t -= g * kGroup * d.q_tiles;
    p.nt = t / rows;
    p.mt = g * kGroup + t - p.nt * rows;
    return p;
}

// The k-th tile of pair `me` of n: in turn, every other round backwards, so that the
// pairs with the longer tiles of one round have the shorter ones of the next.
SADMM_DEV int tile_of(const Args& a, int me, int n, int k)
{
    const int t = k * n + ((k & 1) ? n - 1 - me : me);
    return t < a.t.tiles ? t : -1;
}

// The ring of scales, as the warps that fill it see it.
struct Ring {
    float* slots;
    uint64_t *full, *empty;
    volatile int* abort_flag;
    int* status;
    int s;
    uint32_t phase;
    SADMM_DEV bool wait(int k) { return (k & 3) != 0 || mbar_wait_warp(&empty[s], phase ^ 1u, abort_flag, status); }
    SADMM_DEV float* slot(int k, int next) { return slots + s * kSlotFloats + (k & 3) * next; }
    SADMM_DEV void done(int k, int nk)
    {
        if ((k & 3) != 3 && k + 1 != nk) return;
        cp_async_arrive(&full[s]);
        if (++s == kSlots) { s = 0; phase ^= 1u; }
    }
    // N scales a lane of each of the blocks k0 .. k1-1 of a tile's nk: those of the rows r0, r0 + 32, ... of c (r0 a
    // multiple of 32 and the lane).  They lie `apart` places apart from `at` on, `next` places further for the next of a
    // place's four blocks.
    template <int N>
    SADMM_DEV bool fill(int k0, int k1, int nk, int at, int apart, int next, const Scales& c, long long r0)
    {
        // (eight: the second four are 256 rows on)
        auto row = [&](int j) { return j * 32 + (N == 8 && j >= 4 ? 128 : 0); };
        uint32_t in = 0;
#pragma unroll
        for (int j = 0; j < N; ++j) in |= (r0 + row(j) < c.rows ? 1u : 0u) << j;
        const float* from = c.s + ((in & 1u ? r0 : 0) >> c.shift) * c.s_row;
        const long long more = c.s_row * (c.shift ? 1 : 32);  // a scale further
        const long long step = c.s_block;
        const int same = c.shift ? 2 : 0;                     // 1 << same places of 32 rows share one
        for (int k = k0; k < k1; ++k) {
            if (!wait(k)) return false;
            float* to = slot(k, next) + at;
            if (N > 1 || (threadIdx.x & 31) < 2) {
#pragma unroll
                for (int j = 0; j < N; ++j)
                    cp_async4(to + j * apart, in >> j & 1u ? from + (row(j) / 32 >> same) * more : from, in >> j & 1u);
            }
            from += step;
            done(k, nk);
        }
        return true;
    }
    // Whether 128 scales from a multiple of 128 on are neighbours and start on a 16-byte boundary.
    static SADMM_DEV bool wide(const Scales& c)
    {
        return c.shift == 0 && c.s_row == 1 && (c.s_block & 3) == 0 && (reinterpret_cast<uintptr_t>(c.s) & 15) == 0;
    }
    // The same for N times 128 such, 256 rows apart, from row r0 on: four a lane.  (One by one, two warps could not
    // fetch the 384 of a block while its products run: 0.86 us a block.)
    template <int N>
    SADMM_DEV bool fill_wide(int k0, int k1, int nk, int at, int next, const Scales& c, long long r0)
    {
        const int lane = threadIdx.x & 31;
        int bytes[N];
#pragma unroll
        for (int j = 0; j < N; ++j) bytes[j] = (int)max(0ll, min(4ll, c.rows - r0 - j * 256 - lane * 4)) * 4;
        const float* from = c.s + (bytes[0] ? r0 + lane * 4 : 0);
        const long long step = c.s_block;
        for (int k = k0; k < k1; ++k) {
            if (!wait(k)) return false;
            float* to = slot(k, next) + at + lane * 4;
#pragma unroll
            for (int j = 0; j < N; ++j) cp_async16(to + j * 128, bytes[j] ? from + j * 256 : from, bytes[j]);
            from += step;
            done(k, nk);
        }
        return true;
    }
};

// A warp's two boxes of 32 rows x 128 bytes (64 bf16 or 32 fp32 columns) in shared memory, from
// which the tensor-memory accelerator writes them out while the next tile is added up, and
// leaves out what lies past the matrix.  (Stored by the threads themselves, 32 rows of 32
// bytes at a time, and without WHOLE: 8192 x 4096 -> 4096 162 us instead of 158.)
struct Boxes {
    uint8_t* mem;
    int lane;
    // Whether box b may be written again: all stores but the last `left` have been read.
    template <int LEFT>
    SADMM_DEV void free()
    {
        if (lane == 0) asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(LEFT) : "memory");
        __syncwarp();
    }
    // The lane's row: 16 values to the piece-th of four (bf16) or two (fp32) pieces of the box.
    SADMM_DEV void put(int b, int piece, bool bf16, const float (&v)[16])
    {
        uint8_t* row = mem + b * kBoxBytes + lane * 128;
        if (bf16) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
                *reinterpret_cast<uint4*>(row + (((piece * 2 + h) ^ (lane & 7)) << 4)) =
                    make_uint4(pack_bf16(v[8 * h], v[8 * h + 1]), pack_bf16(v[8 * h + 2], v[8 * h + 3]),
                               pack_bf16(v[8 * h + 4], v[8 * h + 5]), pack_bf16(v[8 * h + 6], v[8 * h + 7]));
        } else {
#pragma unroll
            for (int h = 0; h < 4; ++h)
                *reinterpret_cast<float4*>(row + (((piece * 4 + h) ^ (lane & 7)) << 4)) =
                    make_float4(v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]);
        }
    }
    // Box b to columns c on, rows r on of the m x n matrix behind the map.
    SADMM_DEV void send(int b, const CUtensorMap* map, long long c, long long r, long long n, long long m)
    {
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
            if (c < n && r < m)
                asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%2, %3}], [%1];" ::"l"(map),
                             "r"(smem_u32(mem + b * kBoxBytes)), "r"((int)c), "r"((int)r)
                             : "memory");
            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
        }
    }
    SADMM_DEV void finish()
    {
        if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
        __syncwarp();
    }
};

// v += bias of columns c .. c+15, the same for the whole warp.
SADMM_DEV void add_bias16(const float* bias, long long c, long long n, float (&v)[16])
{
    if (!bias) return;
    if (c + 16 <= n && (reinterpret_cast<uintptr_t>(bias) & 15) == 0) {
#pragma unroll
        for (int j = 0; j < 16; j += 4) {
            const float4 b = __ldg(reinterpret_cast<const float4*>(bias + c + j));
            v[j] += b.x; v[j + 1] += b.y; v[j + 2] += b.z; v[j + 3] += b.w;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 16; ++j)
            if (c + j < n) v[j] += __ldg(bias + c + j);
    }
}

// The same in few instructions, where a group of a 16-byte word is inside the row or outside.
SADMM_DEV void add_bias16_whole(const float* bias, long long c, long long n, float (&v)[16])
{
    if (!bias) return;
#pragma unroll
    for (int j = 0; j < 16; j += 4)
        if (c + j < n) {
            const float4 b = __ldg(reinterpret_cast<const float4*>(bias + c + j));
            v[j] += b.x; v[j + 1] += b.y; v[j + 2] += b.z; v[j + 3] += b.w;
        }
}
SADMM_DEV void add16_whole(const Out& o, long long r, long long c, long long n, float (&v)[16])
{
    if (o.bf16) {
        const __nv_bfloat16* p = static_cast<const __nv_bfloat16*>(o.p) + r * o.ld + c;
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (c + 8 * h < n) {
                const uint4 q = reinterpret_cast<const uint4*>(p)[h];
                const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    v[8 * h + 2 * j] += __uint_as_float(w[j] << 16);
                    v[8 * h + 2 * j + 1] += __uint_as_float(w[j] & 0xffff0000u);
                }
            }
    } else {
        const float* p = static_cast<const float*>(o.p) + r * o.ld + c;
#pragma unroll
        for (int j = 0; j < 16; j += 4)
            if (c + j < n) {
                const float4 q = *reinterpret_cast<const float4*>(p + j);
                v[j] += q.x; v[j + 1] += q.y; v[j + 2] += q.z; v[j + 3] += q.w;
            }
    }
}
SADMM_DEV void store16_whole(const Out& o, long long r, long long c, long long n, const float (&v)[16])
{
    uint4* p = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(o.p) + r * o.ld + c);
#pragma unroll
    for (int h = 0; h < 2; ++h)
        if (c + 8 * h < n)
            p[h] = make_uint4(pack_bf16(v[8 * h], v[8 * h + 1]), pack_bf16(v[8 * h + 2], v[8 * h + 3]),
                              pack_bf16(v[8 * h + 4], v[8 * h + 5]), pack_bf16(v[8 * h + 6], v[8 * h + 7]));
}

// WHOLE: every output goes out by boxes or whole 16-byte words, bias and residual come by such, and
// the general forms' instructions are not there to be jumped over (1 to 3 % with the boxes).
template <bool GATED, bool VEC, bool WHOLE>
__global__ void __launch_bounds__(kThreads, 1)
    k_q8_pair(const __grid_constant__ Maps maps, const __grid_constant__ Args a)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    constexpr uint32_t kStageBytes = Tile<VEC>::bytes;
    float* rings = reinterpret_cast<float*>(smem + kStages * kStageBytes);  // [kSlots][kSlotFloats]
    __shared__ uint64_t full[kStages], empty[kStages], s_full[kSlots], s_empty[kSlots], acc_full[2], acc_empty[2], drain, met[4];
    __shared__ uint32_t tmem_holder;
    __shared__ volatile int abort_flag;
    __shared__ float tops[2][128];
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    const int me = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    int* const status = a.t.status;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(&full[s], 1);
            mbar_init(&empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&acc_full[b], 1);
            mbar_init(&acc_empty[b], 16);  // eight warps of either CTA
        }
        for (int q = 0; q < 4; ++q) mbar_init(&met[q], 2);
        for (int s = 0; s < kSlots; ++s) {
            mbar_init(&s_full[s], 64);
            mbar_init(&s_empty[s], 8);
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

    if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(Regs<VEC>::few));
    if (warp == 0) {
        if (lane == 0) {
            int s = 0;
            uint32_t phase = 0;
            bool ok = true;
            for (int i = 0, t; ok && (t = tile_of(a, me, pairs, i)) >= 0; ++i) {
                const Place pl = place(a, t);
                const Product& p = a.prod[pl.prod];
                const int row0 = pl.mt * Tile<VEC>::rows + (int)rank * 128;
                const int col0 = GATED ? pl.nt * 128 : pl.nt * Tile<VEC>::cols + (int)rank * (Tile<VEC>::cols / 2);
                for (int k = 0; k < p.t.nk; ++k) {
                    if (!mbar_wait(&empty[s], phase ^ 1u, &abort_flag, status)) { ok = false; break; }
                    if (rank == 0) mbar_arrive_expect_tx(&full[s], 2u * kStageBytes);
                    const uint32_t bar = map_rank(smem_u32(&full[s]), 0);
                    const int second = k >= p.t.nk0;  // of a sum
                    const int kc = (second ? k - p.t.nk0 : k) * kQBlock;
                    uint8_t* sp = smem + (size_t)s * kStageBytes;
                    tma_load_pair(sp, &maps.map[p.pm + second], bar, kc, row0);
                    if (VEC) tma_load_pair(sp + kHalfBytes, &maps.map[p.pm + second], bar, kc, row0 + 256);
                    tma_load_pair(sp + Tile<VEC>::p_bytes, &maps.map[p.qm + (GATED ? (int)rank : second)], bar, kc, col0);
                    if (++s == kStages) { s = 0; phase ^= 1u; }
                }
            }
            // every stage filled has been read before the CTA retires; after a failure, time for the copies to land
            for (int i = 0; i < kStages && ok; ++i) {
                ok = mbar_wait(&empty[s], phase ^ 1u, &abort_flag, status);
                if (++s == kStages) { s = 0; phase ^= 1u; }
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
                const int nk = a.prod[place(a, t).prod].t.nk;
                for (int k = 0; k < nk; ++k) {
                    if (!mbar_wait_warp(&acc_empty[buf], bphase ^ 1u, &abort_flag, status) ||
                        !mbar_wait_warp(&full[s], phase, &abort_flag, status)) {
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    const uint32_t st = smem_u32(smem + (size_t)s * kStageBytes);
                    const uint64_t qd = sdesc_kmajor_sw128(st + Tile<VEC>::p_bytes);
#pragma unroll
                    for (int b = 0; b < (VEC ? 2 : 1); ++b) {
                        const uint64_t pd = sdesc_kmajor_sw128(st + b * kHalfBytes);
                        const uint32_t d = tmem + (uint32_t)(buf * 256 + b * 128);
#pragma unroll
                        for (int kk = 0; kk < 4; ++kk) mma_f8_pair_elect(d, pd + kk * 2, qd + kk * 2, a.idesc, kk != 0);
                    }
                    commit_pair_elect(&empty[s]);
                    commit_pair_elect(&acc_full[buf]);
                    if (++s == kStages) { s = 0; phase ^= 1u; }
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
        // warp 2: rows, warp 3: columns; blocks go into the ring in turn
        Ring ring = {rings, s_full, s_empty, &abort_flag, status, 0, 0};
        bool ok = true;
        for (int i = 0, t; ok && (t = tile_of(a, me, pairs, i)) >= 0; ++i) {
            const Place pl = place(a, t);
            const Product& p = a.prod[pl.prod];
            for (int second = 0; ok && second <= p.sum; ++second) {
                const int k0 = second ? p.t.nk0 : 0, k1 = second || !p.sum ? p.t.nk : p.t.nk0;
                const int nt = pl.nt, mt = pl.mt;
                const Scales& cs = p.qs[second];
                constexpr int own = Tile<VEC>::own;
                if (warp == 2) {
                    const Scales& rs = p.ps[second];
                    const long long r0 = (long long)mt * Tile<VEC>::rows + rank * 128;
                    ok = Ring::wide(rs) ? ring.fill_wide<own / 128>(k0, k1, p.t.nk, 0, own, rs, r0)
                                        : ring.fill<own / 32>(k0, k1, p.t.nk, lane, 32, own, rs, r0 + lane);
                } else if (VEC) {
                    ok = Ring::wide(cs) ? ring.fill_wide<1>(k0, k1, p.t.nk, Tile<VEC>::columns, 128, cs, (long long)nt * 128)
                                        : ring.fill<4>(k0, k1, p.t.nk, Tile<VEC>::columns + lane, 32, 128, cs,
                                                       (long long)nt * 128 + lane);
                } else {  // lane 0: the first 128 columns' (g's), lane 1: the others' (u's)
                    ok = ring.fill<1>(k0, k1, p.t.nk, Tile<VEC>::columns + lane * 4, 0, 1, p.qs[GATED ? lane & 1 : second],
                                      (long long)nt * (GATED ? 128 : 256) + (GATED ? 0 : (lane & 1) * 128));
                }
            }
        }
        cp_async_wait_all();
    }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(Regs<VEC>::many));
        const int q = warp & 3, part = (warp - 4) >> 2;
        const uint32_t taddr = tmem + ((uint32_t)(q * 32) << 16);
        const uint32_t freed = map_rank(smem_u32(&acc_empty[0]), 0);
        int buf = 0;
        uint32_t bphase = 0, mphase = 0;
        bool ok = true;
        int t = tile_of(a, me, pairs, 0);
        Place pl = place(a, t < 0 ? 0 : t);
        int slot_at = 0;
        uint32_t sphase = 0;
        Boxes box = {smem + kStages * kStageBytes + kSlots * kSlotFloats * 4 + (warp - 4) * Tile<VEC>::boxes * kBoxBytes, lane};
        int turn = 0;
        for (int i = 0; t >= 0; ++i) {
            const Product& p = a.prod[pl.prod];
            const int nk = p.t.nk;
            float acc[128];
#pragma unroll
            for (int j = 0; j < 128; ++j) acc[j] = 0.0f;
            // the accumulator's columns of the thread's c-th 32
            auto column = [&](int c) { return GATED ? (c >> 1) * 128 + part * 64 + (c & 1) * 32 : part * 128 + c * 32; };
            for (int k = 0; k < nk; ++k) {
                const float* slot = rings + slot_at * kSlotFloats;
                if ((k & 3) == 0) {
                    ok = mbar_wait_warp(&s_full[slot_at], sphase, &abort_flag, status);
                    if (!ok) break;
                }
                // the scales of the thread's rows, and of the tile's columns
                constexpr int R = VEC ? 2 : 1;
                float sp[R], f0 = 0.0f, f1 = 0.0f;
#pragma unroll
                for (int b = 0; b < R; ++b) sp[b] = slot[(k & 3) * Tile<VEC>::own + b * 128 + q * 32 + lane];
                if (!VEC) {
                    f0 = sp[0] * slot[Tile<VEC>::columns + (GATED ? 0 : part * 4) + (k & 3)];
                    f1 = GATED ? sp[0] * slot[Tile<VEC>::columns + 4 + (k & 3)] : f0;
                }
                ok = mbar_wait_warp(&acc_full[buf], bphase, &abort_flag, status);
                if (!ok) break;
                tc_fence_after();
                const uint32_t from = taddr + (uint32_t)buf * 256u;
                auto read = [&]() {  // the accumulator has been read
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_either(freed + (uint32_t)buf * 8u);
                };
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    if (VEC) {
                        // 16 columns of both rows: every thread reads every column's scale, and with two rows
                        // half as many as with one (where they were 1024 cycles of shared memory a block).
                        uint32_t r[2][16];
                        tmem_ld_32x32b_x16(from + part * 64 + c * 16, r[0]);
                        tmem_ld_32x32b_x16(from + 128 + part * 64 + c * 16, r[1]);
                        const float* column_scales = slot + Tile<VEC>::columns + (k & 3) * 128 + part * 64 + c * 16;
                        tmem_ld_wait();
                        if (c == 3) read();
#pragma unroll
                        for (int j = 0; j < 16; j += 4) {
                            const float4 f = *reinterpret_cast<const float4*>(column_scales + j);
#pragma unroll
                            for (int b = 0; b < 2; ++b) {
                                float* v = acc + b * 64 + c * 16 + j;
                                const float s_ = sp[VEC ? b : 0];
                                v[0] = fmaf(__uint_as_float(r[b][j]), s_ * f.x, v[0]);
                                v[1] = fmaf(__uint_as_float(r[b][j + 1]), s_ * f.y, v[1]);
                                v[2] = fmaf(__uint_as_float(r[b][j + 2]), s_ * f.z, v[2]);
                                v[3] = fmaf(__uint_as_float(r[b][j + 3]), s_ * f.w, v[3]);
                            }
                        }
                    } else {
                        // (32 columns a load: of 16, their latencies take a fifth longer)
                        uint32_t r[32];
                        tmem_ld_32x32b_x32(from + column(c), r);
                        tmem_ld_wait();
                        if (c == 3) read();
                        const float f = c < 2 ? f0 : f1;
#pragma unroll
                        for (int j = 0; j < 32; ++j) acc[c * 32 + j] = fmaf(__uint_as_float(r[j]), f, acc[c * 32 + j]);
                    }
                }
                if ((k & 3) == 3 || k + 1 == nk) {
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&s_empty[slot_at]);
                    if (++slot_at == kSlots) { slot_at = 0; sphase ^= 1u; }
                }
                if (++buf == 2) { buf = 0; bphase ^= 1u; }
            }
            if (!ok) break;
            const Place done = pl;
            t = tile_of(a, me, pairs, i + 1);
            if (t >= 0) pl = place(a, t);
            const long long row1 = (long long)done.mt * Tile<VEC>::rows + rank * 128 + q * 32 + lane;
            const long long col0 = (long long)done.nt * (GATED ? 128 : Tile<VEC>::cols) + part * (GATED || VEC ? 64 : 128);
            const bool y_bf16 = p.t.y.bf16, two = a.zm >= 0 || a.um >= 0;  // boxes that are filled together
            float top = 0.0f;
            // 16 (32) columns at a time in one loop, the sums moving up: unrolled, its instructions came
            // from memory every time (11 us a tile with GELU).  A gated pair's outputs take g's place until their scale is
            // known.
            constexpr int D = GATED ? 1 : 2;
            with_act(a.t.act, [&](auto tag) {
#pragma unroll 1
                for (int c = 0; c < (GATED ? 4 : 8); c += D) {
#pragma unroll
                    for (int d = 0; d < D; ++d) {
                        const long long row = VEC ? row1 + (c >> 2) * 256 : row1, row0 = row - lane;
                        const long long col = col0 + (VEC ? (c + d) & 3 : c + d) * 16;
                        const bool in = row < p.t.m;
                        float v[16], w[16];
#pragma unroll
                        for (int j = 0; j < 16; ++j) v[j] = acc[d * 16 + j], w[j] = GATED ? acc[64 + j] : 0.0f;
                        if (WHOLE) {
                            add_bias16_whole(a.t.bias, col, p.t.n, v);
                            if (GATED) add_bias16_whole(a.t.bias2, col, p.t.n, w);
                        } else {
                            add_bias16(a.t.bias, col, p.t.n, v);
                            if (GATED) add_bias16(a.t.bias2, col, p.t.n, w);
                        }
                        const int piece = (c + d) & 3;
                        if (two && piece == 0) box.free<0>();
                        if (GATED && a.um >= 0) {
                            box.put(1, piece, true, w);
                            if (piece == 3) box.send(1, &maps.map[a.um], col - 48, row0, p.t.n, p.t.m);
                        } else if (!WHOLE && GATED && a.t.u.p && in && col < p.t.n) {
                            store16(a.t.u, row, col, p.t.n, w, status);
                        }
                        if (a.zm >= 0) {
                            box.put(0, piece, true, v);
                            if (piece == 3) box.send(0, &maps.map[a.zm], col - 48, row0, p.t.n, p.t.m);
                        } else if (!WHOLE && a.t.z.p && in && col < p.t.n) {
                            store16(a.t.z, row, col, p.t.n, v, status);
                        }
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            v[j] = act_f32<decltype(tag)::value>(v[j]);
                            if (GATED) v[j] *= w[j];
                        }
                        if (GATED && a.y8.q) {
#pragma unroll
                            for (int j = 0; j < 16; ++j)
                                if (col + j >= p.t.n) v[j] = 0.0f;
                            top = fmaxf(top, q8_top(v));
#pragma unroll
                            for (int j = 0; j < 16; ++j) acc[j] = v[j];
                        } else {
                            if (a.t.res.p && in && col < p.t.n) {
                                if (WHOLE)
                                    add16_whole(a.t.res, row, col, p.t.n, v);
                                else
                                    add16(a.t.res, row, col, p.t.n, v, status);
                            }
                            if (!GATED && (WHOLE || p.ym >= 0)) {
                                const int last = y_bf16 ? 3 : 1, at = piece & last;
                                if (at == 0) {
                                    turn = VEC ? 0 : two ? 1 : turn ^ 1;
                                    if (VEC || (two && piece)) box.free<0>();
                                    else if (!two) box.free<1>();
                                }
                                box.put(turn, at, y_bf16, v);
                                if (at == last) box.send(turn, &maps.map[p.ym], col - 16 * last, row0, p.t.n, p.t.m);
                            } else if (in && col < p.t.n) {
                                if (WHOLE)
                                    store16_whole(p.t.y, row, col, p.t.n, v);
                                else
                                    store16(p.t.y, row, col, p.t.n, v, status);
                            }
                        }
                    }
                    if (GATED) {
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            const float done_ = acc[j];
                            acc[j] = acc[j + 16], acc[j + 16] = acc[j + 32], acc[j + 32] = acc[j + 48], acc[j + 48] = done_;
                            acc[j + 64] = acc[j + 80], acc[j + 80] = acc[j + 96], acc[j + 96] = acc[j + 112];
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < 96; ++j) acc[j] = acc[j + 32];
                    }
                }
            });
            if (GATED && a.y8.q) {
                // the other half's largest of the row's 128 units, from the warp that has them
                tops[part][q * 32 + lane] = top;
                __syncwarp();
                if (lane == 0) mbar_arrive(&met[q]);
                ok = mbar_wait_warp(&met[q], mphase, &abort_flag, status);
                mphase ^= 1u;
                if (!ok) break;
                const Q8Scale k = q8_scale(fmaxf(top, tops[part ^ 1][q * 32 + lane]));
                __syncwarp();
                if (lane == 0) mbar_arrive(&met[q]);  // read: the next tile's may be written
                ok = mbar_wait_warp(&met[q], mphase, &abort_flag, status);
                mphase ^= 1u;
                if (!ok) break;
                const long long row = row1;
                if (row < p.t.m && dbg_in(row, p.t.m, status)) {
                    if (part == 0) a.y8.s[row * a.y8.s_row + (long long)done.nt * a.y8.s_block] = k.s;
                    uint8_t* out = static_cast<uint8_t*>(a.y8.q) + row * a.y8.ld + col0;
                    const int live = (int)max(0ll, min(64ll, p.t.n - col0));
                    const bool wide = (reinterpret_cast<uintptr_t>(out) & 15) == 0;
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        uint32_t w[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float* v = acc + c * 16 + j * 4;
                            w[j] = q8_four(v[0], v[1], v[2], v[3], k);
                        }
                        if ((WHOLE || wide) && live >= c * 16 + 16) {
                            reinterpret_cast<uint4*>(out)[c] = make_uint4(w[0], w[1], w[2], w[3]);
                        } else if (WHOLE) {
#pragma unroll
                            for (int j = 0; j < 16; ++j)
                                if (c * 16 + j < live) out[c * 16 + j] = (uint8_t)(w[j >> 2] >> (8 * (j & 3)));
                        } else {
                            store_bytes8(out + c * 16, live - c * 16, w[0], w[1]);
                            store_bytes8(out + c * 16 + 8, live - c * 16 - 8, w[2], w[3]);
                        }
                    }
                }
            }
        }
        box.finish();
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();  // neither CTA's barriers nor TMEM are in use any more
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc2(tmem, 512);
    }
}

// -------------------------------------------------------------------- host --

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

// An output's map, of boxes of 128 bytes x 32 rows; false: it is stored by the threads.
bool encode_out(CUtensorMap* map, const TgMatrix& t, long long m, long long n)
{
    PFN_cuTensorMapEncodeTiled_v12000 enc = get_encode_fn();
    const bool bf16 = t.dt == SADMM_BF16;
    // (a row that ends inside 16 bytes is stored by the threads: by a box, the values behind its last column changed)
    if (!t.p || !enc || !make_out(t, m, n).vec || n % (bf16 ? 8 : 4)) return false;
    memset(map, 0, sizeof(*map));
    const cuuint64_t gdim[2] = {(cuuint64_t)n, (cuuint64_t)m};
    const cuuint64_t gstride[1] = {(cuuint64_t)t.ld * (bf16 ? 2 : 4)};
    const cuuint32_t box[2] = {bf16 ? 64u : 32u, 32u};
    const cuuint32_t estride[2] = {1u, 1u};
    return enc(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 2, t.p, gdim, gstride, box,
               estride, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

Scales scales_of(const Q8Operand& o) { return {o.s, o.s_row, o.s_block, o.rows, o.shift}; }

template <bool GATED, bool VEC, bool WHOLE>
sadmm_status run(const Maps& maps, const Args& a, int ctas, cudaStream_t s)
{
    static bool configured[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return SADMM_ECUDA;
    constexpr int smem = kStages * (int)Tile<VEC>::bytes + kSlots * kSlotFloats * 4 + 8 * Tile<VEC>::boxes * kBoxBytes + 1024;
    auto kern = k_q8_pair<GATED, VEC, WHOLE>;
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
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kern, maps, a) == cudaSuccess ? SADMM_OK : SADMM_ECUDA;
}

long long blocks_of(const Q8Problem& t)
{
    return (t.a[0].k + kQBlock - 1) / kQBlock + (t.mode == kTgSum ? (t.a[1].k + kQBlock - 1) / kQBlock : 0);
}

}  // namespace

sadmm_status launch_q8_pair(const Q8Problem* problems, int count, cudaStream_t s)
{
    // the longest contractions first
    const Q8Problem* t[kProducts];
    for (int i = 0; i < count; ++i) {
        int j = i;
        for (; j > 0 && blocks_of(*t[j - 1]) < blocks_of(problems[i]); --j) t[j] = t[j - 1];
        t[j] = &problems[i];
    }
    Args a;
    Maps maps;
    memset(&a, 0, sizeof(a));
    const bool gated = t[0]->mode == kTgGated;
    bool vec = false;  // a product's columns have scales of single rows
    for (int i = 0; i < count; ++i)
        for (int j = 0; j < (t[i]->mode == kTgSingle ? 1 : 2); ++j) vec = vec || t[i]->b[j].shift == 0;
    if (gated && vec) return SADMM_EUNSUPPORTED;  // (single tiles take those)
    long long tiles = 0;
    int next = 0;
    for (int i = 0; i < count; ++i) {
        Product& p = a.prod[i];
        const Q8Problem& q = *t[i];
        const int cols = gated || vec ? 128 : 256, rows = vec ? 512 : 256;
        p.t.m = q.m;
        p.t.n = q.n;
        if (q.y.p) p.t.y = make_out(q.y, q.m, q.n);
        p.t.p_tiles = (int)((q.m + rows - 1) / rows);
        p.t.q_tiles = (int)((q.n + cols - 1) / cols);
        p.t.first = (int)tiles;
        tiles += (long long)p.t.p_tiles * p.t.q_tiles;
        if (tiles > 0x0fffffffll) return SADMM_EUNSUPPORTED;
        p.sum = q.mode == kTgSum;
        p.t.nk0 = (int)((q.a[0].k + kQBlock - 1) / kQBlock);
        p.t.nk = (int)blocks_of(q);
        const int na = p.sum ? 2 : 1, nb = p.sum || gated ? 2 : 1;
        p.pm = next;
        for (int j = 0; j < na; ++j)
            if (next >= kOperands || !encode8(&maps.map[next++], q.a[j], 128)) return SADMM_ECUDA;
        p.qm = next;
        for (int j = 0; j < nb; ++j)
            if (next >= kOperands || !encode8(&maps.map[next++], q.b[j], vec ? 64 : 128)) return SADMM_ECUDA;
        p.ym = encode_out(&maps.map[kOperands + i], q.y, q.m, q.n) ? kOperands + i : -1;
        for (int j = 0; j < 2; ++j) {
            p.ps[j] = scales_of(q.a[na == 2 ? j : 0]);
            p.qs[j] = scales_of(q.b[nb == 2 ? j : 0]);
        }
    }
    a.t.products = count;
    a.t.tiles = (int)tiles;
    const Q8Problem& f = *t[0];
    a.t.bias = f.bias;
    a.t.bias2 = f.bias2;
    a.t.act = act_for(f.act, f.y.p && f.y.dt == SADMM_BF16);
    if (f.residual.p) a.t.res = make_out(f.residual, f.m, f.n);
    if (f.z.p) a.t.z = make_out(f.z, f.m, f.n);
    if (f.u.p) a.t.u = make_out(f.u, f.m, f.n);
    constexpr int zm = kOperands + kProducts, um = zm + 1;
    a.zm = !vec && encode_out(&maps.map[zm], f.z, f.m, f.n) ? zm : -1;
    a.um = encode_out(&maps.map[um], f.u, f.m, f.n) ? um : -1;
    a.t.status = device_status_ptr();
    a.y8 = f.y8;
    a.idesc = (1u << 4) | (vec ? 128u >> 3 : 256u >> 3) << 17 | (256u >> 4) << 24;  // e4m3 operands, fp32 sums
    const long long pairs = device_sm_count() / 2;
    const int ctas = 2 * (int)(tiles < pairs ? tiles : pairs);
    const Out& y = a.prod[0].t.y;
    const long long n = f.n;
    auto words = [](const float* b) { return (reinterpret_cast<uintptr_t>(b) & 15) == 0; };
    bool whole = (!a.t.z.p || a.zm >= 0) && (!a.t.u.p || a.um >= 0) && words(a.t.bias) && words(a.t.bias2);
    if (a.t.bias || a.t.bias2) whole = whole && n % 4 == 0;
    if (a.t.res.p) whole = whole && a.t.res.vec && n % (a.t.res.bf16 ? 8 : 4) == 0;
    if (gated) whole = whole && (a.y8.q ? q8_aligned(a.y8.q, a.y8.ld) : y.vec && n % 8 == 0);
    for (int i = 0; i < count && !gated; ++i) whole = whole && a.prod[i].ym >= 0;
#ifdef SADMM_DEBUG
    whole = false;  // the general forms check their indexes
#endif
    if (gated) return whole ? run<true, false, true>(maps, a, ctas, s) : run<true, false, false>(maps, a, ctas, s);
    if (whole) return vec ? run<false, true, true>(maps, a, ctas, s) : run<false, false, true>(maps, a, ctas, s);
    return vec ? run<false, true, false>(maps, a, ctas, s) : run<false, false, false>(maps, a, ctas, s);
}

namespace {

// The tiles of a product by itself, a pair's one after the other.
struct Rounds {
    bool rows;  // the columns have scales of single rows
    long long tall, wide, down, across, pairs, rounds;
    explicit Rounds(const Q8Problem& t)
    {
        rows = t.b[0].shift == 0 || (t.mode != kTgSingle && t.b[1].shift == 0);
        tall = rows ? 512 : 256, wide = rows || t.mode == kTgGated ? 128 : 256;
        down = (t.m + tall - 1) / tall, across = (t.n + wide - 1) / wide;
        pairs = device_sm_count() / 2;
        rounds = (down * across + pairs - 1) / pairs;
    }
};

}  // namespace

void q8_pair_less(const Q8Problem& t, long long& rows, long long& cols)
{
    const Rounds r(t);
    rows = (r.rounds - 1) * r.pairs / r.across * r.tall;
    cols = (r.rounds - 1) * r.pairs / r.down * r.wide;
}

// Expected time of a product by itself, ns.  Measured: a block takes 0.41 us, 0.75 where the
// columns have scales of single rows; a round of tiles 3.5 beside its blocks (where
// an output's rows do not start on 16-byte boundaries 25 more: its elements are stored one by one,
// 32 rows a store), a launch 4.
long long time_q8_pair(const Q8Problem& t)
{
    const Rounds r(t);
    const bool rows = r.rows;
    const long long rounds = r.rounds;
    bool apart = false;
    // (not z and u: what is kept beside y must not change y's bits)
    for (const TgMatrix* m : {&t.y, &t.residual}) apart = apart || (m->p && !make_out(*m, t.m, t.n).vec);
    return rounds * (blocks_of(t) * (rows ? 750 : 410) + 3500 + (apart ? 25000 : 0)) + 4000;
}

}  // namespace sadmm
