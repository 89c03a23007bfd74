// norm.cu -- layer norm over the rows of a matrix, forward and backward, with
// the gradients of its weight and bias.
//
//   y = gamma xhat + beta,  xhat = (x - mean) rstd,  rstd = (var + eps)^-1/2
//   d = gamma dy,  dx = rstd (d - avg(d) - xhat avg(d xhat)) [+ dres]
//   dgamma = sum over rows of dy xhat,  dbeta = sum over rows of dy
//
// Bound by memory.  A group of threads (a warp, or a block for long rows) takes
// a row at a time and keeps it in registers in fp32; mean and variance are
// taken one after the other from those registers, so the variance has no
// cancellation.  The group's next rows are on their way meanwhile: bulk copies
// into a ring of rows in shared memory (the row's barrier of the reduction
// frees a place), because the registers that would hold enough loads in flight
// are not there.  The backward's threads own fixed columns, add up their shares
// of dgamma and dbeta over the rows of their block in registers and leave one
// partial sum per block, which a second kernel adds up in a fixed order.  Rows
// too long for registers are read again from cache instead.
//
// Measured (us, us of bytes at the copy's 6.67 TB/s): forward 16384 x 4096 fp32 ->
// bf16 61.5 (60.4); backward 8192 x 4096 bf16 with a residual's gradient 57
// (40.3), of which the sums of the partial sums 6: there the arithmetic of a row
// (in pairs, f32x2) and its reduction take as long as its bytes; backward of
// 3001 x 1153 fp32 rows off 16-byte boundaries 14.5 (5.2), bound by loads and
// stores of single elements.
#include <string.h>

#include "common.cuh"
#include "internal.h"

namespace sadmm {
namespace {

using bf16 = __nv_bfloat16;

SADMM_DEV float to_f32(float v) { return v; }
SADMM_DEV float to_f32(bf16 v) { return __bfloat162float(v); }
SADMM_DEV void put(float* p, float v) { *p = v; }
SADMM_DEV void put(bf16* p, float v) { *p = __float2bfloat16_rn(v); }

SADMM_DEV void load_vec(const bf16* p, float (&v)[8])
{
    const uint4 q = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        v[2 * j] = __uint_as_float(w[j] << 16);
        v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
    }
}
SADMM_DEV void load_vec(const float* p, float (&v)[8])
{
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
SADMM_DEV void store_vec(bf16* p, const float (&v)[8])
{
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
        w[j] = *reinterpret_cast<const uint32_t*>(&h);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
SADMM_DEV void store_vec(float* p, const float (&v)[8])
{
    reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}

// Two fp32 values in a 64-bit register, for the paired instructions.
SADMM_DEV unsigned long long pair(float lo, float hi)
{
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
SADMM_DEV float low(unsigned long long v) { return __uint_as_float((uint32_t)v); }
SADMM_DEV float high(unsigned long long v) { return __uint_as_float((uint32_t)(v >> 32)); }
SADMM_DEV unsigned long long add2(unsigned long long a, unsigned long long b)
{
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
SADMM_DEV unsigned long long mul2(unsigned long long a, unsigned long long b)
{
    unsigned long long r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
SADMM_DEV unsigned long long fma2(unsigned long long a, unsigned long long b, unsigned long long c)
{
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

// A row over G threads, E times 8 elements each.  VEC: the matrices' rows start
// on 16-byte boundaries and thread t's k-th eight are the neighbours from
// column (k G + t) 8; otherwise element j of them is column (8 k + j) G + t, so
// that a warp's loads are neighbours.
template <bool VEC>
struct Cols {
    int g, t, cols;
    int* status;
    // Whether element (k, j) is inside the row.
    SADMM_DEV bool in(int k, int j) const { return at(k, j) < cols; }
    SADMM_DEV int at(int k, int j) const { return VEC ? (k * g + t) * 8 + j : (8 * k + j) * g + t; }
    SADMM_DEV bool whole(int k) const { return VEC && at(k, 0) + 8 <= cols; }
    // Index checks of a whole eight and of one element.
    SADMM_DEV bool ok(int k) const { return dbg_run(at(k, 0), 8, cols, status); }
    SADMM_DEV bool ok(int k, int j) const { return dbg_in(at(k, j), cols, status); }
};

template <bool VEC, typename T>
SADMM_DEV void load_row(const T* p, const Cols<VEC>& c, int k, float fill, float (&v)[8])
{
    if (c.whole(k) && c.ok(k)) {
        load_vec(p + c.at(k, 0), v);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = c.at(k, j) < c.cols && c.ok(k, j) ? to_f32(p[c.at(k, j)]) : fill;
    }
}

template <bool VEC, typename T>
SADMM_DEV void store_row(T* p, const Cols<VEC>& c, int k, const float (&v)[8])
{
    if (c.whole(k) && c.ok(k)) {
        store_vec(p + c.at(k, 0), v);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (c.at(k, j) < c.cols && c.ok(k, j)) put(p + c.at(k, j), v[j]);
    }
}

// Sums over the threads of a row: a warp, or the whole block through shared
// memory.  `slot` alternates between calls, so that one barrier a call is
// enough.  Every thread adds the warps' sums up in the same order.
SADMM_DEV float warp_sum(float v)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

struct __align__(16) RowSums {
    float v[2][2][32];  // [slot][which][warp]
};

template <bool BLOCK>
SADMM_DEV float row_sum(float v, RowSums& red, int slot)
{
    v = warp_sum(v);
    if (BLOCK) {
        const int warp = threadIdx.x >> 5, n = blockDim.x >> 5;
        if ((threadIdx.x & 31) == 0) red.v[slot][0][warp] = v;
        __syncthreads();
        v = 0.0f;
        for (int w = 0; w < n; w += 4) {  // the places past the last warp hold zeros
            const float4 q = *reinterpret_cast<const float4*>(&red.v[slot][0][w]);
            v += (q.x + q.y) + (q.z + q.w);
        }
    }
    return v;
}

template <bool BLOCK>
SADMM_DEV float2 row_sum2(float x, float y, RowSums& red, int slot)
{
    x = warp_sum(x);
    y = warp_sum(y);
    if (BLOCK) {
        const int warp = threadIdx.x >> 5, n = blockDim.x >> 5;
        if ((threadIdx.x & 31) == 0) {
            red.v[slot][0][warp] = x;
            red.v[slot][1][warp] = y;
        }
        __syncthreads();
        x = y = 0.0f;
        for (int w = 0; w < n; w += 4) {
            const float4 p = *reinterpret_cast<const float4*>(&red.v[slot][0][w]);
            const float4 q = *reinterpret_cast<const float4*>(&red.v[slot][1][w]);
            x += (p.x + p.y) + (p.z + p.w);
            y += (q.x + q.y) + (q.z + q.w);
        }
    }
    return make_float2(x, y);
}

SADMM_DEV void clear(RowSums& red)
{
    for (int i = threadIdx.x; i < 128; i += blockDim.x) (&red.v[0][0][0])[i] = 0.0f;
}

// ------------------------------------------------------------------ ring --

constexpr int kRingStages = 8;  // at most

SADMM_DEV void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                     smem_u32(dst)),
                 "l"(src), "r"(bytes), "r"(smem_u32(bar))
                 : "memory");
}

// Every copy has been waited for, unless a wait gave up: then some time for
// those in flight to land before the block's shared memory is given back.
SADMM_DEV void drain_after_failure(volatile int& abort_flag)
{
    if (!abort_flag) return;
    const unsigned long long t0 = globaltimer();
    while (globaltimer() - t0 < 10000000ull) {}
}

// What a bulk copy takes of row r: its whole eights (VEC; the ragged end is read
// from global memory), or the 16-byte words that hold it.  Those of the first
// and last row would reach past the matrix, so these rows are read directly.
template <bool VEC, typename T>
struct Part {
    const T* p;
    long long ld, rows;
    int cols;
    SADMM_DEV bool copied(long long r) const { return VEC || (r > 0 && r < rows - 1); }
    SADMM_DEV const uint8_t* from(long long r) const
    {
        const uintptr_t a = reinterpret_cast<uintptr_t>(p + r * ld);
        return reinterpret_cast<const uint8_t*>(VEC ? a : a & ~uintptr_t(15));
    }
    SADMM_DEV uint32_t bytes(long long r) const
    {
        if (VEC) return (uint32_t)(cols & ~7) * (uint32_t)sizeof(T);
        const uintptr_t a = reinterpret_cast<uintptr_t>(p + r * ld);
        return (uint32_t)(((a + (uintptr_t)cols * sizeof(T) + 15) & ~uintptr_t(15)) - (a & ~uintptr_t(15)));
    }
    // Index check of a copy: in row r where rows are aligned, else in the span from the matrix's first element to its
    // last.
    SADMM_DEV bool ok(long long r, int* status) const
    {
        const long long at = (from(r) - reinterpret_cast<const uint8_t*>(p));
        const long long total = ((rows - 1) * ld + cols) * (long long)sizeof(T);
        return dbg_in(r, rows, status) && dbg_run(at, bytes(r), total, status);
    }
    // Room for a copy of any row.
    static __host__ __device__ int room(int cols) { return (cols * (int)sizeof(T) + 32 + 127) / 128 * 128; }
    // The k-th eight of row r, from its copy at `s` (NULL: from global memory).
    SADMM_DEV void load(const Cols<VEC>& c, const uint8_t* s, long long r, int k, float fill, float (&v)[8]) const
    {
        const T* g = p + r * ld;
        if (VEC) {
            if (s && c.whole(k))
                load_vec(reinterpret_cast<const T*>(s) + c.at(k, 0), v);
            else
                load_row<VEC>(g, c, k, fill, v);
        } else if (s) {
            const T* q = reinterpret_cast<const T*>(s + (reinterpret_cast<uintptr_t>(g) & 15));
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = c.at(k, j) < c.cols ? to_f32(q[c.at(k, j)]) : fill;
        } else {
            load_row<VEC>(g, c, k, fill, v);
        }
    }
};

struct FwdArgs {
    const void* x;
    void* y;
    const float* gamma;
    const float* beta;
    float* mean;
    float* rstd;
    long long rows, ldx, ldy;
    int cols;
    int stages;  // rows of the ring (0: rows are read directly)
    float eps;
    float n;  // cols: sums are divided by it, so that a constant row's mean is that constant
    int* status;
};

// CAP: threads of a block at most; 0: rows are taken by warps, eight a block.
// Up to 16 columns a thread, gamma and beta stay in registers too.
template <typename X, typename Y, bool VEC, int CAP, int E>
__global__ void __launch_bounds__(CAP ? CAP : 256, CAP == 256 || CAP == 0 ? 3 : 1) k_ln_fwd(const FwdArgs a)
{
    constexpr bool BLOCK = CAP > 0, KEEP = E <= 2;
    extern __shared__ __align__(128) uint8_t ring[];
    __shared__ RowSums red;
    __shared__ uint64_t bars[BLOCK ? 1 : 8][kRingStages];
    __shared__ volatile int abort_flag;
    const int G = BLOCK ? blockDim.x : 32, R = BLOCK ? 1 : blockDim.x / 32;
    const int group = BLOCK ? 0 : threadIdx.x >> 5;
    const Cols<VEC> c = {G, BLOCK ? (int)threadIdx.x : (int)(threadIdx.x & 31), a.cols, a.status};
    const long long first = (long long)blockIdx.x * R + group, step = (long long)gridDim.x * R;
    const Part<VEC, X> x = {static_cast<const X*>(a.x), a.ldx, a.rows, a.cols};
    const int room = Part<VEC, X>::room(a.cols);
    uint8_t* mine = ring + (size_t)group * a.stages * room;
    uint64_t* bar = bars[group];
    if (threadIdx.x == 0) abort_flag = 0;
    if (c.t == 0) {
        for (int s = 0; s < a.stages; ++s) mbar_init(&bar[s], 1);
        fence_mbar_init();
    }
    clear(red);
    __syncthreads();
    pdl_wait();
    pdl_trigger();
    auto fetch = [&](long long r, int s) {  // by the group's first thread
        if (r >= a.rows) return;
        if (x.copied(r) && x.ok(r, a.status)) {
            mbar_arrive_expect_tx(&bar[s], x.bytes(r));
            bulk_load(mine + s * room, x.from(r), x.bytes(r), &bar[s]);
        } else {
            mbar_arrive(&bar[s]);
        }
    };
    if (c.t == 0)
        for (int s = 0; s < a.stages; ++s) fetch(first + s * step, s);
    float g[KEEP ? E : 1][8], b[KEEP ? E : 1][8];
    auto affine = [&](int k, float (&gk)[8], float (&bk)[8]) {
#pragma unroll
        for (int j = 0; j < 8; ++j) gk[j] = 1.0f, bk[j] = 0.0f;
        if (a.gamma) load_row<VEC>(a.gamma, c, k, 0.0f, gk);
        if (a.beta) load_row<VEC>(a.beta, c, k, 0.0f, bk);
    };
    if (KEEP) {
#pragma unroll
        for (int k = 0; k < E; ++k) affine(k, g[KEEP ? k : 0], b[KEEP ? k : 0]);
    }
    int s = 0;
    uint32_t phase = 0;
    for (long long r = first; r < a.rows; r += step) {
        const uint8_t* row = nullptr;
        if (a.stages) {
            mbar_wait(&bar[s], phase, &abort_flag, a.status);
            if (x.copied(r)) row = mine + s * room;
        }
        float v[E][8];
        float sum = 0.0f;
#pragma unroll
        for (int k = 0; k < E; ++k) {
            x.load(c, row, r, k, 0.0f, v[k]);
            float t = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) t += v[k][j];
            sum += t;
        }
        const float mean = row_sum<BLOCK>(sum, red, 0) / a.n;
        if (a.stages) {  // the whole group has read its row
            if (!BLOCK) __syncwarp();
            if (c.t == 0) fetch(r + a.stages * step, s);
            if (++s == a.stages) { s = 0; phase ^= 1u; }
        }
        sum = 0.0f;
#pragma unroll
        for (int k = 0; k < E; ++k) {
            float t = 0.0f;
            if (c.whole(k)) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float d = v[k][j] - mean;
                    t += d * d;
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float d = c.at(k, j) < a.cols ? v[k][j] - mean : 0.0f;
                    t += d * d;
                }
            }
            sum += t;
        }
        const float rstd = rsqrtf(row_sum<BLOCK>(sum, red, 1) / a.n + a.eps);
        if (c.t == 0) {
            if (a.mean) a.mean[r] = mean;
            if (a.rstd) a.rstd[r] = rstd;
        }
        Y* y = static_cast<Y*>(a.y) + r * a.ldy;
#pragma unroll
        for (int k = 0; k < E; ++k) {
            if (!KEEP) affine(k, g[0], b[0]);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[k][j] = (v[k][j] - mean) * rstd * g[KEEP ? k : 0][j] + b[KEEP ? k : 0][j];
            store_row<VEC>(y, c, k, v[k]);
        }
    }
    drain_after_failure(abort_flag);
}

// Rows of any length: a block a row, read three times (from cache after the first).
template <typename X, typename Y>
__global__ void __launch_bounds__(1024) k_ln_fwd_long(const FwdArgs a)
{
    __shared__ RowSums red;
    clear(red);
    pdl_wait();
    pdl_trigger();
    __syncthreads();
    const long long r = blockIdx.x;
    const X* x = static_cast<const X*>(a.x) + r * a.ldx;
    float s = 0.0f;
    for (int c = threadIdx.x; c < a.cols; c += 1024) s += to_f32(x[c]);
    const float mean = row_sum<true>(s, red, 0) / a.n;
    s = 0.0f;
    for (int c = threadIdx.x; c < a.cols; c += 1024) {
        const float d = to_f32(x[c]) - mean;
        s += d * d;
    }
    const float rstd = rsqrtf(row_sum<true>(s, red, 1) / a.n + a.eps);
    if (threadIdx.x == 0) {
        if (a.mean) a.mean[r] = mean;
        if (a.rstd) a.rstd[r] = rstd;
    }
    Y* y = static_cast<Y*>(a.y) + r * a.ldy;
    for (int c = threadIdx.x; c < a.cols; c += 1024)
        put(y + c, (to_f32(x[c]) - mean) * rstd * (a.gamma ? a.gamma[c] : 1.0f) + (a.beta ? a.beta[c] : 0.0f));
}

struct BwdArgs {
    const void* x;
    const void* dy;
    const void* dres;
    void* dx;
    const float* gamma;
    const float* mean;
    const float* rstd;
    float* part_g;  // [blocks][cols] partial dgamma, dbeta; NULL: not wanted
    float* part_b;
    long long rows, ldx, lddy, lddres, lddx;
    int cols;
    int stages;
    float inv_n;
    int* status;
};

template <typename X, typename Y, bool VEC, int CAP, int E>
__global__ void __launch_bounds__(CAP ? CAP : 256, CAP == 512 ? 1 : CAP && E == 1 ? 3 : 2) k_ln_bwd(const BwdArgs a)
{
    constexpr bool BLOCK = CAP > 0;
    extern __shared__ __align__(128) uint8_t ring[];
    __shared__ RowSums red;
    __shared__ float comb[BLOCK ? 1 : 8][BLOCK ? 1 : 256];
    __shared__ uint64_t bars[BLOCK ? 1 : 8][kRingStages];
    __shared__ volatile int abort_flag;
    const int G = BLOCK ? blockDim.x : 32, R = BLOCK ? 1 : blockDim.x / 32;
    const int warp = threadIdx.x >> 5, group = BLOCK ? 0 : warp;
    const Cols<VEC> c = {G, BLOCK ? (int)threadIdx.x : (int)(threadIdx.x & 31), a.cols, a.status};
    const long long first = (long long)blockIdx.x * R + group, step = (long long)gridDim.x * R;
    const Part<VEC, X> x = {static_cast<const X*>(a.x), a.ldx, a.rows, a.cols};
    const Part<VEC, Y> dy = {static_cast<const Y*>(a.dy), a.lddy, a.rows, a.cols};
    const Part<VEC, X> dres = {static_cast<const X*>(a.dres), a.lddres, a.rows, a.cols};
    const int room_x = Part<VEC, X>::room(a.cols), room_y = Part<VEC, Y>::room(a.cols);
    const int room = room_x + room_y + (a.dres ? room_x : 0);
    uint8_t* mine = ring + (size_t)group * a.stages * room;
    uint64_t* bar = bars[group];
    if (threadIdx.x == 0) abort_flag = 0;
    if (c.t == 0) {
        for (int s = 0; s < a.stages; ++s) mbar_init(&bar[s], 1);
        fence_mbar_init();
    }
    clear(red);
    __syncthreads();
    pdl_wait();
    pdl_trigger();
    auto fetch = [&](long long r, int s) {  // by the group's first thread
        if (r >= a.rows) return;
        if (x.copied(r) && x.ok(r, a.status) && dy.ok(r, a.status) && (!a.dres || dres.ok(r, a.status))) {
            uint8_t* to = mine + s * room;
            mbar_arrive_expect_tx(&bar[s], x.bytes(r) + dy.bytes(r) + (a.dres ? dres.bytes(r) : 0u));
            bulk_load(to, x.from(r), x.bytes(r), &bar[s]);
            bulk_load(to + room_x, dy.from(r), dy.bytes(r), &bar[s]);
            if (a.dres) bulk_load(to + room_x + room_y, dres.from(r), dres.bytes(r), &bar[s]);
        } else {
            mbar_arrive(&bar[s]);
        }
    };
    if (c.t == 0)
        for (int s = 0; s < a.stages; ++s) fetch(first + s * step, s);
    unsigned long long g[E][4], dg[E][4], db[E][4];
#pragma unroll
    for (int k = 0; k < E; ++k) {
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = 1.0f;
        if (a.gamma) load_row<VEC>(a.gamma, c, k, 0.0f, v);
#pragma unroll
        for (int j = 0; j < 4; ++j) g[k][j] = pair(v[2 * j], v[2 * j + 1]), dg[k][j] = db[k][j] = 0;
    }
    int slot = 0, s = 0, last = 0;
    uint32_t phase = 0;
    float next_mean = 0.0f, next_rstd = 0.0f;
    if (first < a.rows) next_mean = a.mean[first], next_rstd = a.rstd[first];
    for (long long r = first; r < a.rows; r += step) {
        const float mean = next_mean, rstd = next_rstd;
        if (r + step < a.rows) next_mean = a.mean[r + step], next_rstd = a.rstd[r + step];
        const uint8_t* row = nullptr;
        if (a.stages) {
            mbar_wait(&bar[s], phase, &abort_flag, a.status);
            if (x.copied(r)) row = mine + s * room;
        }
        // pairs of neighbouring elements (f32x2): half the instructions
        unsigned long long xh[E][4], d[E][4], t1 = 0, t2 = 0;
        const unsigned long long minus = pair(-mean, -mean), scale = pair(rstd, rstd);
#pragma unroll
        for (int k = 0; k < E; ++k) {
            float xv[8], dv[8];
            x.load(c, row, r, k, mean, xv);  // past the row's end: xhat = dy = 0
            dy.load(c, row ? row + room_x : nullptr, r, k, 0.0f, dv);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                xh[k][j] = mul2(add2(pair(xv[2 * j], xv[2 * j + 1]), minus), scale);
                const unsigned long long v = pair(dv[2 * j], dv[2 * j + 1]);
                dg[k][j] = fma2(v, xh[k][j], dg[k][j]);
                db[k][j] = add2(db[k][j], v);
                d[k][j] = mul2(v, g[k][j]);
                t1 = add2(t1, d[k][j]);
                t2 = fma2(d[k][j], xh[k][j], t2);
            }
        }
        const float s1 = low(t1) + high(t1), s2 = low(t2) + high(t2);
        const float2 sum = row_sum2<BLOCK>(s1, s2, red, slot);
        slot ^= 1;
        // the whole group is done with the row before: its place takes the one `stages` rows on
        if (a.stages && c.t == 0 && r != first) fetch(r + (a.stages - 1) * step, last);
        if (a.dx) {
            const float c1 = sum.x * a.inv_n, c2 = sum.y * a.inv_n;
            const unsigned long long m1 = pair(-c1, -c1), m2 = pair(-c2, -c2);
            X* dx = static_cast<X*>(a.dx) + r * a.lddx;
#pragma unroll
            for (int k = 0; k < E; ++k) {
                float e[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) e[j] = 0.0f;
                if (a.dres) dres.load(c, row ? row + room_x + room_y : nullptr, r, k, 0.0f, e);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const unsigned long long v =
                        fma2(fma2(xh[k][j], m2, add2(d[k][j], m1)), scale, pair(e[2 * j], e[2 * j + 1]));
                    e[2 * j] = low(v);
                    e[2 * j + 1] = high(v);
                }
                store_row<VEC>(dx, c, k, e);
            }
        }
        last = s;
        if (++s == a.stages) { s = 0; phase ^= 1u; }
        if (!BLOCK) __syncwarp();
    }
    drain_after_failure(abort_flag);
    if (!a.part_g) return;
    float* pg = a.part_g + (long long)blockIdx.x * a.cols;
    float* pb = a.part_b + (long long)blockIdx.x * a.cols;
    if (BLOCK) {
#pragma unroll
        for (int k = 0; k < E; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (c.at(k, j) < a.cols) {
                    pg[c.at(k, j)] = (j & 1) ? high(dg[k][j / 2]) : low(dg[k][j / 2]);
                    pb[c.at(k, j)] = (j & 1) ? high(db[k][j / 2]) : low(db[k][j / 2]);
                }
    } else {
        // the warps' sums added up in warp order, thread (j, lane) for element j of lane's eight
#pragma unroll
        for (int k = 0; k < E; ++k)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                __syncthreads();
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const unsigned long long v = half ? db[k][j / 2] : dg[k][j / 2];
                    comb[BLOCK ? 0 : warp][BLOCK ? 0 : j * 32 + c.t] = (j & 1) ? high(v) : low(v);
                }
                __syncthreads();
                float v = 0.0f;
                for (int w = 0; w < R; ++w) v += comb[BLOCK ? 0 : w][BLOCK ? 0 : threadIdx.x];
                const int col = c.at(k, warp);
                if (col < a.cols) (half ? pb : pg)[col] = v;
            }
    }
}

// Rows of any length: dx, a block a row, read twice.
template <typename X, typename Y>
__global__ void __launch_bounds__(1024) k_ln_bwd_long(const BwdArgs a)
{
    __shared__ RowSums red;
    clear(red);
    pdl_wait();
    pdl_trigger();
    __syncthreads();
    const long long r = blockIdx.x;
    const X* x = static_cast<const X*>(a.x) + r * a.ldx;
    const Y* dy = static_cast<const Y*>(a.dy) + r * a.lddy;
    const float mean = a.mean[r], rstd = a.rstd[r];
    float2 s = make_float2(0.0f, 0.0f);
    for (int c = threadIdx.x; c < a.cols; c += 1024) {
        const float d = to_f32(dy[c]) * (a.gamma ? a.gamma[c] : 1.0f);
        s.x += d;
        s.y += d * (to_f32(x[c]) - mean) * rstd;
    }
    s = row_sum2<true>(s.x, s.y, red, 0);
    const float c1 = s.x * a.inv_n, c2 = s.y * a.inv_n;
    const X* dres = a.dres ? static_cast<const X*>(a.dres) + r * a.lddres : nullptr;
    X* dx = static_cast<X*>(a.dx) + r * a.lddx;
    for (int c = threadIdx.x; c < a.cols; c += 1024) {
        const float d = to_f32(dy[c]) * (a.gamma ? a.gamma[c] : 1.0f);
        const float o = rstd * (d - c1 - (to_f32(x[c]) - mean) * rstd * c2);
        put(dx + c, o + (dres ? to_f32(dres[c]) : 0.0f));
    }
}

// Rows of any length: partial dgamma and dbeta of 256 columns over the rows
// blockIdx.y, blockIdx.y + gridDim.y, ...
template <typename X, typename Y>
__global__ void __launch_bounds__(256) k_ln_cols_long(const BwdArgs a)
{
    pdl_wait();
    pdl_trigger();
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= a.cols) return;
    float g = 0.0f, b = 0.0f;
    for (long long r = blockIdx.y; r < a.rows; r += gridDim.y) {
        const float dy = to_f32(static_cast<const Y*>(a.dy)[r * a.lddy + c]);
        g += dy * (to_f32(static_cast<const X*>(a.x)[r * a.ldx + c]) - a.mean[r]) * a.rstd[r];
        b += dy;
    }
    a.part_g[(long long)blockIdx.y * a.cols + c] = g;
    a.part_b[(long long)blockIdx.y * a.cols + c] = b;
}

// out[c] = the sum of part[0 .. parts-1][c], 32 groups of parts at a time, then
// the groups in order.  blockIdx.y: dgamma or dbeta.
__global__ void __launch_bounds__(1024) k_ln_sums(const float* __restrict__ part_g, const float* __restrict__ part_b,
                                                  float* __restrict__ dgamma, float* __restrict__ dbeta, int cols,
                                                  int parts)
{
    pdl_wait();
    pdl_trigger();
    __shared__ float red[32][33];
    const float* p = blockIdx.y ? part_b : part_g;
    float* o = blockIdx.y ? dbeta : dgamma;
    if (!o) return;
    const int g = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int c = blockIdx.x * 32 + lane;
    float v = 0.0f;
    if (c < cols) {
#pragma unroll 16
        for (int k = g; k < parts; k += 32) v += p[(size_t)k * cols + c];
    }
    red[g][lane] = v;
    __syncthreads();
    // warp g adds up column g of the 32
    v = warp_sum(red[lane][g]);
    if (lane == 0 && blockIdx.x * 32 + g < cols) o[blockIdx.x * 32 + g] = v;
}

// -------------------------------------------------------------------- host --

// A warp takes a row up to this length (16 elements a lane), a block up to
// these: 512 threads of 16 (forward: 1024 of 32).
constexpr int kWarpCols = 512;
constexpr int kFwdBlockCols = 32768, kBwdBlockCols = 8192;
// Backward: up to here 8 elements a thread, above it 16 (8192 x 4096 from DRAM: 57 us
// with 16 and 256 threads, 64 with 8 and 512).
constexpr int kBwdShortCols = 2048;

// Threads of a block that share a row of `cols`, at e times 8 elements each.
int block_threads(int cols, int e) { return (int)round_up((cols + 8 * e - 1) / (8 * e), 32); }

// Blocks an SM holds: of eight warps with a row each, or of one row, where the
// kernels' registers allow 768 threads (forward: 16 elements each; backward: 8,
// and 512 of 16).
int fwd_blocks_per_sm(int cols)
{
    if (cols <= kWarpCols) return 3;
    const int threads = block_threads(cols, 2);
    return threads > 256 ? 1 : 768 / threads < 8 ? 768 / threads : 8;
}
int bwd_blocks_per_sm(int cols)
{
    if (cols <= kWarpCols) return 2;
    if (cols <= kBwdShortCols) return 768 / block_threads(cols, 1) < 4 ? 768 / block_threads(cols, 1) : 4;
    return cols <= 4096 ? 2 : 1;
}

// Blocks of the backward: each leaves a partial sum.
int bwd_blocks(long long rows, int cols)
{
    const int per = cols <= kWarpCols ? 8 : 1;
    const long long want = (rows + per - 1) / per, most = (long long)bwd_blocks_per_sm(cols) * device_sm_count();
    return (int)(want < most ? want : most);
}

bool rows16(const void* p, long long ld, int dt)
{
    return !p || ((reinterpret_cast<uintptr_t>(p) | (uintptr_t)(ld * (dt == SADMM_BF16 ? 2 : 4))) & 15) == 0;
}

constexpr int kMostRing = 212 * 1024;

// Rows of the ring: what `blocks` CTAs an SM can hold, with one group or eight
// (warps) a block, beside the kernels' static shared memory; none where a group
// has one row, a row has no whole eight, or fewer than `least` fit.
int ring_stages(long long rows, long long groups, int per_block, int blocks, int room, int cols, int least)
{
    if (rows <= groups || cols < 8) return 0;
    int bytes = (224 / blocks - (per_block > 1 ? 10 : 3)) * 1024;
    if (bytes > kMostRing) bytes = kMostRing;
    int s = bytes / (room * per_block);
    const long long most = (rows + groups - 1) / groups;
    if (s > kRingStages) s = kRingStages;
    if (s > most) s = (int)most;
    return s < least ? 0 : s;
}

// Lets a kernel have the shared memory of its ring (once per device and kernel).
template <typename K>
bool allow_ring(K kern, bool (&done)[64])
{
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return false;
    if (!done[dev])
        done[dev] = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostRing) == cudaSuccess;
    return done[dev];
}

template <typename X, typename Y, bool VEC, int CAP, int E>
sadmm_status fwd_run(FwdArgs a, cudaStream_t s)
{
    static bool allowed[64];
    auto kern = k_ln_fwd<X, Y, VEC, CAP, E>;
    if (!allow_ring(kern, allowed)) return SADMM_ECUDA;
    const int threads = CAP ? block_threads(a.cols, E) : 256, per = CAP ? 1 : 8;
    const int blocks = fwd_blocks_per_sm(a.cols);
    const long long want = (a.rows + per - 1) / per, most = (long long)blocks * device_sm_count();
    const long long grid = want < most ? want : most;
    const int room = Part<VEC, X>::room(a.cols);
    a.stages = ring_stages(a.rows, grid * per, per, blocks, room, a.cols, 1);
    return launch_pdl(kern, dim3((unsigned)grid), dim3(threads), (size_t)a.stages * room * per, s, a) == cudaSuccess
               ? SADMM_OK
               : SADMM_ECUDA;
}

template <typename X, typename Y, bool VEC>
sadmm_status fwd(const FwdArgs& a, cudaStream_t s)
{
    if (a.cols <= 256) return fwd_run<X, Y, VEC, 0, 1>(a, s);
    if (a.cols <= kWarpCols) return fwd_run<X, Y, VEC, 0, 2>(a, s);
    if (a.cols <= 4096) return fwd_run<X, Y, VEC, 256, 2>(a, s);
    if (a.cols <= 8192) return fwd_run<X, Y, VEC, 512, 2>(a, s);
    if (a.cols <= kFwdBlockCols) return fwd_run<X, Y, VEC, 1024, 4>(a, s);
    return launch_pdl(k_ln_fwd_long<X, Y>, dim3((unsigned)a.rows), dim3(1024), 0, s, a) == cudaSuccess ? SADMM_OK
                                                                                                        : SADMM_ECUDA;
}

template <typename X, typename Y, bool VEC, int CAP, int E>
sadmm_status bwd_run(BwdArgs a, cudaStream_t s)
{
    static bool allowed[64];
    auto kern = k_ln_bwd<X, Y, VEC, CAP, E>;
    if (!allow_ring(kern, allowed)) return SADMM_ECUDA;
    const int threads = CAP ? block_threads(a.cols, E) : 256, per = CAP ? 1 : 8;
    const int grid = bwd_blocks(a.rows, a.cols);
    const int room = Part<VEC, X>::room(a.cols) * (a.dres ? 2 : 1) + Part<VEC, Y>::room(a.cols);
    a.stages = ring_stages(a.rows, (long long)grid * per, per, bwd_blocks_per_sm(a.cols), room, a.cols, 2);
    return launch_pdl(kern, dim3((unsigned)grid), dim3(threads), (size_t)a.stages * room * per, s, a) == cudaSuccess
               ? SADMM_OK
               : SADMM_ECUDA;
}

template <typename X, typename Y, bool VEC>
sadmm_status bwd(const BwdArgs& a, cudaStream_t s)
{
    if (a.cols <= 256) return bwd_run<X, Y, VEC, 0, 1>(a, s);
    if (a.cols <= kWarpCols) return bwd_run<X, Y, VEC, 0, 2>(a, s);
    if (a.cols <= kBwdShortCols) return bwd_run<X, Y, VEC, 256, 1>(a, s);
    if (a.cols <= 4096) return bwd_run<X, Y, VEC, 256, 2>(a, s);
    if (a.cols <= kBwdBlockCols) return bwd_run<X, Y, VEC, 512, 2>(a, s);
    cudaError_t err = cudaSuccess;
    if (a.dx) err = launch_pdl(k_ln_bwd_long<X, Y>, dim3((unsigned)a.rows), dim3(1024), 0, s, a);
    if (err == cudaSuccess && a.part_g)
        err = launch_pdl(k_ln_cols_long<X, Y>,
                         dim3((unsigned)((a.cols + 255) / 256), (unsigned)bwd_blocks(a.rows, a.cols)), dim3(256), 0, s, a);
    return err == cudaSuccess ? SADMM_OK : SADMM_ECUDA;
}

}  // namespace

size_t layernorm_bwd_bytes(const sadmm_layernorm_bwd_args& a)
{
    if (!a.dgamma && !a.dbeta) return 0;
    return 2 * (size_t)bwd_blocks(a.rows, a.cols) * (size_t)round_up(a.cols, 64) * 4;
}

sadmm_status launch_layernorm_fwd(const sadmm_layernorm_fwd_args& a, cudaStream_t s)
{
    if (a.rows == 0) return SADMM_OK;
    const FwdArgs f = {a.x, a.y, a.gamma, a.beta, a.mean, a.rstd, a.rows, a.ldx, a.ldy, a.cols, 0,
                       a.eps, (float)a.cols, device_status_ptr()};
    const bool vec = rows16(a.x, a.ldx, a.xdt) && rows16(a.y, a.ldy, a.ydt) && rows16(a.gamma, 0, SADMM_FP32) &&
                     rows16(a.beta, 0, SADMM_FP32);
    if (a.xdt == SADMM_BF16) {
        if (a.ydt == SADMM_BF16) return vec ? fwd<bf16, bf16, true>(f, s) : fwd<bf16, bf16, false>(f, s);
        return vec ? fwd<bf16, float, true>(f, s) : fwd<bf16, float, false>(f, s);
    }
    if (a.ydt == SADMM_BF16) return vec ? fwd<float, bf16, true>(f, s) : fwd<float, bf16, false>(f, s);
    return vec ? fwd<float, float, true>(f, s) : fwd<float, float, false>(f, s);
}

sadmm_status launch_layernorm_bwd(const sadmm_layernorm_bwd_args& a, void* ws, cudaStream_t s)
{
    const bool cols = a.dgamma || a.dbeta;
    if (a.rows == 0) {
        if (a.dgamma && cudaMemsetAsync(a.dgamma, 0, (size_t)a.cols * 4, s) != cudaSuccess) return SADMM_ECUDA;
        if (a.dbeta && cudaMemsetAsync(a.dbeta, 0, (size_t)a.cols * 4, s) != cudaSuccess) return SADMM_ECUDA;
        return SADMM_OK;
    }
    const int blocks = bwd_blocks(a.rows, a.cols);
    float* pg = cols ? static_cast<float*>(ws) : nullptr;
    float* pb = cols ? pg + (size_t)blocks * (size_t)round_up(a.cols, 64) : nullptr;
    const BwdArgs b = {a.x, a.dy, a.dres, a.dx, a.gamma, a.mean, a.rstd, pg, pb, a.rows, a.ldx, a.lddy, a.lddres,
                       a.lddx, a.cols, 0, (float)(1.0 / a.cols), device_status_ptr()};
    const bool vec = rows16(a.x, a.ldx, a.xdt) && rows16(a.dy, a.lddy, a.dydt) && rows16(a.dres, a.lddres, a.xdt) &&
                     rows16(a.dx, a.lddx, a.xdt) && rows16(a.gamma, 0, SADMM_FP32);
    sadmm_status st;
    if (a.xdt == SADMM_BF16) {
        if (a.dydt == SADMM_BF16)
            st = vec ? bwd<bf16, bf16, true>(b, s) : bwd<bf16, bf16, false>(b, s);
        else
            st = vec ? bwd<bf16, float, true>(b, s) : bwd<bf16, float, false>(b, s);
    } else if (a.dydt == SADMM_BF16) {
        st = vec ? bwd<float, bf16, true>(b, s) : bwd<float, bf16, false>(b, s);
    } else {
        st = vec ? bwd<float, float, true>(b, s) : bwd<float, float, false>(b, s);
    }
    if (st != SADMM_OK || !cols) return st;
    return launch_pdl(k_ln_sums, dim3((unsigned)((a.cols + 31) / 32), 2), dim3(1024), 0, s, pg, pb, a.dgamma, a.dbeta,
                      a.cols, blocks) == cudaSuccess
               ? SADMM_OK
               : SADMM_ECUDA;
}

}  // namespace sadmm
