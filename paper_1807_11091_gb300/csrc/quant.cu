// quant.cu -- matrices in 8 bits: e4m3 values with an fp32 scale for each block
// of 128 columns of a row (or 128 x 128), of a matrix and of its transpose, in one
// pass over the source.  The source is a matrix, or what a backward pass has
// to make 8-bit: dy act'(z), or the gated pair's dg = dh u act'(g) and
// du = dh act(g), whose column sums (the bias's gradient) are taken on the way.
//
// Measured: 10240 x 4096 bf16 in tiles, both ways, 51 us (25 of its 168 MB at 6.79 TB/s), bound by
// issuing (58 % of the cycles) and shared memory; the gated pair's dg and du of 4096 x 5461, both
// ways, 100 us cold (33 of its 224 MB), bound by issuing (67 %): act, its slope and two quotients a value;
// 131 with both in one CTA, a quotient and a row's scale at a time.
#include "act.cuh"
#include "q8.cuh"

namespace sadmm {
namespace {

struct Args {
    const void *x, *z, *u;
    long long ldx, ldz, ldu;
    int xdt, act, tile;
    long long rows, cols;
    sadmm_q8_out out[2], out_t[2];
    float* part[2];         // [row tiles][cols] column sums of a tile's rows; NULL: not wanted
    long long row_tiles, col_tiles;
    int x_aligned, z_aligned, u_aligned;  // rows start on 16-byte boundaries
    int* status;
};

enum { kPlain = 0, kSlope = 1, kGate = 2 };

SADMM_DEV Span span_of(const void* p, long long ld, long long rows, long long cols, int size)
{
    const uint8_t* b = static_cast<const uint8_t*>(p);
    return {b, b + ((rows - 1) * ld + cols) * size};
}

struct Spans {
    Span x, z, u;
};
template <int PRO>
SADMM_DEV Spans spans_of(const Args& a)
{
    Spans s;
    s.x = span_of(a.x, a.ldx, a.rows, a.cols, a.xdt == SADMM_BF16 ? 2 : 4);
    s.z = PRO != kPlain && a.z ? span_of(a.z, a.ldz, a.rows, a.cols, 2) : s.x;
    s.u = PRO == kGate ? span_of(a.u, a.ldu, a.rows, a.cols, 2) : s.x;
    return s;
}

// Columns c .. c+7 of N rows from r on (with `step` between them): the words first, then the values.
template <int ES, int N, bool AL>
struct Rows8 {
    Raw8<ES, AL> raw[N];
    SADMM_DEV void ask(const void* p, long long ld, bool aligned, const Span& m, const Args& a, long long r, long long step,
                       long long c)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const long long row = r + i * step;
            const bool in = row < a.rows && c < a.cols && dbg_in(row, a.rows, a.status) && dbg_in(c, a.cols, a.status);
            ask8(static_cast<const uint8_t*>(p) + (in ? (row * ld + c) * ES : 0), in, aligned, m, raw[i]);
        }
    }
    SADMM_DEV void take(const void* p, long long ld, bool aligned, const Span& m, const Args& a, long long r, long long step,
                        long long c, int i, float (&v)[8]) const
    {
        take8(static_cast<const uint8_t*>(p) + ((r + i * step) * ld + c) * ES, (int)min(8ll, a.cols - c), aligned, m, raw[i], v);
    }
};

// The source's values in the same places, zeros outside the matrix (which: dg or du).
template <int PRO, int ACT, int ES, int N, bool AL>
SADMM_DEV void load_source(const Args& a, const Spans& s, int which, long long r, long long step, long long c, float (*v)[8])
{
    constexpr bool Z = PRO == kGate || (PRO == kSlope && ACT != SADMM_ACT_NONE);
    Rows8<ES, N, AL> x;
    Rows8<2, Z ? N : 1, AL> z;
    Rows8<2, PRO == kGate ? N : 1, AL> u;
    x.ask(a.x, a.ldx, a.x_aligned, s.x, a, r, step, c);
    if (Z) z.ask(a.z, a.ldz, a.z_aligned, s.z, a, r, step, c);
    if (PRO == kGate && which == 0) u.ask(a.u, a.ldu, a.u_aligned, s.u, a, r, step, c);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (r + i * step >= a.rows || c >= a.cols) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = 0.0f;
            continue;
        }
        x.take(a.x, a.ldx, a.x_aligned, s.x, a, r, step, c, i, v[i]);
        if (!Z) continue;
        float zv[8], uv[8];
        z.take(a.z, a.ldz, a.z_aligned, s.z, a, r, step, c, Z ? i : 0, zv);
        if (PRO == kGate && which == 0) u.take(a.u, a.ldu, a.u_aligned, s.u, a, r, step, c, PRO == kGate ? i : 0, uv);
        float f[8], slope[8];
        if (PRO == kGate && which) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                act_slope_exact<ACT>(zv[j], f[j], slope[j]);
                v[i][j] *= f[j];
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                act_slope_exact<ACT>(zv[j], f[j], slope[j]);
                v[i][j] = PRO == kGate ? v[i][j] * uv[j] * slope[j] : v[i][j] * slope[j];
            }
        }
        if (c + 8 <= a.cols) continue;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (c + j >= a.cols) v[i][j] = 0.0f;  // (the slope there may be 0 times an infinity)
    }
}

SADMM_DEV void store_scale(const sadmm_q8_out& o, long long r, long long b, float s) { o.s[r * o.s_row + b * o.s_block] = s; }

constexpr int kRowSteps = 4;  // column blocks of a half warp

// Blocks of one row, the matrix alone: a half warp takes four neighbouring blocks
// of a row, a lane 8 values of each.
template <int ES>
__global__ void __launch_bounds__(256) k_q8_rows(const Args a)
{
    pdl_wait();
    pdl_trigger();
    const long long groups = (a.col_tiles + kRowSteps - 1) / kRowSteps;
    const long long rg = blockIdx.x / groups, cg = blockIdx.x - rg * groups;
    const long long r = rg * 16 + (threadIdx.x >> 4);
    const int lane = threadIdx.x & 15;
    const Spans s = spans_of<kPlain>(a);
    float v[kRowSteps][8];
    Raw8<ES> raw[kRowSteps];
    auto at = [&](int i) { return (cg * kRowSteps + i) * kQBlock + lane * 8; };
#pragma unroll
    for (int i = 0; i < kRowSteps; ++i) {
        const bool in = r < a.rows && at(i) < a.cols && dbg_in(r, a.rows, a.status) && dbg_in(at(i), a.cols, a.status);
        ask8(static_cast<const uint8_t*>(a.x) + (in ? (r * a.ldx + at(i)) * ES : 0), in, a.x_aligned, s.x, raw[i]);
    }
#pragma unroll
    for (int i = 0; i < kRowSteps; ++i)
        take8(static_cast<const uint8_t*>(a.x) + (r * a.ldx + at(i)) * ES, (int)min(8ll, a.cols - at(i)), a.x_aligned, s.x,
              raw[i], v[i]);
    float top[kRowSteps];
    Q8Scale scale[kRowSteps];
#pragma unroll
    for (int i = 0; i < kRowSteps; ++i) top[i] = q8_top(v[i]);
    scales16(top, scale);
#pragma unroll
    for (int i = 0; i < kRowSteps; ++i) {
        const long long b = cg * kRowSteps + i, c = b * kQBlock + lane * 8;
        const Q8Scale k = scale[i];
        if (r >= a.rows || c >= a.cols || !dbg_in(r, a.rows, a.status) || !dbg_in(c, a.cols, a.status)) continue;
        if (lane == 0) store_scale(a.out[0], r, b, k.s);
        store_bytes8(static_cast<uint8_t*>(a.out[0].q) + r * a.out[0].ld + c, (int)min(8ll, a.cols - c),
                     q8_four(v[i][0], v[i][1], v[i][2], v[i][3], k), q8_four(v[i][4], v[i][5], v[i][6], v[i][7], k));
    }
}

// A tile of 128 x 128 a CTA.  A half warp takes a row (a lane 8 columns), so that a
// row's block is quantised as it comes (with `tile` after the whole tile has); the values
// also go to shared memory, where the transpose's blocks are read: a thread a column, 16
// rows at a time.  Loops of few rows: unrolled over the
// tile, the instructions came from memory (no instruction to issue for a third of the time).
template <int PRO, int ACT, int ES, bool AL>
__global__ void __launch_bounds__(256, AL ? 3 : 2) k_q8_tile(const Args a)
{
    constexpr int U = PRO == kGate || (PRO == kSlope && ACT != SADMM_ACT_NONE) ? 2 : 4;  // rows whose loads are in flight together
    extern __shared__ __align__(16) float vals[];  // [128][128]
    __shared__ float red[8][kQBlock], sums[PRO == kPlain ? 1 : 8][PRO == kPlain ? 1 : kQBlock], top_s[kQBlock];
    pdl_wait();
    pdl_trigger();
    const int hw = threadIdx.x >> 4, lane = threadIdx.x & 15, col = lane * 8;
    // every other four lanes' two 16 bytes change places: eight of them meet no bank twice
    const int late = lane >> 2 & 1;
    const int which = PRO == kGate ? blockIdx.x & 1 : 0;  // (the CTAs of dg and du of a tile run side by side)
    const long long at = PRO == kGate ? blockIdx.x >> 1 : blockIdx.x;
    const long long rt = at / a.col_tiles, ct = at - rt * a.col_tiles;
    const long long r0 = rt * kQBlock, c0 = ct * kQBlock;
    const Spans s = spans_of<PRO>(a);
    const int live = (int)max(0ll, min(8ll, a.cols - c0 - col));  // the lane's columns inside the matrix
    const int rows = (int)min((long long)kQBlock, a.rows - r0);    // the tile's
    auto put_row = [&](const sadmm_q8_out& o, int row, const Q8Scale& k, const float (&v)[8]) {
        const long long r = r0 + row;
        if (row >= rows || live == 0 || !dbg_in(r, a.rows, a.status) || !dbg_run(c0 + col, live, a.cols, a.status)) return;
        if (!a.tile && lane == 0) store_scale(o, r, ct, k.s);
        store_bytes8(static_cast<uint8_t*>(o.q) + r * o.ld + c0 + col, live, q8_four(v[0], v[1], v[2], v[3], k),
                     q8_four(v[4], v[5], v[6], v[7], k));
    };
    const sadmm_q8_out &o = a.out[which], &ot = a.out_t[which];
    const bool keep = ot.q || a.tile;
    float top[8], sum[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) top[j] = sum[j] = 0.0f;
#pragma unroll 1
    for (int i = 0; i < 8; i += U) {
        float v[U][8];
        load_source<PRO, ACT, ES, U, AL>(a, s, which, r0 + i * 16 + hw, 16, c0 + col, v);
        float row_top[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int row = (i + u) * 16 + hw;
            if (PRO != kPlain) {
#pragma unroll
                for (int j = 0; j < 8; ++j) sum[j] += v[u][j];
            }
            row_top[u] = q8_top(v[u]);
#pragma unroll
            for (int j = 0; j < 8; ++j) top[j] = fmaxf(top[j], fabsf(v[u][j]));
            if (keep) {
                float4* to = reinterpret_cast<float4*>(vals + row * kQBlock + col);
                to[late] = make_float4(v[u][0], v[u][1], v[u][2], v[u][3]);
                to[late ^ 1] = make_float4(v[u][4], v[u][5], v[u][6], v[u][7]);
            }
        }
        if (!a.tile && o.q) {
            Q8Scale k[U];
            scales16(row_top, k);
#pragma unroll
            for (int u = 0; u < U; ++u) put_row(o, (i + u) * 16 + hw, k[u], v[u]);
        }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        top[j] = fmaxf(top[j], __shfl_xor_sync(0xffffffffu, top[j], 16));
        if (PRO != kPlain) sum[j] += __shfl_xor_sync(0xffffffffu, sum[j], 16);
        if (hw & 1) continue;
        red[hw >> 1][col + j] = top[j];
        if (PRO != kPlain) sums[PRO == kPlain ? 0 : hw >> 1][PRO == kPlain ? 0 : col + j] = sum[j];
    }
    __syncthreads();
    if (threadIdx.x < kQBlock) {
        float t = 0.0f;
#pragma unroll
        for (int w = 0; w < 8; ++w) t = fmaxf(t, red[w][threadIdx.x]);
        top_s[threadIdx.x] = t;
        if (PRO != kPlain && a.part[which] && c0 + threadIdx.x < a.cols) {
            float p = 0.0f;
#pragma unroll
            for (int w = 0; w < 8; ++w) p += sums[PRO == kPlain ? 0 : w][PRO == kPlain ? 0 : threadIdx.x];
            a.part[which][rt * a.cols + c0 + threadIdx.x] = p;
        }
    }
    if (keep) {
        __syncthreads();
        Q8Scale tile = {};
        if (a.tile) {
            float t = 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j) t = fmaxf(t, top_s[(threadIdx.x & 31) * 4 + j]);
#pragma unroll
            for (int d = 16; d; d >>= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, d));
            tile = q8_scale(t);
            if (threadIdx.x == 0) {
                if (o.q) store_scale(o, rt, ct, tile.s);
                if (ot.q) store_scale(ot, ct, rt, tile.s);
            }
            if (o.q) {
#pragma unroll 2
                for (int row = hw; row < kQBlock; row += 16) {
                    const float4* from = reinterpret_cast<const float4*>(vals + row * kQBlock + col);
                    const float4 x = from[late], y = from[late ^ 1];
                    const float v[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
                    put_row(o, row, tile, v);
                }
            }
        }
        if (ot.q) {
            const int c = threadIdx.x & 127;
            const Q8Scale k = a.tile ? tile : q8_scale(top_s[c]);
            const bool in = c0 + c < a.cols && dbg_in(c0 + c, a.cols, a.status);
            if (!a.tile && in && threadIdx.x < kQBlock) store_scale(ot, c0 + c, rt, k.s);
            uint8_t* to = static_cast<uint8_t*>(ot.q) + (in ? (c0 + c) * ot.ld : 0) + r0;
#pragma unroll 1
            for (int row = (threadIdx.x >> 7) * 16; row < kQBlock; row += 32) {
                uint32_t w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float* f = vals + (row + 4 * i) * kQBlock + (c ^ (c >> 5 & 1) << 2);
                    w[i] = q8_four(f[0], f[kQBlock], f[2 * kQBlock], f[3 * kQBlock], k);
                }
                const int n = (int)min(16ll, a.rows - r0 - row);
                if (!in || n <= 0 || !dbg_run(r0 + row, n, a.rows, a.status)) continue;
                if (n == 16 && (reinterpret_cast<uintptr_t>(to + row) & 15) == 0) {
                    *reinterpret_cast<uint4*>(to + row) = make_uint4(w[0], w[1], w[2], w[3]);
                } else {
                    store_bytes8(to + row, n, w[0], w[1]);
                    store_bytes8(to + row + 8, n - 8, w[2], w[3]);
                }
            }
        }
    }
}

// out[c] = the sum of part[0 .. parts-1][c] in the order of 32 groups of parts, then of
// the groups.  blockIdx.y: which output.
__global__ void __launch_bounds__(1024) k_q8_sums(const float* __restrict__ part0, const float* __restrict__ part1,
                                                  float* __restrict__ out0, float* __restrict__ out1, long long cols,
                                                  long long parts)
{
    __shared__ float red[32][33];
    pdl_wait();
    pdl_trigger();
    const float* part = blockIdx.y ? part1 : part0;
    float* out = blockIdx.y ? out1 : out0;
    if (!out) return;
    const int g = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long long c = blockIdx.x * 32ll + lane;
    float v = 0.0f;
    if (c < cols) {
#pragma unroll 8
        for (long long k = g; k < parts; k += 32) v += part[k * cols + c];
    }
    red[g][lane] = v;
    __syncthreads();
    v = red[lane][g];
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    const long long at = blockIdx.x * 32ll + g;
    if (lane == 0 && at < cols) out[at] = v;
}

template <int PRO, int ACT, int ES, bool AL>
cudaError_t launch_tiles(const Args& a, long long grid, cudaStream_t s)
{
    static bool configured[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    constexpr int smem = kQBlock * kQBlock * 4;
    auto kern = k_q8_tile<PRO, ACT, ES, AL>;
    if (!configured[dev]) {
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != cudaSuccess) return e;
        configured[dev] = true;
    }
    return launch_pdl(kern, dim3((unsigned)grid), dim3(256), smem, s, a);
}
template <int PRO, int ACT, int ES>
cudaError_t launch_tiles(const Args& a, bool al, long long grid, cudaStream_t s)
{
    return al ? launch_tiles<PRO, ACT, ES, true>(a, grid, s) : launch_tiles<PRO, ACT, ES, false>(a, grid, s);
}
template <int PRO, int ES>
cudaError_t launch_tiles(const Args& a, int act, bool al, long long grid, cudaStream_t s)
{
    switch (act) {
    case SADMM_ACT_RELU: return launch_tiles<PRO, SADMM_ACT_RELU, ES>(a, al, grid, s);
    case SADMM_ACT_GELU: return launch_tiles<PRO, SADMM_ACT_GELU, ES>(a, al, grid, s);
    case SADMM_ACT_SILU: return launch_tiles<PRO, SADMM_ACT_SILU, ES>(a, al, grid, s);
    default: return launch_tiles<PRO, SADMM_ACT_NONE, ES>(a, al, grid, s);
    }
}

}  // namespace

size_t q8_source_bytes(const Q8Source& a)
{
    const size_t one = (size_t)((a.rows + kQBlock - 1) / kQBlock) * (size_t)a.cols * 4;
    return round_up(one, 256) * ((a.sums[0] != nullptr) + (a.sums[1] != nullptr));
}

sadmm_status launch_q8_source(const Q8Source& q, void* ws, cudaStream_t s)
{
    Args a = {};
    a.x = q.x, a.u = q.u, a.z = q.u || q.act != SADMM_ACT_NONE ? q.z : nullptr;
    a.ldx = q.ldx, a.ldz = q.ldz, a.ldu = q.ldu;
    a.xdt = q.xdt, a.act = q.act, a.tile = q.tile;
    a.rows = q.rows, a.cols = q.cols;
    a.row_tiles = (q.rows + kQBlock - 1) / kQBlock;
    a.col_tiles = (q.cols + kQBlock - 1) / kQBlock;
    a.status = device_status_ptr();
    uint8_t* at = static_cast<uint8_t*>(ws);
    for (int i = 0; i < 2; ++i) {
        a.out[i] = q.out[i];
        a.out_t[i] = q.out_t[i];
        if (q.sums[i]) {
            a.part[i] = reinterpret_cast<float*>(at);
            at += round_up((size_t)a.row_tiles * (size_t)q.cols * 4, 256);
        }
    }
    auto aligned = [](const void* p, long long ld, int es) {
        return ((reinterpret_cast<uintptr_t>(p) | (uintptr_t)(ld * es)) & 15) == 0;
    };
    const bool fp32 = q.xdt == SADMM_FP32;
    a.x_aligned = aligned(a.x, a.ldx, fp32 ? 4 : 2);
    a.z_aligned = !a.z || aligned(a.z, a.ldz, 2);
    a.u_aligned = !a.u || aligned(a.u, a.ldu, 2);
    const bool al = a.x_aligned && a.z_aligned && a.u_aligned;
    cudaError_t err;
    if (!a.z && !q.tile && !q.out_t[0].q && !q.sums[0]) {
        const long long grid = (q.rows + 15) / 16 * ((a.col_tiles + kRowSteps - 1) / kRowSteps);
        if (grid > 0x7fffffffll) return SADMM_EUNSUPPORTED;
        err = launch_pdl(fp32 ? k_q8_rows<4> : k_q8_rows<2>, dim3((unsigned)grid), dim3(256), 0, s, a);
    } else {
        const long long grid = a.row_tiles * a.col_tiles * (q.u ? 2 : 1);
        if (grid > 0x7fffffffll) return SADMM_EUNSUPPORTED;
        const int act = a.z ? a.act : SADMM_ACT_NONE;
        if (q.u)
            err = launch_tiles<kGate, 2>(a, act, al, grid, s);
        else if (a.z || q.sums[0])
            err = fp32 ? launch_tiles<kSlope, 4>(a, act, al, grid, s) : launch_tiles<kSlope, 2>(a, act, al, grid, s);
        else
            err = fp32 ? launch_tiles<kPlain, SADMM_ACT_NONE, 4>(a, al, grid, s)
                       : launch_tiles<kPlain, SADMM_ACT_NONE, 2>(a, al, grid, s);
    }
    if (err == cudaSuccess && (q.sums[0] || q.sums[1]))
        err = launch_pdl(k_q8_sums, dim3((unsigned)((q.cols + 31) / 32), 2), dim3(1024), 0, s, a.part[0], a.part[1],
                         q.sums[0], q.sums[1], q.cols, a.row_tiles);
    return err == cudaSuccess ? SADMM_OK : SADMM_ECUDA;
}

sadmm_status launch_quantize(const sadmm_quantize_args& a, cudaStream_t s)
{
    Q8Source q = {};
    q.x = a.x, q.ldx = a.ldx, q.xdt = a.xdt;
    q.rows = a.rows, q.cols = a.cols, q.tile = a.tile;
    q.out[0] = a.out, q.out_t[0] = a.out_t;
    return launch_q8_source(q, nullptr, s);
}

}  // namespace sadmm
