// quant.cu -- matrices in 8 bits: e4m3 values with an fp32 scale for each block
// of 128 columns of a row (or 128 x 128), of a matrix and of its transpose, in one
// pass over the source.  The source is a matrix, or what a backward pass has
// to make 8-bit: dy act'(z), or the gated pair's dg = dh u act'(g) and
// du = dh act(g), whose column sums (the bias's gradient) are taken on the way.
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
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float f, slope;
            act_slope_f32<ACT>(zv[j], f, slope);
            if (PRO == kGate)
                v[i][j] = which ? v[i][j] * f : v[i][j] * uv[j] * slope;
            else
                v[i][j] *= slope;
            if (c + j >= a.cols) v[i][j] = 0.0f;  // (the slope there may be 0 times an infinity)
        }
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
#pragma unroll
    for (int i = 0; i < kRowSteps; ++i) {
        const long long b = cg * kRowSteps + i, c = b * kQBlock + lane * 8;
        float top = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) top = fmaxf(top, q8_size(v[i][j]));
        const Q8Scale k = q8_scale(max16(top));
        if (r >= a.rows || c >= a.cols || !dbg_in(r, a.rows, a.status) || !dbg_in(c, a.cols, a.status)) continue;
        if (lane == 0) store_scale(a.out[0], r, b, k.s);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = q8_quotient(v[i][j], k);
        store_bytes8(static_cast<uint8_t*>(a.out[0].q) + r * a.out[0].ld + c, (int)min(8ll, a.cols - c),
                     q8_four(v[i][0], v[i][1], v[i][2], v[i][3]), q8_four(v[i][4], v[i][5], v[i][6], v[i][7]));
    }
}

// A tile of 128 x 128 a CTA: warp w's half h takes rows 16 w + 8 h ... + 7, a lane 8
// columns of them, so that it holds 8 x 8 values.  The transpose goes through shared
// memory in 8-byte words of 8 rows of a column, at word (row / 8) ^ (column / 8) of the
// column's 16, so that neither side meets a bank twice.
template <int PRO, int ACT, int ES, bool AL>
__global__ void __launch_bounds__(256, 2) k_q8_tile(const Args a)
{
    __shared__ __align__(16) uint2 turned[kQBlock][16];
    __shared__ float red[8][kQBlock], col_top[kQBlock], sums[8][kQBlock];
    pdl_wait();
    pdl_trigger();
    const int warp = threadIdx.x >> 5, half = (threadIdx.x >> 4) & 1, lane = threadIdx.x & 15;
    const long long rt = blockIdx.x / a.col_tiles, ct = blockIdx.x - rt * a.col_tiles;
    const long long r0 = rt * kQBlock, c0 = ct * kQBlock;
    const int row0 = warp * 16 + half * 8, col = lane * 8;
    const Spans s = spans_of<PRO>(a);
    for (int which = 0; which < (PRO == kGate ? 2 : 1); ++which) {
        const sadmm_q8_out &o = a.out[which], &ot = a.out_t[which];
        float v[8][8];
        constexpr int N = PRO == kPlain ? 8 : PRO == kSlope ? 4 : 2;  // rows whose loads are in flight together
#pragma unroll
        for (int i = 0; i < 8; i += N)
            load_source<PRO, ACT, ES, N, AL>(a, s, which, r0 + row0 + i, 1, c0 + col, v + i);
        float top[8];  // of the lane's columns
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            top[j] = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) top[j] = fmaxf(top[j], q8_size(v[i][j]));
        }
        if (PRO != kPlain && a.part[which]) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float p = 0.0f;
#pragma unroll
                for (int i = 0; i < 8; ++i) p += v[i][j];
                p += __shfl_xor_sync(0xffffffffu, p, 16);
                if (half == 0) sums[warp][col + j] = p;
            }
        }
        Q8Scale tile = {1.0f, 1.0f};
        if (a.tile || ot.q) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float t = fmaxf(top[j], __shfl_xor_sync(0xffffffffu, top[j], 16));
                if (half == 0) red[warp][col + j] = t;
            }
            __syncthreads();
            if (threadIdx.x < kQBlock) {
                float t = 0.0f;
#pragma unroll
                for (int w = 0; w < 8; ++w) t = fmaxf(t, red[w][threadIdx.x]);
                col_top[threadIdx.x] = t;
            }
            __syncthreads();
            if (a.tile) {
                float t = 0.0f;
                for (int j = 0; j < 4; ++j) t = fmaxf(t, col_top[(threadIdx.x & 31) * 4 + j]);
#pragma unroll
                for (int d = 16; d; d >>= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, d));
                tile = q8_scale(t);
                if (threadIdx.x == 0) {
                    if (o.q) store_scale(o, rt, ct, tile.s);
                    if (ot.q) store_scale(ot, ct, rt, tile.s);
                }
            }
        } else if (PRO != kPlain && a.part[which]) {
            __syncthreads();
        }
        if (PRO != kPlain && a.part[which] && threadIdx.x < kQBlock && c0 + threadIdx.x < a.cols) {
            float p = 0.0f;
#pragma unroll
            for (int w = 0; w < 8; ++w) p += sums[w][threadIdx.x];
            a.part[which][rt * a.cols + c0 + threadIdx.x] = p;
        }
        if (o.q) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const long long r = r0 + row0 + i;
                Q8Scale k = tile;
                if (!a.tile) {
                    float t = 0.0f;
#pragma unroll
                    for (int j = 0; j < 8; ++j) t = fmaxf(t, q8_size(v[i][j]));
                    k = q8_scale(max16(t));
                }
                if (r >= a.rows || c0 + col >= a.cols || !dbg_in(r, a.rows, a.status) ||
                    !dbg_in(c0 + col, a.cols, a.status))
                    continue;
                if (!a.tile && lane == 0) store_scale(o, r, ct, k.s);
                float q[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) q[j] = q8_quotient(v[i][j], k);
                store_bytes8(static_cast<uint8_t*>(o.q) + r * o.ld + c0 + col, (int)min(8ll, a.cols - c0 - col),
                             q8_four(q[0], q[1], q[2], q[3]), q8_four(q[4], q[5], q[6], q[7]));
            }
        }
        if (ot.q) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const Q8Scale k = a.tile ? tile : q8_scale(col_top[col + j]);
                if (!a.tile && row0 == 0 && c0 + col + j < a.cols) store_scale(ot, c0 + col + j, rt, k.s);
                float q[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) q[i] = q8_quotient(v[i][j], k);
                turned[col + j][(warp * 2 + half) ^ lane] =
                    make_uint2(q8_four(q[0], q[1], q[2], q[3]), q8_four(q[4], q[5], q[6], q[7]));
            }
            __syncthreads();
            const int n = (int)min(8ll, a.rows - r0 - lane * 8);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int c = (threadIdx.x >> 4) * 8 + i;
                const uint2 w = turned[c][lane ^ (c >> 3)];
                if (c0 + c >= a.cols || n <= 0 || !dbg_in(c0 + c, a.cols, a.status) ||
                    !dbg_in(r0 + lane * 8, a.rows, a.status))
                    continue;
                store_bytes8(static_cast<uint8_t*>(ot.q) + (c0 + c) * ot.ld + r0 + lane * 8, n, w.x, w.y);
            }
        }
        if (PRO == kGate) __syncthreads();  // shared memory is written again
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

using TileKernel = void (*)(const Args);

template <int PRO, int ES>
TileKernel tile_kernel(int act, bool al)
{
    switch (act) {
    case SADMM_ACT_RELU: return al ? k_q8_tile<PRO, SADMM_ACT_RELU, ES, true> : k_q8_tile<PRO, SADMM_ACT_RELU, ES, false>;
    case SADMM_ACT_GELU: return al ? k_q8_tile<PRO, SADMM_ACT_GELU, ES, true> : k_q8_tile<PRO, SADMM_ACT_GELU, ES, false>;
    case SADMM_ACT_SILU: return al ? k_q8_tile<PRO, SADMM_ACT_SILU, ES, true> : k_q8_tile<PRO, SADMM_ACT_SILU, ES, false>;
    default: return al ? k_q8_tile<PRO, SADMM_ACT_NONE, ES, true> : k_q8_tile<PRO, SADMM_ACT_NONE, ES, false>;
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
        const long long grid = a.row_tiles * a.col_tiles;
        if (grid > 0x7fffffffll) return SADMM_EUNSUPPORTED;
        TileKernel kern;
        if (q.u)
            kern = tile_kernel<kGate, 2>(a.act, al);
        else if (a.z || q.sums[0])
            kern = fp32 ? tile_kernel<kSlope, 4>(a.z ? a.act : SADMM_ACT_NONE, al) : tile_kernel<kSlope, 2>(a.z ? a.act : SADMM_ACT_NONE, al);
        else
            kern = fp32 ? (al ? k_q8_tile<kPlain, SADMM_ACT_NONE, 4, true> : k_q8_tile<kPlain, SADMM_ACT_NONE, 4, false>)
                        : (al ? k_q8_tile<kPlain, SADMM_ACT_NONE, 2, true> : k_q8_tile<kPlain, SADMM_ACT_NONE, 2, false>);
        err = launch_pdl(kern, dim3((unsigned)grid), dim3(256), 0, s, a);
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
