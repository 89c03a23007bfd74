// output.cuh -- an output (or residual) matrix as the feed-forward kernels'
// epilogues address it.
#pragma once

#include "common.cuh"
#include "tgemm.cuh"

namespace sadmm {

// vec: 2 / 1 / 0 for rows on
// 32-byte / 16-byte / other boundaries.
struct Out {
    void* p;
    long long ld;
    long long total;  // elements from p to the end of the last row
    int bf16;
    int vec;
};

inline Out make_out(const TgMatrix& m, long long rows, long long cols)
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

}  // namespace sadmm
