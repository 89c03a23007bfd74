// abi_q8.cu -- the extern "C" entry points of the feed-forward operators with
// 8-bit operands (RMS norm, quantiser, linear, gated pair): host-side validation,
// then the launches.  Nothing is enqueued before every argument has been checked.
#include <math.h>

#include "checks.h"
#include "internal.h"

namespace sadmm {
namespace {

constexpr long long kMostStride = 1ll << 38;

// An 8-bit operand of `cols` columns: present, rows at least as far apart as they are long.
bool q8(const sadmm_q8& m, long long cols)
{
    return m.q && m.ld >= cols && m.ld < kMostStride && m.s && vec32(m.s) && m.s_row >= 0 && m.s_block >= 0 &&
           m.s_row < kMostStride && m.s_block < kMostStride;
}

// An 8-bit output: as above, and every scale has a place of its own.  rows: of scales.
bool q8_out(const sadmm_q8_out& m, long long rows, long long cols)
{
    const long long blocks = (cols + 127) / 128;
    if (!m.q || m.ld < cols || m.ld >= kMostStride || !m.s || !vec32(m.s)) return false;
    if (m.s_row < 0 || m.s_block < 0 || m.s_row >= kMostStride || m.s_block >= kMostStride) return false;
    if ((rows > 1 && m.s_row < 1) || (blocks > 1 && m.s_block < 1)) return false;
    if (rows <= 1 || blocks <= 1) return true;
    return m.s_block > (rows - 1) * m.s_row || m.s_row > (blocks - 1) * m.s_block;
}

sadmm_status check(const sadmm_rmsnorm_fwd_args* a)
{
    if (!a || !is_dtype(a->xdt) || !(a->eps >= 0.0f) || isinf(a->eps)) return SADMM_EINVAL;
    const bool eight = a->ydt == SADMM_E4M3;
    if (!eight && !is_dtype(a->ydt)) return SADMM_EINVAL;
    const sadmm_status st = extents(a->rows, a->cols, 1);
    if (st != SADMM_OK) return st;
    if (!vec32(a->gamma) || !vec32(a->rstd)) return SADMM_EINVAL;
    if (!a->rows) return SADMM_OK;
    if (!matrix(a->x, a->xdt, a->ldx, a->cols) || !matrix_or_null(a->residual, a->rdt, a->ldr, a->cols) ||
        !matrix_or_null(a->h, a->rdt, a->ldh, a->cols))
        return SADMM_EINVAL;
    if (a->h && !a->residual) return SADMM_EINVAL;
    if (eight ? !q8_out(a->y8, a->rows, a->cols) : !matrix(a->y, a->ydt, a->ldy, a->cols)) return SADMM_EINVAL;
    const void* y = eight ? a->y8.q : a->y;
    const void* s = eight ? a->y8.s : nullptr;
    if (!distinct({a->h, y, s, a->rstd}, {a->gamma}) || !distinct({y, s, a->rstd}, {a->residual}) ||
        !distinct({s, a->rstd}, {a->x}))
        return SADMM_EINVAL;
    if (a->h && a->h == a->residual && !in_place(a->h, a->ldh, a->residual, a->ldr, a->rows)) return SADMM_EINVAL;
    if (a->h && a->h == a->x && (a->rdt != a->xdt || !in_place(a->h, a->ldh, a->x, a->ldx, a->rows))) return SADMM_EINVAL;
    if (y == a->x && (a->ydt != a->xdt || !in_place(a->y, a->ldy, a->x, a->ldx, a->rows))) return SADMM_EINVAL;
    return SADMM_OK;
}

sadmm_status check(const sadmm_rmsnorm_bwd_args* a)
{
    if (!a || !is_dtype(a->hdt) || !is_dtype(a->dydt)) return SADMM_EINVAL;
    const sadmm_status st = extents(a->rows, a->cols, 1);
    if (st != SADMM_OK) return st;
    if (!vec32(a->gamma) || !vec32(a->rstd) || !vec32(a->dgamma)) return SADMM_EINVAL;
    if (!a->rows) return SADMM_OK;
    if ((!a->dx && !a->dgamma) || (a->dres && !a->dx)) return SADMM_EINVAL;
    if (!a->rstd || !matrix(a->h, a->hdt, a->ldh, a->cols) || !matrix(a->dy, a->dydt, a->lddy, a->cols) ||
        !matrix_or_null(a->dres, a->hdt, a->lddres, a->cols) || !matrix_or_null(a->dx, a->hdt, a->lddx, a->cols))
        return SADMM_EINVAL;
    if (!distinct({a->dx, a->dgamma}, {a->h, a->dy, a->gamma, a->rstd}) || !distinct({a->dgamma}, {a->dres}))
        return SADMM_EINVAL;
    if (a->dres && !in_place(a->dx, a->lddx, a->dres, a->lddres, a->rows)) return SADMM_EINVAL;
    return SADMM_OK;
}

sadmm_status check(const sadmm_quantize_args* a)
{
    if (!a || !is_dtype(a->xdt)) return SADMM_EINVAL;
    const sadmm_status st = extents(a->rows, a->cols, 1);
    if (st != SADMM_OK) return st;
    if (!a->out.q && !a->out_t.q) return a->rows ? SADMM_EINVAL : SADMM_OK;
    if (!a->rows) return SADMM_OK;
    const int high = a->tile ? 128 : 1;
    if (!matrix(a->x, a->xdt, a->ldx, a->cols)) return SADMM_EINVAL;
    if (a->out.q && !q8_out(a->out, (a->rows + high - 1) / high, a->cols)) return SADMM_EINVAL;
    if (a->out_t.q && !q8_out(a->out_t, (a->cols + high - 1) / high, a->rows)) return SADMM_EINVAL;
    const void* s = a->out.q ? a->out.s : nullptr;
    const void* st_ = a->out_t.q ? a->out_t.s : nullptr;
    return distinct({a->out.q, a->out_t.q, s, st_}, {a->x}) ? SADMM_OK : SADMM_EINVAL;
}

sadmm_status check(const sadmm_linear8_fwd_args* a)
{
    if (!a || !is_act(a->act) || !is_dtype(a->ydt)) return SADMM_EINVAL;
    const sadmm_status st = extents(a->tokens, a->n_in, a->n_out);
    if (st != SADMM_OK) return st;
    if (!q8(a->w, a->n_in) || !vec32(a->bias)) return SADMM_EINVAL;
    if (!a->tokens) return SADMM_OK;
    if (!q8(a->x, a->n_in) || !matrix(a->y, a->ydt, a->ldy, a->n_out) ||
        !matrix_or_null(a->residual, a->ydt, a->ldr, a->n_out) || !matrix_or_null(a->z, SADMM_BF16, a->ldz, a->n_out))
        return SADMM_EINVAL;
    if (!distinct({a->y, a->z}, {a->x.q, a->x.s, a->w.q, a->w.s, a->bias}) || !distinct({a->z}, {a->residual}))
        return SADMM_EINVAL;
    if (!in_place(a->y, a->ldy, a->residual, a->ldr, a->tokens)) return SADMM_EINVAL;
    return SADMM_OK;
}

sadmm_status check(const sadmm_linear8_bwd_args* a)
{
    if (!a || !is_act(a->act) || !is_dtype(a->dydt)) return SADMM_EINVAL;
    const sadmm_status st = extents(a->tokens, a->n_in, a->n_out);
    if (st != SADMM_OK) return st;
    if (!vec32(a->db) || !matrix_or_null(a->dw, a->dwdt, a->lddw, a->n_in)) return SADMM_EINVAL;
    if (!a->tokens) return SADMM_OK;
    if (!a->dx && !a->dw && !a->db) return SADMM_EINVAL;
    if (!matrix(a->dy, a->dydt, a->lddy, a->n_out) || !matrix_or_null(a->dx, a->dxdt, a->lddx, a->n_in))
        return SADMM_EINVAL;
    if (a->act != SADMM_ACT_NONE && !matrix(a->z, SADMM_BF16, a->ldz, a->n_out)) return SADMM_EINVAL;
    if ((a->dx && !q8(a->wt, a->n_out)) || (a->dw && !q8(a->xt, a->tokens))) return SADMM_EINVAL;
    if (!distinct({a->dx, a->dw, a->db}, {a->dy, a->xt.q, a->xt.s, a->wt.q, a->wt.s})) return SADMM_EINVAL;
    if (a->act != SADMM_ACT_NONE && !distinct({a->dx, a->dw, a->db}, {a->z})) return SADMM_EINVAL;
    return SADMM_OK;
}

sadmm_status check(const sadmm_gated8_fwd_args* a)
{
    if (!a || !is_act(a->act) || (a->hdt != SADMM_E4M3 && a->hdt != SADMM_BF16)) return SADMM_EINVAL;
    const sadmm_status st = extents(a->tokens, a->n_in, a->n_hidden);
    if (st != SADMM_OK) return st;
    if (!q8(a->wg, a->n_in) || !q8(a->wu, a->n_in) || !vec32(a->bg) || !vec32(a->bu)) return SADMM_EINVAL;
    if (!a->tokens) return SADMM_OK;
    const bool eight = a->hdt == SADMM_E4M3;
    if (!q8(a->x, a->n_in) ||
        (eight ? !q8_out(a->h8, a->tokens, a->n_hidden) : !matrix(a->h, SADMM_BF16, a->ldh, a->n_hidden)) ||
        !matrix_or_null(a->g, SADMM_BF16, a->ldg, a->n_hidden) || !matrix_or_null(a->u, SADMM_BF16, a->ldu, a->n_hidden))
        return SADMM_EINVAL;
    const void* h = eight ? a->h8.q : a->h;
    const void* s = eight ? a->h8.s : nullptr;
    return distinct({h, s, a->g, a->u}, {a->x.q, a->x.s, a->wg.q, a->wg.s, a->wu.q, a->wu.s, a->bg, a->bu}) ? SADMM_OK
                                                                                                         : SADMM_EINVAL;
}

sadmm_status check(const sadmm_gated8_bwd_args* a)
{
    if (!a || !is_act(a->act)) return SADMM_EINVAL;
    const sadmm_status st = extents(a->tokens, a->n_in, a->n_hidden);
    if (st != SADMM_OK) return st;
    if (!vec32(a->dbg) || !vec32(a->dbu) || !a->dwg != !a->dwu) return SADMM_EINVAL;
    if (!matrix_or_null(a->dwg, a->dwdt, a->lddwg, a->n_in) || !matrix_or_null(a->dwu, a->dwdt, a->lddwu, a->n_in))
        return SADMM_EINVAL;
    if (!a->tokens) return SADMM_OK;
    if (!a->dx && !a->dwg && !a->dbg && !a->dbu) return SADMM_EINVAL;
    if (!matrix(a->dh, SADMM_BF16, a->lddh, a->n_hidden) || !matrix(a->g, SADMM_BF16, a->ldg, a->n_hidden) ||
        !matrix(a->u, SADMM_BF16, a->ldu, a->n_hidden) || !matrix_or_null(a->dx, a->dxdt, a->lddx, a->n_in))
        return SADMM_EINVAL;
    if (a->dx && (!q8(a->wgt, a->n_hidden) || !q8(a->wut, a->n_hidden))) return SADMM_EINVAL;
    if (a->dwg && !q8(a->xt, a->tokens)) return SADMM_EINVAL;
    return distinct({a->dx, a->dwg, a->dwu, a->dbg, a->dbu},
                    {a->dh, a->xt.q, a->xt.s, a->wgt.q, a->wgt.s, a->wut.q, a->wut.s, a->g, a->u})
               ? SADMM_OK
               : SADMM_EINVAL;
}

// A product's call: checked arguments, scratch, a device that has the instructions.
template <typename A>
sadmm_status call(const A* a, size_t (*bytes)(const A&), sadmm_status (*launch)(const A&, void*, cudaStream_t),
                  void* workspace, size_t ws_bytes, void* stream)
{
    const sadmm_status st = check(a);
    if (st != SADMM_OK) return st;
    if (!scratch(workspace, ws_bytes, bytes(*a))) return SADMM_EINVAL;
    if (device_cc_major() < 10) return SADMM_EUNSUPPORTED;
    return launch(*a, workspace, static_cast<cudaStream_t>(stream));
}

}  // namespace
}  // namespace sadmm

using namespace sadmm;

extern "C" {

sadmm_status sadmm_rmsnorm_fwd(const sadmm_rmsnorm_fwd_args* a, void* stream)
{
    NvtxRange range("sadmm_rmsnorm_fwd");
    const sadmm_status st = check(a);
    if (st != SADMM_OK) return st;
    return launch_rmsnorm_fwd(*a, static_cast<cudaStream_t>(stream));
}

size_t sadmm_rmsnorm_bwd_workspace_size(const sadmm_rmsnorm_bwd_args* a)
{
    return check(a) == SADMM_OK ? rmsnorm_bwd_bytes(*a) : 0;
}

sadmm_status sadmm_rmsnorm_bwd(const sadmm_rmsnorm_bwd_args* a, void* workspace, size_t ws_bytes, void* stream)
{
    NvtxRange range("sadmm_rmsnorm_bwd");
    const sadmm_status st = check(a);
    if (st != SADMM_OK) return st;
    if (!scratch(workspace, ws_bytes, rmsnorm_bwd_bytes(*a))) return SADMM_EINVAL;
    return launch_rmsnorm_bwd(*a, workspace, static_cast<cudaStream_t>(stream));
}

sadmm_status sadmm_quantize(const sadmm_quantize_args* a, void* stream)
{
    NvtxRange range("sadmm_quantize");
    const sadmm_status st = check(a);
    if (st != SADMM_OK || !a->rows) return st;
    return launch_quantize(*a, static_cast<cudaStream_t>(stream));
}

size_t sadmm_linear8_fwd_workspace_size(const sadmm_linear8_fwd_args* a)
{
    return check(a) == SADMM_OK ? linear8_fwd_bytes(*a) : 0;
}

sadmm_status sadmm_linear8_fwd(const sadmm_linear8_fwd_args* a, void* workspace, size_t ws_bytes, void* stream)
{
    NvtxRange range("sadmm_linear8_fwd");
    return call(a, linear8_fwd_bytes, launch_linear8_fwd, workspace, ws_bytes, stream);
}

size_t sadmm_linear8_bwd_workspace_size(const sadmm_linear8_bwd_args* a)
{
    return check(a) == SADMM_OK ? linear8_bwd_bytes(*a) : 0;
}

sadmm_status sadmm_linear8_bwd(const sadmm_linear8_bwd_args* a, void* workspace, size_t ws_bytes, void* stream)
{
    NvtxRange range("sadmm_linear8_bwd");
    return call(a, linear8_bwd_bytes, launch_linear8_bwd, workspace, ws_bytes, stream);
}

size_t sadmm_gated8_fwd_workspace_size(const sadmm_gated8_fwd_args* a)
{
    return check(a) == SADMM_OK ? gated8_fwd_bytes(*a) : 0;
}

sadmm_status sadmm_gated8_fwd(const sadmm_gated8_fwd_args* a, void* workspace, size_t ws_bytes, void* stream)
{
    NvtxRange range("sadmm_gated8_fwd");
    return call(a, gated8_fwd_bytes, launch_gated8_fwd, workspace, ws_bytes, stream);
}

size_t sadmm_gated8_bwd_workspace_size(const sadmm_gated8_bwd_args* a)
{
    return check(a) == SADMM_OK ? gated8_bwd_bytes(*a) : 0;
}

sadmm_status sadmm_gated8_bwd(const sadmm_gated8_bwd_args* a, void* workspace, size_t ws_bytes, void* stream)
{
    NvtxRange range("sadmm_gated8_bwd");
    return call(a, gated8_bwd_bytes, launch_gated8_bwd, workspace, ws_bytes, stream);
}

}  // extern "C"
