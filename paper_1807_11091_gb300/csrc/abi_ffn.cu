// abi_ffn.cu -- the extern "C" entry points of the feed-forward operators
// (layer norm, linear, gated pair): host-side validation, then the launches.
// Nothing is enqueued before every argument has been checked.
#include <math.h>

#include "checks.h"
#include "internal.h"

namespace sadmm {
namespace {

sadmm_status check(const sadmm_layernorm_fwd_args* a)
{
    if (!a || !is_dtype(a->xdt) || !is_dtype(a->ydt) || !(a->eps >= 0.0f) || isinf(a->eps)) return SADMM_EINVAL;
    const sadmm_status st = extents(a->rows, a->cols, 1);
    if (st != SADMM_OK) return st;
    if (!vec32(a->gamma) || !vec32(a->beta) || !vec32(a->mean) || !vec32(a->rstd)) return SADMM_EINVAL;
    if (!a->rows) return SADMM_OK;
    if (!matrix(a->x, a->xdt, a->ldx, a->cols) || !matrix(a->y, a->ydt, a->ldy, a->cols)) return SADMM_EINVAL;
    if (!distinct({a->y, a->mean, a->rstd}, {a->gamma, a->beta}) || !distinct({a->mean, a->rstd}, {a->x}))
        return SADMM_EINVAL;
    if (a->y == a->x && (a->xdt != a->ydt || !in_place(a->y, a->ldy, a->x, a->ldx, a->rows))) return SADMM_EINVAL;
    return SADMM_OK;
}

sadmm_status check(const sadmm_layernorm_bwd_args* a)
{
    if (!a || !is_dtype(a->xdt) || !is_dtype(a->dydt)) return SADMM_EINVAL;
    const sadmm_status st = extents(a->rows, a->cols, 1);
    if (st != SADMM_OK) return st;
    if (!vec32(a->gamma) || !vec32(a->mean) || !vec32(a->rstd) || !vec32(a->dgamma) || !vec32(a->dbeta))
        return SADMM_EINVAL;
    if (!a->rows) return SADMM_OK;
    if (!a->dx && !a->dgamma && !a->dbeta) return SADMM_EINVAL;
    if (a->dres && !a->dx) return SADMM_EINVAL;
    if (!a->mean || !a->rstd || !matrix(a->x, a->xdt, a->ldx, a->cols) || !matrix(a->dy, a->dydt, a->lddy, a->cols) ||
        !matrix_or_null(a->dres, a->xdt, a->lddres, a->cols) || !matrix_or_null(a->dx, a->xdt, a->lddx, a->cols))
        return SADMM_EINVAL;
    if (!distinct({a->dx, a->dgamma, a->dbeta}, {a->x, a->dy, a->gamma, a->mean, a->rstd}) ||
        !distinct({a->dgamma, a->dbeta}, {a->dres}))
        return SADMM_EINVAL;
    if (a->dres && !in_place(a->dx, a->lddx, a->dres, a->lddres, a->rows)) return SADMM_EINVAL;
    return SADMM_OK;
}

sadmm_status check(const sadmm_linear_fwd_args* a)
{
    if (!a || !is_act(a->act) || !is_dtype(a->ydt)) return SADMM_EINVAL;
    const sadmm_status st = extents(a->tokens, a->n_in, a->n_out);
    if (st != SADMM_OK) return st;
    if (!matrix(a->w, SADMM_BF16, a->ldw, a->n_in) || !vec32(a->bias)) return SADMM_EINVAL;
    if (!a->tokens) return SADMM_OK;
    if (!matrix(a->x, SADMM_BF16, a->ldx, a->n_in) || !matrix(a->y, a->ydt, a->ldy, a->n_out) ||
        !matrix_or_null(a->residual, a->ydt, a->ldr, a->n_out) || !matrix_or_null(a->z, SADMM_BF16, a->ldz, a->n_out))
        return SADMM_EINVAL;
    if (!distinct({a->y, a->z}, {a->x, a->w, a->bias}) || !distinct({a->z}, {a->residual})) return SADMM_EINVAL;
    if (!in_place(a->y, a->ldy, a->residual, a->ldr, a->tokens)) return SADMM_EINVAL;
    return SADMM_OK;
}

sadmm_status check(const sadmm_linear_bwd_args* a)
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
    if (a->dx && !matrix(a->w, SADMM_BF16, a->ldw, a->n_in)) return SADMM_EINVAL;
    if (a->dw && !matrix(a->x, SADMM_BF16, a->ldx, a->n_in)) return SADMM_EINVAL;
    if (!distinct({a->dx, a->dw, a->db}, {a->dy, a->x, a->w}) || !distinct({a->dx}, {a->z})) return SADMM_EINVAL;
    if (a->act != SADMM_ACT_NONE && !distinct({a->dw, a->db}, {a->z})) return SADMM_EINVAL;
    return SADMM_OK;
}

sadmm_status check(const sadmm_gated_fwd_args* a)
{
    if (!a || !is_act(a->act)) return SADMM_EINVAL;
    const sadmm_status st = extents(a->tokens, a->n_in, a->n_hidden);
    if (st != SADMM_OK) return st;
    if (!matrix(a->wg, SADMM_BF16, a->ldwg, a->n_in) || !matrix(a->wu, SADMM_BF16, a->ldwu, a->n_in) ||
        !vec32(a->bg) || !vec32(a->bu))
        return SADMM_EINVAL;
    if (!a->tokens) return SADMM_OK;
    if (!matrix(a->x, SADMM_BF16, a->ldx, a->n_in) || !matrix(a->h, SADMM_BF16, a->ldh, a->n_hidden) ||
        !matrix_or_null(a->g, SADMM_BF16, a->ldg, a->n_hidden) || !matrix_or_null(a->u, SADMM_BF16, a->ldu, a->n_hidden))
        return SADMM_EINVAL;
    return distinct({a->h, a->g, a->u}, {a->x, a->wg, a->wu, a->bg, a->bu}) ? SADMM_OK : SADMM_EINVAL;
}

sadmm_status check(const sadmm_gated_bwd_args* a)
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
    if (a->dx && (!matrix(a->wg, SADMM_BF16, a->ldwg, a->n_in) || !matrix(a->wu, SADMM_BF16, a->ldwu, a->n_in)))
        return SADMM_EINVAL;
    if (a->dwg && !matrix(a->x, SADMM_BF16, a->ldx, a->n_in)) return SADMM_EINVAL;
    return distinct({a->dx, a->dwg, a->dwu, a->dbg, a->dbu}, {a->dh, a->x, a->wg, a->wu, a->g, a->u}) ? SADMM_OK
                                                                                                       : SADMM_EINVAL;
}

}  // namespace
}  // namespace sadmm

using namespace sadmm;

extern "C" {

sadmm_status sadmm_layernorm_fwd(const sadmm_layernorm_fwd_args* a, void* stream)
{
    NvtxRange range("sadmm_layernorm_fwd");
    const sadmm_status st = check(a);
    if (st != SADMM_OK) return st;
    return launch_layernorm_fwd(*a, static_cast<cudaStream_t>(stream));
}

size_t sadmm_layernorm_bwd_workspace_size(const sadmm_layernorm_bwd_args* a)
{
    return check(a) == SADMM_OK ? layernorm_bwd_bytes(*a) : 0;
}

sadmm_status sadmm_layernorm_bwd(const sadmm_layernorm_bwd_args* a, void* workspace, size_t ws_bytes, void* stream)
{
    NvtxRange range("sadmm_layernorm_bwd");
    const sadmm_status st = check(a);
    if (st != SADMM_OK) return st;
    if (!scratch(workspace, ws_bytes, layernorm_bwd_bytes(*a))) return SADMM_EINVAL;
    return launch_layernorm_bwd(*a, workspace, static_cast<cudaStream_t>(stream));
}

size_t sadmm_linear_fwd_workspace_size(const sadmm_linear_fwd_args* a)
{
    return check(a) == SADMM_OK ? linear_fwd_bytes(*a) : 0;
}

sadmm_status sadmm_linear_fwd(const sadmm_linear_fwd_args* a, void* workspace, size_t ws_bytes, void* stream)
{
    NvtxRange range("sadmm_linear_fwd");
    const sadmm_status st = check(a);
    if (st != SADMM_OK) return st;
    if (!scratch(workspace, ws_bytes, linear_fwd_bytes(*a))) return SADMM_EINVAL;
    if (device_cc_major() < 10) return SADMM_EUNSUPPORTED;
    return launch_linear_fwd(*a, workspace, static_cast<cudaStream_t>(stream));
}

size_t sadmm_linear_bwd_workspace_size(const sadmm_linear_bwd_args* a)
{
    return check(a) == SADMM_OK ? linear_bwd_bytes(*a) : 0;
}

sadmm_status sadmm_linear_bwd(const sadmm_linear_bwd_args* a, void* workspace, size_t ws_bytes, void* stream)
{
    NvtxRange range("sadmm_linear_bwd");
    const sadmm_status st = check(a);
    if (st != SADMM_OK) return st;
    if (!scratch(workspace, ws_bytes, linear_bwd_bytes(*a))) return SADMM_EINVAL;
    if (device_cc_major() < 10) return SADMM_EUNSUPPORTED;
    return launch_linear_bwd(*a, workspace, static_cast<cudaStream_t>(stream));
}

size_t sadmm_gated_fwd_workspace_size(const sadmm_gated_fwd_args* a)
{
    return check(a) == SADMM_OK ? gated_fwd_bytes(*a) : 0;
}

sadmm_status sadmm_gated_fwd(const sadmm_gated_fwd_args* a, void* workspace, size_t ws_bytes, void* stream)
{
    NvtxRange range("sadmm_gated_fwd");
    const sadmm_status st = check(a);
    if (st != SADMM_OK) return st;
    if (!scratch(workspace, ws_bytes, gated_fwd_bytes(*a))) return SADMM_EINVAL;
    if (device_cc_major() < 10) return SADMM_EUNSUPPORTED;
    return launch_gated_fwd(*a, workspace, static_cast<cudaStream_t>(stream));
}

size_t sadmm_gated_bwd_workspace_size(const sadmm_gated_bwd_args* a)
{
    return check(a) == SADMM_OK ? gated_bwd_bytes(*a) : 0;
}

sadmm_status sadmm_gated_bwd(const sadmm_gated_bwd_args* a, void* workspace, size_t ws_bytes, void* stream)
{
    NvtxRange range("sadmm_gated_bwd");
    const sadmm_status st = check(a);
    if (st != SADMM_OK) return st;
    if (!scratch(workspace, ws_bytes, gated_bwd_bytes(*a))) return SADMM_EINVAL;
    if (device_cc_major() < 10) return SADMM_EUNSUPPORTED;
    return launch_gated_bwd(*a, workspace, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
