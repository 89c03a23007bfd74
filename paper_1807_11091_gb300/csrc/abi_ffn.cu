// abi_ffn.cu -- the extern "C" entry points of the feed-forward operators
// (layer norm, linear, gated pair): host-side validation, then the launches.
// Nothing is enqueued before every argument has been checked.
#include <math.h>

#include "internal.h"

namespace sadmm {
namespace {

bool is_dtype(int dt) { return dt == SADMM_BF16 || dt == SADMM_FP32; }
bool is_act(int act) { return act >= SADMM_ACT_NONE && act <= SADMM_ACT_SILU; }

// A pointer on its element's boundary.
bool at_element(const void* p, int dt) { return (reinterpret_cast<uintptr_t>(p) & (dt == SADMM_FP32 ? 3 : 1)) == 0; }

// A matrix: present, on its element's boundary, rows at least as far apart as
// they are long and no further than a tensor map can say (2^40 bytes).
bool matrix(const void* p, int dt, long long ld, long long cols)
{
    return p && is_dtype(dt) && at_element(p, dt) && ld >= cols && ld < (1ll << 38);
}
bool matrix_or_null(const void* p, int dt, long long ld, long long cols) { return !p || matrix(p, dt, ld, cols); }
bool vec32(const void* p) { return at_element(p, SADMM_FP32); }

constexpr long long kMaxRows = 0x7fffff00ll;   // row tiles and coordinates are 32-bit
constexpr int kMaxWidth = 1 << 28;

sadmm_status extents(long long rows, long long a, long long b)
{
    if (rows < 0 || a < 1 || b < 1) return SADMM_EINVAL;
    return rows > kMaxRows || a > kMaxWidth || b > kMaxWidth ? SADMM_EUNSUPPORTED : SADMM_OK;
}

sadmm_status check(const sadmm_layernorm_fwd_args* a)
{
    if (!a || !is_dtype(a->xdt) || !is_dtype(a->ydt) || !(a->eps >= 0.0f) || isinf(a->eps)) return SADMM_EINVAL;
    const sadmm_status st = extents(a->rows, a->cols, 1);
    if (st != SADMM_OK) return st;
    if (!vec32(a->gamma) || !vec32(a->beta) || !vec32(a->mean) || !vec32(a->rstd)) return SADMM_EINVAL;
    if (a->rows && (!matrix(a->x, a->xdt, a->ldx, a->cols) || !matrix(a->y, a->ydt, a->ldy, a->cols)))
        return SADMM_EINVAL;
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
    if (a->dx && (a->dx == a->x || a->dx == a->dy)) return SADMM_EINVAL;
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
    if (a->y == a->x || a->y == a->w || a->y == a->z || (a->z && (a->z == a->x || a->z == a->w))) return SADMM_EINVAL;
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
    if (a->dx && (a->dx == a->x || a->dx == a->dy || a->dx == a->w || a->dx == a->z)) return SADMM_EINVAL;
    if (a->dw && (a->dw == a->x || a->dw == a->dy || a->dw == a->w || a->dw == a->dx)) return SADMM_EINVAL;
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
    const void* const in[3] = {a->x, a->wg, a->wu};
    const void* const out[3] = {a->h, a->g, a->u};
    for (int o = 0; o < 3; ++o) {
        if (!out[o]) continue;
        for (int i = 0; i < 3; ++i)
            if (out[o] == in[i] || (i != o && out[o] == out[i])) return SADMM_EINVAL;
    }
    return SADMM_OK;
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
    const void* const in[6] = {a->dh, a->x, a->wg, a->wu, a->g, a->u};
    const void* const out[3] = {a->dx, a->dwg, a->dwu};
    for (int o = 0; o < 3; ++o) {
        if (!out[o]) continue;
        for (int i = 0; i < 6; ++i)
            if (out[o] == in[i] || (i < o && out[o] == out[i])) return SADMM_EINVAL;
    }
    return SADMM_OK;
}

// Scratch: `need` bytes on a 256-byte boundary.
bool scratch(const void* ws, size_t bytes, size_t need)
{
    return need == 0 || (ws && bytes >= need && (reinterpret_cast<uintptr_t>(ws) & 255) == 0);
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
