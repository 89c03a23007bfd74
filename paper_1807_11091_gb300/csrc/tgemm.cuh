// tgemm.cuh -- host interface of the tensor-core products behind the
// feed-forward operators (tgemm.cu): C = A B^T, with either operand contiguous
// along the contraction or along its rows, and an epilogue that finishes an
// operator's output in registers.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "sadmm.h"

namespace sadmm {

// One bf16 operand: `rows` rows of the output's row (or column) index, each
// `k` long.  kmajor: element (r, k) at p[r * ld + k]; otherwise p[k * ld + r].
// p is 16-byte aligned and ld a multiple of 8.
struct TgOperand {
    const void* p;
    long long rows, k, ld;
    bool kmajor;
};

// An output (or residual) matrix, row-major; dt is SADMM_BF16 or SADMM_FP32.
struct TgMatrix {
    void* p;
    long long ld;
    int dt;
};

enum TgMode {
    kTgSingle = 0,   // C = A0 B0^T
    kTgSum = 1,      // C = A0 B0^T + A1 B1^T (one contraction of twice the length)
    kTgPair = 2,     // y = A0 B0^T, y2 = A1 B0^T (two products in one launch)
    kTgGated = 3,    // g = A0 B0^T + bias, u = A0 B1^T + bias2, y = act(g) * u
};

struct TgProblem {
    int mode;
    TgOperand a[2], b[2];
    long long m, n;        // output rows and columns
    const float* bias;     // [n] or NULL
    const float* bias2;    // kTgGated: u's bias
    int act;               // sadmm_act
    TgMatrix y;
    TgMatrix y2;           // kTgPair: the second product's output
    TgMatrix residual;     // p NULL: none; type of y
    TgMatrix z;            // bf16 pre-activation (kTgGated: g), p NULL: not kept
    TgMatrix u;            // kTgGated: u, p NULL: not kept
};

// Whether an operand can be read by the tensor-memory accelerator where it lies.
inline bool tg_aligned(const void* p, long long ld)
{
    return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && (ld & 7) == 0;
}

// Runs a checked problem (m, n >= 1; k >= 1).
sadmm_status launch_tgemm(const TgProblem& t, cudaStream_t s);

}  // namespace sadmm
