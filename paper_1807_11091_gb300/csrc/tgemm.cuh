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
    kTgSingle = 0,   // y = A0 B0^T, finished by the epilogue
    kTgSum = 1,      // y = A0 B0^T + A1 B1^T (one contraction of twice the length)
    kTgGated = 2,    // g = A0 B0^T + bias, u = A0 B1^T + bias2, y = act(g) * u
};

struct TgProblem {
    int mode;
    bool skip;             // not wanted: weighed in the choice of tiles and cuts (so that the others' bits do not
                           // depend on it), then left out; its pointers are not looked at
    TgOperand a[2], b[2];
    long long m, n;        // output rows and columns
    const float* bias;     // [n] or NULL
    const float* bias2;    // kTgGated: u's bias
    int act;               // sadmm_act
    TgMatrix y;
    TgMatrix residual;     // p NULL: none; type of y
    TgMatrix z;            // bf16 pre-activation (kTgGated: g), p NULL: not kept
    TgMatrix u;            // kTgGated: u, p NULL: not kept
};

// Whether an operand can be read by the tensor-memory accelerator where it lies.
inline bool tg_aligned(const void* p, long long ld)
{
    return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && (ld & 7) == 0;
}

// Runs one to three checked problems (m, n, k >= 1).  Several are products
// without epilogue (kTgSingle or kTgSum; bias, residual, z and u not given, no
// activation); they share launches where they can.
sadmm_status launch_tgemm(const TgProblem* t, int count, cudaStream_t s);

// The same by CTA pairs (tgemm_pair.cu) with tiles of 256 x bn, bn a multiple
// of 64 (of 32 where choose_tgemm_pair says so) up to 256; choose_tgemm_pair gives the width it takes and an estimate
// of the time in 10 ns.
struct TgPairChoice {
    int bn;
    long long time;
};
TgPairChoice choose_tgemm_pair(const TgProblem* t, int count);
sadmm_status launch_tgemm_pair(const TgProblem* t, int count, int bn, cudaStream_t s);

}  // namespace sadmm
