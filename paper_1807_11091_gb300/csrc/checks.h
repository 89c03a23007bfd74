// checks.h -- what the feed-forward operators' entry points check of their
// arguments (abi_ffn.cu, abi_q8.cu).
#pragma once

#include <stdint.h>

#include <initializer_list>

#include "internal.h"

namespace sadmm {

inline bool is_dtype(int dt) { return dt == SADMM_BF16 || dt == SADMM_FP32; }
inline bool is_act(int act) { return act >= SADMM_ACT_NONE && act <= SADMM_ACT_SILU; }

// A pointer on its element's boundary.
inline bool at_element(const void* p, int dt) { return (reinterpret_cast<uintptr_t>(p) & (dt == SADMM_FP32 ? 3 : 1)) == 0; }

// A matrix: present, on its element's boundary, rows at least as far apart as
// they are long and no further than a tensor map can say (2^40 bytes).
inline bool matrix(const void* p, int dt, long long ld, long long cols)
{
    return p && is_dtype(dt) && at_element(p, dt) && ld >= cols && ld < (1ll << 38);
}
inline bool matrix_or_null(const void* p, int dt, long long ld, long long cols) { return !p || matrix(p, dt, ld, cols); }
inline bool vec32(const void* p) { return at_element(p, SADMM_FP32); }

// Whether every output given is at an address of its own, apart from the other
// outputs and the inputs.
inline bool distinct(std::initializer_list<const void*> outputs, std::initializer_list<const void*> inputs)
{
    for (const void* const* o = outputs.begin(); o != outputs.end(); ++o) {
        if (!*o) continue;
        for (const void* const* p = outputs.begin(); p != o; ++p)
            if (*p == *o) return false;
        for (const void* i : inputs)
            if (i == *o) return false;
    }
    return true;
}

// An output that may take an input's place: elsewhere, or on the same rows.
inline bool in_place(const void* out, long long ldo, const void* in, long long ldi, long long rows)
{
    return out != in || ldo == ldi || rows == 1;
}

constexpr long long kMaxRows = 0x7fffff00ll;   // row tiles and coordinates are 32-bit
constexpr int kMaxWidth = 1 << 28;

inline sadmm_status extents(long long rows, long long a, long long b)
{
    if (rows < 0 || a < 1 || b < 1) return SADMM_EINVAL;
    return rows > kMaxRows || a > kMaxWidth || b > kMaxWidth ? SADMM_EUNSUPPORTED : SADMM_OK;
}

// Scratch: `need` bytes on a 256-byte boundary.
inline bool scratch(const void* ws, size_t bytes, size_t need)
{
    return need == 0 || (ws && bytes >= need && (reinterpret_cast<uintptr_t>(ws) & 255) == 0);
}

}  // namespace sadmm
