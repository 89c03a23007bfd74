// act.cuh -- the activations of the feed-forward operators and their slopes, in
// fp32.
#pragma once

#include "common.cuh"

namespace sadmm {

// Codes beside sadmm_act: the same functions for results that are rounded to
// bf16, by act_slope_f32's faster forms.
constexpr int kGeluBf16 = 4, kSiluBf16 = 5;
inline int act_for(int act, bool bf16)
{
    return !bf16 ? act : act == SADMM_ACT_GELU ? kGeluBf16 : act == SADMM_ACT_SILU ? kSiluBf16 : act;
}

template <int ACT>
SADMM_DEV void act_slope_f32(float z, float& a, float& s);

// act(z): max(z, 0) (NaN kept); z Phi(z) with the normal distribution Phi; z sigmoid(z).
template <int ACT>
SADMM_DEV float act_f32(float z)
{
    if (ACT == kGeluBf16 || ACT == kSiluBf16) {
        float a, s;
        act_slope_f32<ACT == kGeluBf16 ? SADMM_ACT_GELU : SADMM_ACT_SILU>(z, a, s);
        return a;
    }
    if (ACT == SADMM_ACT_RELU) return z < 0.0f ? 0.0f : z;
    if (ACT == SADMM_ACT_GELU) return 0.5f * z * (1.0f + erff(z * 0.70710678118654752f));
    if (ACT == SADMM_ACT_SILU) return __fdividef(z, 1.0f + expf(-z));
    return z;
}

// act(z) and the slope act'(z) ([z > 0]; Phi(z) + z phi(z); s + z s (1 - s) with
// s = 1 / (1 + exp(-z)), where an infinite exp gives 0) together, for the backward pass, where both are operands
// rounded to bf16: exp by its fast form, whose error (2^-21 and |z| 2^-23, below
// 2e-6 for |z| up to 16) is far below that.
template <int ACT>
SADMM_DEV void act_slope_f32(float z, float& a, float& s)
{
    if (ACT == SADMM_ACT_SILU) {
        const float p = __fdividef(1.0f, 1.0f + __expf(-z));
        a = z * p;
        s = p + a * (1.0f - p);
    } else if (ACT == SADMM_ACT_GELU) {
        // Phi(-|z|) = erfc(|z| / sqrt 2) / 2 by Abramowitz and Stegun's 7.1.26 (within 0.75e-7), which needs the
        // exp(-z^2 / 2) that phi(z) needs too
        const float x = fabsf(z) * 0.70710678f, e = __expf(-0.5f * z * z);
        const float t = __fdividef(1.0f, 1.0f + 0.3275911f * x);
        const float q =
            0.5f * e * t *
            (0.254829592f + t * (-0.284496736f + t * (1.421413741f + t * (-1.453152027f + t * 1.061405429f))));
        const float p = z > 0.0f ? 1.0f - q : q;
        a = z * p;
        s = p + z * 0.39894228040143268f * e;
    } else {
        a = act_f32<ACT>(z);
        s = ACT == SADMM_ACT_RELU ? (z > 0.0f ? 1.0f : 0.0f) : 1.0f;
    }
}

// Calls f(std::integral_constant-like tag) for a run-time activation.
template <int A>
struct ActTag {
    static constexpr int value = A;
};
template <typename F>
SADMM_DEV void with_act(int act, F f)
{
    switch (act) {
    case SADMM_ACT_RELU: f(ActTag<SADMM_ACT_RELU>()); break;
    case SADMM_ACT_GELU: f(ActTag<SADMM_ACT_GELU>()); break;
    case SADMM_ACT_SILU: f(ActTag<SADMM_ACT_SILU>()); break;
    case kGeluBf16: f(ActTag<kGeluBf16>()); break;
    case kSiluBf16: f(ActTag<kSiluBf16>()); break;
    default: f(ActTag<SADMM_ACT_NONE>()); break;
    }
}

}  // namespace sadmm
