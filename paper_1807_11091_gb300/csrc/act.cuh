// act.cuh -- the activations of the feed-forward operators and their slopes, in
// fp32.
#pragma once

#include "common.cuh"

namespace sadmm {

// 1 / (1 + exp(-z)); exp overflows to infinity for z below -88, which gives 0.
SADMM_DEV float sigmoid_f32(float z) { return __fdividef(1.0f, 1.0f + expf(-z)); }

// act(z): max(z, 0) (NaN kept); z Phi(z) with the normal distribution Phi; z sigmoid(z).
template <int ACT>
SADMM_DEV float act_f32(float z)
{
    if (ACT == SADMM_ACT_RELU) return z < 0.0f ? 0.0f : z;
    if (ACT == SADMM_ACT_GELU) return 0.5f * z * (1.0f + erff(z * 0.70710678118654752f));
    if (ACT == SADMM_ACT_SILU) return __fdividef(z, 1.0f + expf(-z));
    return z;
}

// act'(z): [z > 0]; Phi(z) + z phi(z); s + z s (1 - s) with s = sigmoid(z).
template <int ACT>
SADMM_DEV float dact_f32(float z)
{
    if (ACT == SADMM_ACT_RELU) return z > 0.0f ? 1.0f : 0.0f;
    if (ACT == SADMM_ACT_GELU)
        return 0.5f * (1.0f + erff(z * 0.70710678118654752f)) + z * 0.39894228040143268f * expf(-0.5f * z * z);
    if (ACT == SADMM_ACT_SILU) {
        const float s = sigmoid_f32(z);
        return s * (1.0f + z * (1.0f - s));
    }
    return 1.0f;
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
    default: f(ActTag<SADMM_ACT_NONE>()); break;
    }
}

}  // namespace sadmm
