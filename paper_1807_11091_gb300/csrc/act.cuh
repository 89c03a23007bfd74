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

// 2^x for x <= 0, 0 below 2^-126; within 2 units.
SADMM_DEV float exp2_fast(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// z Phi(z) with the normal distribution Phi, of which 1 + erf would leave no digit in
// the tail: Phi's smaller side is exp(-z^2 / 2) t P(t), t = 1 / (1 + 0.3 |z|), with P of
// degree 7 fitted to that quotient for |z| up to 13.5 (least maximum of the relative
// error, 1.3e-7; with its rounding 4.4e-7).  The exponent c z^2, c = -log2(e) / 2, is
// taken in two parts, because the power would enlarge its rounding.  4096^3 in fp32
// takes 134 us so and with erf, 205 with CUDA's normcdff, which is as exact.
// e: exp(-z^2 / 2); returns Phi(z).
SADMM_DEV float phi_f32(float z, float& e)
{
    const float w = fminf(fabsf(z), 15.0f);  // past which the smaller side is 0
    constexpr float c = -0.721347511f, c_low = -9.62981517e-09f;
    const float s = w * w, h = s * c;
    const float low = fmaf(s, c, -h) + fmaf(s, c_low, fmaf(w, w, -s) * c);
    const float p = exp2_fast(h);
    e = fmaf(p, low * 0.693147181f, p);
    const float t = __fdividef(1.0f, 1.0f + 0.3f * w);
    float g = 0.0359317213f;
    g = fmaf(g, t, -0.158275947f);
    g = fmaf(g, t, 0.208206505f);
    g = fmaf(g, t, -0.0553937592f);
    g = fmaf(g, t, 0.129469156f);
    g = fmaf(g, t, 0.0996375084f);
    g = fmaf(g, t, 0.120798357f);
    g = fmaf(g, t, 0.119626388f);
    const float q = e * (t * g);
    return z > 0.0f ? 1.0f - q : q;
}
SADMM_DEV float gelu_f32(float z)
{
    float e;
    return z * phi_f32(z, e);
}

// act(z): max(z, 0) (NaN kept); gelu_f32; z sigmoid(z).
template <int ACT>
SADMM_DEV float act_f32(float z)
{
    if (ACT == kGeluBf16 || ACT == kSiluBf16) {
        float a, s;
        act_slope_f32<ACT == kGeluBf16 ? SADMM_ACT_GELU : SADMM_ACT_SILU>(z, a, s);
        return a;
    }
    if (ACT == SADMM_ACT_RELU) return z < 0.0f ? 0.0f : z;
    if (ACT == SADMM_ACT_GELU) return gelu_f32(z);
    if (ACT == SADMM_ACT_SILU) return __fdividef(z, 1.0f + expf(-z));
    return z;
}

// act(z) and the slope act'(z) ([z > 0]; Phi(z) + z phi(z); s + z s (1 - s) with
// s = 1 / (1 + exp(-z)), where an infinite exp gives 0) together, for results that
// are rounded to bf16, an error of 2^-9 to 2^-8 (and the column sums of those of a bf16 block).  Chosen for speed, far below that:
// exp by its fast form (2^-21 and |z| 2^-23 of the value; with z^2 / 2 for |z|
// below 2e-5), and Phi's smaller side as exp(-z^2 / 2) t P(t), t = 1 / (1 + 0.29 |z|),
// with P of degree 5 fitted to that quotient for |z| up to 13.5 (least weighted
// maximum: 0.72e-7 of 1 and 7.2e-5 of the value, where GELU and its slope are small).
template <int ACT>
SADMM_DEV void act_slope_f32(float z, float& a, float& s)
{
    if (ACT == SADMM_ACT_SILU) {
        const float p = __fdividef(1.0f, 1.0f + __expf(-z));
        a = z * p;
        s = p + a * (1.0f - p);
    } else if (ACT == SADMM_ACT_GELU) {
        const float w = fabsf(z), e = __expf(-0.5f * z * z);
        const float t = __fdividef(1.0f, 1.0f + 0.29f * w);
        const float q = e * t *
                        (0.116863564f +
                         t * (0.100840715f +
                              t * (0.179055156f + t * (-0.0923723266f + t * (0.284238196f + t * -0.0886252389f)))));
        const float p = z > 0.0f ? 1.0f - q : q;
        a = z * p;
        s = p + z * 0.39894228040143268f * e;
    } else {
        a = act_f32<ACT>(z);
        s = ACT == SADMM_ACT_RELU ? (z > 0.0f ? 1.0f : 0.0f) : 1.0f;
    }
}

// The same for what becomes fp32 sums or 8-bit values (a backward pass of 8-bit operands), at fp32's
// precision: GELU by phi_f32 (its slope is some 30 units of its terms off by the form above; 8 us of the 354 that the
// gated pair's backward of 4096 x 2048 -> 5461 takes); SiLU by the form above, which is within 12 units of its
// terms too (expf would be 6 us of 328).
template <int ACT>
SADMM_DEV void act_slope_exact(float z, float& a, float& s)
{
    if (ACT == SADMM_ACT_GELU) {
        float e;
        const float p = phi_f32(z, e);
        a = z * p;
        s = p + z * 0.39894228040143268f * e;
    } else {
        act_slope_f32<ACT>(z, a, s);
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
