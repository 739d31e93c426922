// The activations of a gated block and their derivatives, in fp32.
#pragma once

#include "atb_device.h"

namespace atb {

ATB_DEV float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.0f + __expf(-x)); }      // exp may be infinite: 1 / inf = 0

constexpr float kGeluC = 0.7978845608028654f;      // sqrt(2 / pi)
constexpr float kGeluA = 0.044715f;

// The standard normal's distribution function at x, and e = exp(-x^2 / 2): Abramowitz and Stegun 7.1.26, erfc(v) = (a1 t + .. + a5 t^5) exp(-v^2) with
// t = 1 / (1 + p v) to 1.5e-7 absolutely, for v = |x| / sqrt 2.  (x times it is 2.2e-7 off at most; of its own size far out on the left, where it is nearly 0, 1.6e-3 at -5 and
// 1e-2 at -8.)  Without a branch, which the library's erff has in every element of a tile (60 KiB of
// code, and accumulators spilled round it).
ATB_DEV float normal_cdf(float x, float &e)
{
    const float v = fabsf(x) * 0.7071067811865476f;
    const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, v, 1.0f));
    e = __expf(-0.5f * x * x);
    const float poly = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f);
    const float tail = 0.5f * poly * e;                   // at -|x|
    return x < 0.0f ? tail : 1.0f - tail;
}

// act(g), of ATB_ACT_NONE g itself.  The activation is a constant of the code around it: a wave-uniform branch per element costs more than the function.
template <int act>
ATB_DEV float activate(float g)
{
    if (act == ATB_ACT_NONE) return g;
    if (act == ATB_ACT_SILU) return g * sigmoid(g);
    if (act == ATB_ACT_GELU) {
        float e;
        return g * normal_cdf(g, e);
    }
    return g * sigmoid(2.0f * kGeluC * (g + kGeluA * g * g * g));       // (1 + tanh v) / 2 = sigmoid(2 v)
}

// act(g) and act'(g)
template <int act>
ATB_DEV void activate_grad(float g, float &a, float &slope)
{
    if (act == ATB_ACT_SILU) {
        const float s = sigmoid(g);
        a = g * s;
        slope = s * (1.0f + g * (1.0f - s));
    } else if (act == ATB_ACT_GELU) {
        float e;
        const float s = normal_cdf(g, e);
        a = g * s;
        slope = s + g * e * 0.3989422804014327f;
    } else {
        const float s = sigmoid(2.0f * kGeluC * (g + kGeluA * g * g * g));
        const float c = fminf(fmaxf(g, -64.0f), 64.0f);                 // s (1 - s) is 0 long before; keeps 0 x inf out
        a = g * s;
        slope = s + c * s * (1.0f - s) * (2.0f * kGeluC) * (1.0f + 3.0f * kGeluA * c * c);
    }
}

// f, called with the activation as a constant
template <int act> struct Activation { static constexpr int value = act; };
template <class F>
ATB_DEV void with_activation(int act, F f)
{
    if (act == ATB_ACT_SILU) f(Activation<ATB_ACT_SILU>());
    else if (act == ATB_ACT_GELU) f(Activation<ATB_ACT_GELU>());
    else f(Activation<ATB_ACT_GELU_TANH>());
}
// ... where there may be none
template <class F>
ATB_DEV void with_activation_or_none(int act, F f)
{
    if (act == ATB_ACT_NONE) f(Activation<ATB_ACT_NONE>());
    else with_activation(act, f);
}

}  // namespace atb
