// Activations of a hidden layer and their derivatives.
#pragma once
#include <type_traits>

#include "train_common.cuh"

namespace scar {

// a = act(z), slope = act'(z).  The Gaussian's distribution function comes from Abramowitz and Stegun's formula 7.1.26 for erf
// (off by 1.5e-7 at most): it needs one reciprocal and the exponential that its derivative needs anyway, and takes the lower
// tail as a product, so nothing cancels there.
template <int ACT> __device__ __forceinline__ void activate(float z, float &a, float &slope) {
    if (ACT == SCAR_ACT_IDENTITY) {
        a = z;
        slope = 1.f;
    } else if (ACT == SCAR_ACT_RELU) {
        slope = z > 0.f ? 1.f : 0.f;
        a = z < 0.f ? 0.f : z;  // a NaN stays one
    } else if (ACT == SCAR_ACT_GELU) {
        const float e = exp2f(z * z * -0.72134752f);  // exp(-z^2 / 2)
        const float t = __frcp_rn(fmaf(0.23164189f, fabsf(z), 1.f));  // 1 / (1 + 0.3275911 |z| / sqrt 2)
        float p = fmaf(t, 1.061405429f, -1.453152027f);
        p = fmaf(t, p, 1.421413741f);
        p = fmaf(t, p, -0.284496736f);
        p = fmaf(t, p, 0.254829592f);
        const float tail = 0.5f * p * t * e;  // of the distribution beyond |z|
        const float cdf = z < 0.f ? tail : 1.f - tail;
        a = z * cdf;
        slope = fmaf(z * 0.39894228f, e, cdf);
    } else {
        const float s = __fdividef(1.f, 1.f + __expf(-z));
        a = z * s;
        slope = s * fmaf(z, 1.f - s, 1.f);
    }
}

// f(std::integral_constant<int, ACT>) for an activation.
template <typename F> inline void dispatch_activation(int act, F &&f) {
    if (act == SCAR_ACT_IDENTITY) f(std::integral_constant<int, SCAR_ACT_IDENTITY>());
    else if (act == SCAR_ACT_RELU) f(std::integral_constant<int, SCAR_ACT_RELU>());
    else if (act == SCAR_ACT_GELU) f(std::integral_constant<int, SCAR_ACT_GELU>());
    else f(std::integral_constant<int, SCAR_ACT_SILU>());
}

}  // namespace scar
