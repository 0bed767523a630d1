// Activations of a hidden layer and their derivatives.
#pragma once
#include <type_traits>

#include "pairs.cuh"

namespace scar {

__device__ __forceinline__ float2 ex2_pair(float2 x) {
    float2 y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y.x) : "f"(x.x));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y.y) : "f"(x.y));
    return y;
}
__device__ __forceinline__ float2 rcp_pair(float2 x) {
    float2 y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y.x) : "f"(x.x));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y.y) : "f"(x.y));
    return y;
}

// a = act(z), slope = act'(z), of two values.  The Gaussian's distribution function comes from Abramowitz and Stegun's formula 7.1.26
// for erf (off by 1.5e-7 at most): it needs one reciprocal and the exponential that its derivative needs anyway, and takes the
// lower tail as a product, so nothing cancels there.
template <int ACT> __device__ __forceinline__ void activate(float2 z, float2 &a, float2 &slope) {
    if (ACT == SCAR_ACT_IDENTITY) {
        a = z;
        slope = both(1.f);
    } else if (ACT == SCAR_ACT_RELU) {
        slope = make_float2(z.x > 0.f ? 1.f : 0.f, z.y > 0.f ? 1.f : 0.f);
        a = make_float2(z.x < 0.f ? 0.f : z.x, z.y < 0.f ? 0.f : z.y);  // a NaN stays one
    } else if (ACT == SCAR_ACT_GELU) {
        const float2 e = ex2_pair(mul2(mul2(z, z), both(-0.72134752f)));  // exp(-z^2 / 2)
        const float2 t = rcp_pair(fma2(make_float2(fabsf(z.x), fabsf(z.y)), both(0.23164189f), both(1.f)));  // 1 / (1 + 0.3275911 |z| / sqrt 2)
        // half of the formula's coefficients: the distribution beyond |z|
        float2 p = fma2(t, both(0.5307027145f), both(-0.7265760135f));
        p = fma2(t, p, both(0.7107068705f));
        p = fma2(t, p, both(-0.142248368f));
        p = fma2(t, p, both(0.127414796f));
        const float2 tail = mul2(mul2(p, t), e);
        const float2 body = fma2(tail, both(-1.f), both(1.f));
        const float2 cdf = make_float2(z.x < 0.f ? tail.x : body.x, z.y < 0.f ? tail.y : body.y);
        a = mul2(z, cdf);
        slope = fma2(mul2(z, both(0.39894228f)), e, cdf);
    } else {
        const float2 s = rcp_pair(add2(ex2_pair(mul2(z, both(-1.4426950409f))), both(1.f)));
        a = mul2(z, s);
        slope = mul2(s, fma2(z, fma2(s, both(-1.f), both(1.f)), both(1.f)));
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
