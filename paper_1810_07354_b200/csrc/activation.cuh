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

// The Gaussian's distribution function and e = exp(-z^2 / 2) to a few units of float32.  The function is its power series around 0, which
// takes six terms up to 0.6, and beyond that e times a polynomial of degree eight in t = 1 / (1 + 0.275 |z|), fitted to 2^-28 of
// itself by weighted least squares up to |z| = 14, from where on e is 0 in float32.  e's exponent comes in two parts: that the square
// and its product with 1 / (2 ln 2) are rounded would cost z^2 2^-25 of e.
__device__ __forceinline__ float2 horner(float2, float2 p) { return p; }
template <typename... C> __device__ __forceinline__ float2 horner(float2 x, float2 p, float next, C... rest) { return horner(x, fma2(x, p, both(next)), rest...); }
__device__ __forceinline__ void gaussian(float2 z, float2 &cdf, float2 &e) {
    const float2 v = make_float2(fminf(fabsf(z.x), 14.f), fminf(fabsf(z.y), 14.f));
    const float2 h = mul2(v, v), half_log2e = both(-0.72134752f), x = mul2(h, half_log2e);
    float2 more = fma2(h, half_log2e, make_float2(-x.x, -x.y));
    more = fma2(h, both(-9.6298149e-9f), more);  // -1 / (2 ln 2) + 0.72134752
    more = fma2(fma2(v, v, make_float2(-h.x, -h.y)), half_log2e, more);
    e = ex2_pair(x);
    e = fma2(e, mul2(more, both(0.69314718f)), e);
    const float2 t = rcp_pair(fma2(v, both(0.275f), both(1.f)));
    const float2 p = horner(t, both(0.0312250451f), -0.127670346f, 0.160190437f, -0.0642568446f, 0.104863903f, 0.0729800932f, 0.103439847f, 0.10951235f, 0.109717387f);
    const float2 tail = mul2(mul2(p, t), e), body = fma2(tail, both(-1.f), both(1.f));
    const float2 near = fma2(z, horner(h, both(-9.44465626e-06f), 0.000115434688f, -0.00118732822f, 0.00997355701f, -0.0664903801f, 0.39894228f), both(0.5f));
    cdf.x = v.x < 0.6f ? near.x : z.x < 0.f ? tail.x : body.x;
    cdf.y = v.y < 0.6f ? near.y : z.y < 0.f ? tail.y : body.y;
}

// a = act(z), slope = act'(z), of two values on their way to results of type T.  Beside 16 bits the Gaussian's distribution function
// comes from Abramowitz and Stegun's formula 7.1.26 for erf (off by 1.5e-7 at most): it needs one reciprocal and the exponential that its
// derivative needs anyway, and takes the lower tail as a product, so nothing cancels there.  For float32 that is too little: 7e-7 of
// the result around 0, 5e-5 at -3, 4e-3 at -6, where gaussian() stays below 5e-7 (8192 x 128 -> 4096 with the derivative: 136 us, the
// formula 132; one row of 4096 -> 4096 14.9 and 14.2).
template <int ACT, typename T> __device__ __forceinline__ void activate(float2 z, float2 &a, float2 &slope) {
    if (ACT == SCAR_ACT_IDENTITY) {
        a = z;
        slope = both(1.f);
    } else if (ACT == SCAR_ACT_RELU) {
        slope = make_float2(z.x > 0.f ? 1.f : 0.f, z.y > 0.f ? 1.f : 0.f);
        a = make_float2(z.x < 0.f ? 0.f : z.x, z.y < 0.f ? 0.f : z.y);  // a NaN stays one
    } else if (ACT == SCAR_ACT_GELU && sizeof(T) == 4) {
        float2 e, cdf;
        gaussian(z, cdf, e);
        a = mul2(z, cdf);
        slope = fma2(mul2(z, both(0.39894228f)), e, cdf);
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
