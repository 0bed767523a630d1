// float32 arithmetic on pairs: one instruction for two values (sm_100's f32x2), each result rounded as the single instruction's.
#pragma once
#include "train_common.cuh"

namespace scar {

__device__ __forceinline__ unsigned long long pair_bits(float2 a) {
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a.x), "f"(a.y));
    return r;
}
__device__ __forceinline__ float2 bits_pair(unsigned long long a) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(a));
    return r;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(pair_bits(a)), "l"(pair_bits(b)), "l"(pair_bits(c)));
    return bits_pair(r);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    unsigned long long r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(pair_bits(a)), "l"(pair_bits(b)));
    return bits_pair(r);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(pair_bits(a)), "l"(pair_bits(b)));
    return bits_pair(r);
}
__device__ __forceinline__ float2 both(float a) { return make_float2(a, a); }

// Two neighbours of a packed row.
template <typename T> struct Two;
template <> struct Two<float> {
    static __device__ __forceinline__ float2 get(const float *v) { return make_float2(v[0], v[1]); }
    static __device__ __forceinline__ void put(float *v, float2 x) { v[0] = x.x; v[1] = x.y; }
};
template <> struct Two<__nv_bfloat16> {
    static __device__ __forceinline__ float2 get(const __nv_bfloat16 *v) {
        const unsigned u = *reinterpret_cast<const unsigned *>(v);
        return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
    }
    static __device__ __forceinline__ void put(__nv_bfloat16 *v, float2 x) { *reinterpret_cast<__nv_bfloat162 *>(v) = __float22bfloat162_rn(x); }
};
template <> struct Two<__half> {
    static __device__ __forceinline__ float2 get(const __half *v) { return __half22float2(*reinterpret_cast<const __half2 *>(v)); }
    static __device__ __forceinline__ void put(__half *v, float2 x) { *reinterpret_cast<__half2 *>(v) = __float22half2_rn(x); }
};

}  // namespace scar
