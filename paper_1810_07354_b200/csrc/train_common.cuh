// What the operators of the training step (xent.cu, gnorm.cu) share: element types, conversions, allocation.
#pragma once
#include <cstddef>
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "scar.h"

namespace scar {

#define TRAIN_TRY(expr)                              \
    do {                                             \
        cudaError_t e_ = (expr);                     \
        if (e_ != cudaSuccess) {                     \
            cudaGetLastError();                      \
            return SCAR_ERR_CUDA;                    \
        }                                            \
    } while (0)

inline bool is_operand_type(int dt) { return dt == SCAR_F32 || dt == SCAR_BF16 || dt == SCAR_F16; }
inline unsigned elem_size(int dt) { return dt == SCAR_F32 ? 4u : 2u; }
inline uint64_t round_up(uint64_t v, uint64_t m) { return (v + m - 1) / m * m; }

template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_f32<__half>(__half v) { return __half2float(v); }

template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

// Calls f with a value of the element type dt stands for.
template <typename F> inline void dispatch_operand(int dt, F &&f) {
    if (dt == SCAR_F32) f(float{});
    else if (dt == SCAR_BF16) f(__nv_bfloat16{});
    else f(__half{});
}

inline int check_current_device(int device) {
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess) return SCAR_ERR_CUDA;
    return dev == device ? SCAR_OK : SCAR_ERR_STATE;
}

}  // namespace scar
