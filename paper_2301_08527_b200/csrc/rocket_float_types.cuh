// The element types of the training operators (ROCKET_F32, ROCKET_F16, ROCKET_BF16): loads to and stores from fp32.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cstdint>

#include "rocket.h"

namespace rocket {

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }

// One rounding, to nearest with ties to even.
template <class T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

inline bool is_float_type(int type) { return type == ROCKET_F32 || type == ROCKET_F16 || type == ROCKET_BF16; }
inline int float_type_bytes(int type) { return type == ROCKET_F32 ? 4 : 2; }

// Calls f with a null pointer of the C++ type that `type` names.
template <class F>
auto with_float_type(int type, F&& f) {
    return type == ROCKET_F32 ? f((float*)nullptr) : type == ROCKET_F16 ? f((__half*)nullptr) : f((__nv_bfloat16*)nullptr);
}

}  // namespace rocket
