// The element types of the training operators (ROCKET_F32, ROCKET_F16, ROCKET_BF16): loads to and stores from fp32.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cstdint>
#include <type_traits>

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

// W values of T that lie next to one another, as they are in memory: loaded and stored in words of up to 16 bytes, which the
// address has to be a multiple of (W = 1: any element's).
template <class T, int W>
struct alignas(sizeof(T) * W < 16 ? sizeof(T) * W : 16) Packed {
    T v[W];
};

template <class T, int W>
__device__ __forceinline__ Packed<T, W> load_packed(const T* p) { return *reinterpret_cast<const Packed<T, W>*>(p); }

// The same for data that no thread writes while the kernel runs.
template <class T, int W>
__device__ __forceinline__ Packed<T, W> load_packed_ro(const T* p) {
    constexpr int bytes = (int)sizeof(T) * W;
    Packed<T, W> r;
    if constexpr (bytes % 16 == 0) {
#pragma unroll
        for (int i = 0; i < bytes / 16; ++i) reinterpret_cast<uint4*>(&r)[i] = __ldg(reinterpret_cast<const uint4*>(p) + i);
    } else if constexpr (bytes == 8) {
        *reinterpret_cast<uint2*>(&r) = __ldg(reinterpret_cast<const uint2*>(p));
    } else if constexpr (bytes == 4) {
        *reinterpret_cast<uint32_t*>(&r) = __ldg(reinterpret_cast<const unsigned*>(p));
    } else {
        static_assert(bytes == 2, "");
        *reinterpret_cast<uint16_t*>(&r) = __ldg(reinterpret_cast<const unsigned short*>(p));
    }
    return r;
}

template <class T, int W>
__device__ __forceinline__ void store_packed(T* p, const float (&v)[W]) {
    Packed<T, W> r;
#pragma unroll
    for (int i = 0; i < W; ++i) r.v[i] = from_float<T>(v[i]);
    *reinterpret_cast<Packed<T, W>*>(p) = r;
}

// Values `i` to `i` + W - 1 of an array whose type is known at run time only (the branch is the same for all threads).
template <int W>
__device__ __forceinline__ void load_typed(const void* p, int type, int64_t i, float (&v)[W]) {
    auto get = [&](auto* t) {
        using T = std::remove_const_t<std::remove_pointer_t<decltype(t)>>;
        const Packed<T, W> r = load_packed_ro<T, W>(t + i);
#pragma unroll
        for (int k = 0; k < W; ++k) v[k] = to_float(r.v[k]);
    };
    if (type == ROCKET_F32) get(static_cast<const float*>(p));
    else if (type == ROCKET_F16) get(static_cast<const __half*>(p));
    else get(static_cast<const __nv_bfloat16*>(p));
}

template <int W>
__device__ __forceinline__ void store_typed(void* p, int type, int64_t i, const float (&v)[W]) {
    if (type == ROCKET_F32) store_packed<float, W>(static_cast<float*>(p) + i, v);
    else if (type == ROCKET_F16) store_packed<__half, W>(static_cast<__half*>(p) + i, v);
    else store_packed<__nv_bfloat16, W>(static_cast<__nv_bfloat16*>(p) + i, v);
}

// Whether words of W values of `type` can be taken at base + k * stride (in values) for every k.
inline bool packs(const void* base, int type, int64_t stride, int W) {
    const uintptr_t word = (uintptr_t)(float_type_bytes(type) * W), unit = word < 16 ? word : 16;
    return reinterpret_cast<uintptr_t>(base) % unit == 0 && (uintptr_t)stride * float_type_bytes(type) % unit == 0;
}

}  // namespace rocket
