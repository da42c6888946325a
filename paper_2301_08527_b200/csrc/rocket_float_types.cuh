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

// W values of T that lie next to one another, as the words of up to 16 bytes they are loaded and stored in (addresses are multiples
// of a word's size).
template <class T, int W>
struct Packed {
    static constexpr int kBytes = (int)sizeof(T) * W, kWord = kBytes < 16 ? kBytes : 16, kWords = kBytes / kWord;
    using Word = std::conditional_t<kWord == 16, uint4, std::conditional_t<kWord == 8, uint2, std::conditional_t<kWord == 4, unsigned, unsigned short>>>;
    Word w[kWords];
    __device__ __forceinline__ T get(int i) const { return reinterpret_cast<const T*>(w)[i]; }
    __device__ __forceinline__ uint32_t pair(int i) const { return reinterpret_cast<const uint32_t*>(w)[i]; }
};

template <class T, int W>
__device__ __forceinline__ Packed<T, W> load_packed(const T* p) {
    using P = Packed<T, W>;
    P r;
#pragma unroll
    for (int i = 0; i < P::kWords; ++i) r.w[i] = reinterpret_cast<const typename P::Word*>(p)[i];
    return r;
}

// The same for data that no thread writes while the kernel runs.
template <class T, int W>
__device__ __forceinline__ Packed<T, W> load_packed_ro(const T* p) {
    using P = Packed<T, W>;
    P r;
#pragma unroll
    for (int i = 0; i < P::kWords; ++i) r.w[i] = __ldg(reinterpret_cast<const typename P::Word*>(p) + i);
    return r;
}

// The values as fp32, 16-bit ones in pairs from the words that hold them.
template <class T, int W>
__device__ __forceinline__ void unpack(const Packed<T, W>& r, float (&v)[W]) {
    if constexpr (sizeof(T) == 2 && W % 2 == 0) {
#pragma unroll
        for (int i = 0; i < W / 2; ++i) {
            const uint32_t w = r.pair(i);
            if constexpr (std::is_same_v<T, __half>) {
                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
                v[2 * i] = f.x;
                v[2 * i + 1] = f.y;
            } else {                       // a bfloat16 is the upper half of the fp32 value
                v[2 * i] = __uint_as_float(w << 16);
                v[2 * i + 1] = __uint_as_float(w & 0xffff0000u);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] = to_float(r.get(i));
    }
}

// The same for data that is read once: it takes no place in L1, which is left to what is read again.
template <class T, int W>
__device__ __forceinline__ Packed<T, W> load_packed_once(const T* p) {
    using P = Packed<T, W>;
    P r;
    if constexpr (P::kWord == 16) {
#pragma unroll
        for (int i = 0; i < P::kWords; ++i)
            asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                         : "=r"(r.w[i].x), "=r"(r.w[i].y), "=r"(r.w[i].z), "=r"(r.w[i].w) : "l"(reinterpret_cast<const uint4*>(p) + i));
    } else if constexpr (P::kWord == 8) {
        asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(r.w[0].x), "=r"(r.w[0].y) : "l"(p));
    } else {
        r = load_packed_ro<T, W>(p);
    }
    return r;
}

template <class T, int W>
__device__ __forceinline__ void store_packed(T* p, const float (&v)[W]) {
    using P = Packed<T, W>;
    P r;
    if constexpr (sizeof(T) == 2 && W % 2 == 0) {
#pragma unroll
        for (int i = 0; i < W / 2; ++i) {
            uint32_t& w = reinterpret_cast<uint32_t*>(r.w)[i];
            if constexpr (std::is_same_v<T, __half>) {
                const __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
                w = *reinterpret_cast<const uint32_t*>(&h);
            } else {
                const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
                w = *reinterpret_cast<const uint32_t*>(&h);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const T t = from_float<T>(v[i]);
            if constexpr (sizeof(T) == 4) reinterpret_cast<uint32_t*>(r.w)[i] = __float_as_uint(t);
            else reinterpret_cast<unsigned short*>(r.w)[i] = *reinterpret_cast<const unsigned short*>(&t);
        }
    }
#pragma unroll
    for (int i = 0; i < P::kWords; ++i) reinterpret_cast<typename P::Word*>(p)[i] = r.w[i];
}

// Values `i` to `i` + W - 1 of an array whose type is known at run time only (the branch is the same for all threads).
template <int W>
__device__ __forceinline__ void load_typed(const void* p, int type, int64_t i, float (&v)[W]) {
    auto get = [&](auto* t) {
        using T = std::remove_const_t<std::remove_pointer_t<decltype(t)>>;
        unpack<T, W>(load_packed_ro<T, W>(t + i), v);
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
