// The 2-norm of a gradient held in many tensors, and clipping by it: the step between the backward passes and the optimiser.
//
//   n = sqrt(sum over tensors and values of g^2)    c = min(1, max_norm / (n + 1e-6))    out = c g
//
// Squares and sums are kept in double precision: fp32 gradients of 1e-20 and 1e20 both have squares outside fp32.  The sums'
// order depends on the sizes alone.
//
// Bound: memory.
#include <algorithm>
#include <cmath>
#include <new>
#include <utility>
#include <vector>

#include "rocket_float_types.cuh"
#include "rocket_internal.h"

namespace rocket {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kBlocks = 148 * 8;         // most blocks, and partial sums, of one launch
constexpr int kTensors = 112;            // of one launch: the table travels in its arguments
constexpr int64_t kChunk = 16384;        // values of one tensor that a block takes at a time

struct Table {
    const void* g[kTensors];
    void* out[kTensors];
    int64_t size[kTensors];
    int first[kTensors + 1];             // chunk with which the tensor begins
    uint8_t g_type[kTensors], out_type[kTensors];
    int tensors;
};

__device__ __forceinline__ double block_sum(double a) {
    __shared__ double red[kWarps];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) a += __shfl_xor_sync(0xffffffffu, a, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = a;
    __syncthreads();
    a = 0.0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) a += red[w];
    return a;
}

// The tensor that a chunk belongs to.
__device__ __forceinline__ int tensor_of(const Table& t, int chunk) {
    int lo = 0, hi = t.tensors;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        (t.first[mid] <= chunk ? lo : hi) = mid;
    }
    return lo;
}

template <class T>
__device__ __forceinline__ double sum_squares(const void* g, int64_t beg, int64_t end) {
    double s = 0.0;
    for (int64_t i = beg + threadIdx.x; i < end; i += kThreads) {
        const double v = (double)to_float(static_cast<const T*>(g)[i]);
        s += v * v;
    }
    return s;
}

__global__ void __launch_bounds__(kThreads) squares_kernel(const __grid_constant__ Table t, double* __restrict__ part) {
    double s = 0.0;
    for (int c = blockIdx.x; c < t.first[t.tensors]; c += gridDim.x) {
        const int k = tensor_of(t, c);
        const int64_t beg = (int64_t)(c - t.first[k]) * kChunk, end = min(t.size[k], beg + kChunk);
        s += t.g_type[k] == ROCKET_F32 ? sum_squares<float>(t.g[k], beg, end)
             : t.g_type[k] == ROCKET_F16 ? sum_squares<__half>(t.g[k], beg, end) : sum_squares<__nv_bfloat16>(t.g[k], beg, end);
    }
    s = block_sum(s);
    if (threadIdx.x == 0) part[blockIdx.x] = s;
}

__global__ void __launch_bounds__(kThreads) norm_kernel(const double* __restrict__ part, int n, float* __restrict__ norm) {
    double s = 0.0;
    for (int i = threadIdx.x; i < n; i += kThreads) s += part[i];
    s = block_sum(s);
    if (threadIdx.x == 0) *norm = (float)sqrt(s);
}

template <class TG, class TO>
__device__ __forceinline__ void scale(const void* g, void* out, int64_t beg, int64_t end, float c) {
    for (int64_t i = beg + threadIdx.x; i < end; i += kThreads)
        static_cast<TO*>(out)[i] = from_float<TO>(to_float(static_cast<const TG*>(g)[i]) * c);
}

__global__ void __launch_bounds__(kThreads) scale_kernel(const __grid_constant__ Table t, const float* __restrict__ norm, float max_norm) {
    const float q = max_norm / (*norm + 1e-6f), c = q > 1.0f ? 1.0f : q;      // a NaN stays one
    for (int i = blockIdx.x; i < t.first[t.tensors]; i += gridDim.x) {
        const int k = tensor_of(t, i);
        const int64_t beg = (int64_t)(i - t.first[k]) * kChunk, end = min(t.size[k], beg + kChunk);
        if (t.g_type[k] == ROCKET_F32) scale<float, float>(t.g[k], t.out[k], beg, end, c);
        else if (t.g_type[k] == ROCKET_F16) t.out_type[k] == ROCKET_F32 ? scale<__half, float>(t.g[k], t.out[k], beg, end, c) : scale<__half, __half>(t.g[k], t.out[k], beg, end, c);
        else t.out_type[k] == ROCKET_F32 ? scale<__nv_bfloat16, float>(t.g[k], t.out[k], beg, end, c) : scale<__nv_bfloat16, __nv_bfloat16>(t.g[k], t.out[k], beg, end, c);
    }
}

int status_of(cudaError_t e) {
    if (e == cudaSuccess) return ROCKET_OK;
    cudaGetLastError();
    return e == cudaErrorMemoryAllocation ? ROCKET_ENOMEM : ROCKET_ECUDA;
}

using Span = std::pair<uintptr_t, uintptr_t>;

// Whether two of the spans share a byte (sorts them).
bool any_overlap(std::vector<Span>& s) {
    std::sort(s.begin(), s.end());
    for (size_t i = 1; i < s.size(); ++i) if (s[i].first < s[i - 1].second) return true;
    return false;
}

int64_t workspace_bytes_for(int count) { return 16 + (int64_t)sizeof(double) * kBlocks * ((count + (int64_t)kTensors - 1) / kTensors); }

// The arguments of both entry points; clip: whether gradients are written, to `out` or, where it is NULL, in place.
int check(int count, const void* const* grads, const int64_t* sizes, const int32_t* types, bool clip, void* const* out, const int32_t* out_types,
          const float* norm, const void* workspace, int64_t workspace_bytes) {
    if (count < 0 || !norm || (reinterpret_cast<uintptr_t>(norm) & 3u)) return ROCKET_EINVAL;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 15u) || workspace_bytes < workspace_bytes_for(count)) return ROCKET_EINVAL;
    if (count > 0 && (!grads || !sizes || !types || (out && !out_types))) return ROCKET_EINVAL;
    const Span own[] = {{(uintptr_t)norm, (uintptr_t)norm + 4}, {(uintptr_t)workspace, (uintptr_t)workspace + (uintptr_t)workspace_bytes_for(count)}};
    std::vector<Span> written(own, own + 2), read;
    int64_t chunks = 0;
    for (int i = 0; i < count; ++i) {
        if (sizes[i] < 0 || sizes[i] > (int64_t(1) << 40) || !is_float_type(types[i])) return ROCKET_EINVAL;
        if (out && (!is_float_type(out_types[i]) || (out_types[i] != types[i] && out_types[i] != ROCKET_F32))) return ROCKET_EINVAL;
        if (sizes[i] == 0) continue;
        chunks += (sizes[i] + kChunk - 1) / kChunk;
        const uintptr_t g = (uintptr_t)grads[i], o = out ? (uintptr_t)out[i] : g;
        const int gb = float_type_bytes(types[i]), ob = out ? float_type_bytes(out_types[i]) : gb;
        if (!g || !o || g % gb || o % ob) return ROCKET_EINVAL;
        if (clip) written.push_back({o, o + (uintptr_t)sizes[i] * ob});
        if (!clip || o != g || ob != gb) read.push_back({g, g + (uintptr_t)sizes[i] * gb});
    }
    if (chunks > 0x7fffffff) return ROCKET_EUNSUPPORTED;
    // what is written overlaps nothing; what is read may overlap itself (one tensor under two names counts twice)
    if (any_overlap(written)) return ROCKET_EINVAL;
    std::sort(read.begin(), read.end());
    size_t w = 0;
    for (const Span& r : read) {
        while (w < written.size() && written[w].second <= r.first) ++w;
        if (w < written.size() && written[w].first < r.second) return ROCKET_EINVAL;
    }
    return ROCKET_OK;
}

void fill(Table& t, int beg, int end, const void* const* grads, const int64_t* sizes, const int32_t* types, void* const* out, const int32_t* out_types) {
    t.tensors = end - beg;
    t.first[0] = 0;
    for (int i = beg; i < end; ++i) {
        const int k = i - beg;
        t.g[k] = grads[i];
        t.out[k] = out ? out[i] : const_cast<void*>(grads[i]);
        t.size[k] = sizes[i];
        t.g_type[k] = (uint8_t)types[i];
        t.out_type[k] = (uint8_t)(out ? out_types[i] : types[i]);
        t.first[k + 1] = t.first[k] + (int)((sizes[i] + kChunk - 1) / kChunk);
    }
}

int run(int count, const void* const* grads, const int64_t* sizes, const int32_t* types, bool clip, void* const* out, const int32_t* out_types,
        float max_norm, float* norm, void* workspace, cudaStream_t stream) {
    double* part = static_cast<double*>(workspace);
    int parts = 0;
    Table t;
    for (int beg = 0; beg < count; beg += kTensors) {
        fill(t, beg, std::min(count, beg + kTensors), grads, sizes, types, out, out_types);
        const int blocks = std::min(t.first[t.tensors], kBlocks);
        if (!blocks) continue;
        squares_kernel<<<blocks, kThreads, 0, stream>>>(t, part + parts);
        count_launch();
        parts += blocks;
    }
    norm_kernel<<<1, kThreads, 0, stream>>>(part, parts, norm);
    count_launch();
    for (int beg = 0; clip && beg < count; beg += kTensors) {
        fill(t, beg, std::min(count, beg + kTensors), grads, sizes, types, out, out_types);
        const int blocks = std::min(t.first[t.tensors], kBlocks);
        if (!blocks) continue;
        scale_kernel<<<blocks, kThreads, 0, stream>>>(t, norm, max_norm);
        count_launch();
    }
    return status_of(cudaGetLastError());
}

}  // namespace
}  // namespace rocket

using namespace rocket;

extern "C" int64_t rocket_grad_norm_workspace(int count) { return count < 0 ? ROCKET_EINVAL : workspace_bytes_for(count); }

extern "C" int rocket_grad_norm(int count, const void* const* grads_dev, const int64_t* sizes, const int32_t* types, float* norm_dev,
                                void* workspace_dev, int64_t workspace_bytes, void* cuda_stream) {
    try {
        const int st = check(count, grads_dev, sizes, types, false, nullptr, nullptr, norm_dev, workspace_dev, workspace_bytes);
        if (st != ROCKET_OK) return st;
    } catch (const std::bad_alloc&) {
        return ROCKET_ENOMEM;
    }
    return run(count, grads_dev, sizes, types, false, nullptr, nullptr, 0.0f, norm_dev, workspace_dev, static_cast<cudaStream_t>(cuda_stream));
}

extern "C" int rocket_clip_grad_norm(int count, const void* const* grads_dev, const int64_t* sizes, const int32_t* types,
                                     void* const* out_dev, const int32_t* out_types, float max_norm, float* norm_dev,
                                     void* workspace_dev, int64_t workspace_bytes, void* cuda_stream) {
    if (!(max_norm >= 0.0f)) return ROCKET_EINVAL;
    try {
        const int st = check(count, grads_dev, sizes, types, true, out_dev, out_types, norm_dev, workspace_dev, workspace_bytes);
        if (st != ROCKET_OK) return st;
    } catch (const std::bad_alloc&) {
        return ROCKET_ENOMEM;
    }
    return run(count, grads_dev, sizes, types, true, out_dev, out_types, max_norm, norm_dev, workspace_dev, static_cast<cudaStream_t>(cuda_stream));
}
