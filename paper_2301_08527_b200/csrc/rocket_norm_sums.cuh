// Sums over the threads that own a row, shared by the layer norm kernels of both directions.
#pragma once

#include <cooperative_groups.h>

#include <algorithm>
#include <atomic>
#include <cstdint>
#include <type_traits>

namespace rocket {
namespace norm {

namespace cg = cooperative_groups;

constexpr int kSms = 148;
constexpr int kMostParts = 8;             // blocks of a cluster

enum Owner { kWarp, kBlock, kCluster };

// Sums of a value over all threads that own the row, the same bits in each.  The two reductions of a row have buffers of their own,
// so that one barrier each is enough: a warp that writes for the next row has passed the other's, behind everybody's reads.
__device__ __forceinline__ float add_lanes(float v, int from) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        if (o <= from) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

template <Owner OWNER>
__device__ __forceinline__ float row_sum(float v, int parts, int rank, int half) {
    v = add_lanes(v, 16);
    if constexpr (OWNER != kWarp) {
        __shared__ float red[32];
        const int lane = threadIdx.x & 31, warps = blockDim.x >> 5;
        if (lane == 0) red[threadIdx.x >> 5] = v;
        __syncthreads();
        const int l = half ? lane & (2 * half - 1) : 0;                     // 2 half: the warps, rounded up to a power of two
        v = add_lanes(l < warps ? red[l] : 0.0f, half);
        if constexpr (OWNER == kCluster) {
            __shared__ float share[kMostParts];
            cg::cluster_group cluster = cg::this_cluster();
            if ((int)threadIdx.x < parts) *cluster.map_shared_rank(&share[rank], threadIdx.x) = v;
            cluster.sync();
            v = share[0];
            for (int p = 1; p < parts; ++p) v += share[p];
        }
    }
    return v;
}

// The same of two values: each half of a warp goes on with one of them, which saves nearly half of the shuffles.  A kernel that has this
// reduction alone gives its rows' numbers as `phase`: with two sets of buffers one barrier a row is enough again.
template <Owner OWNER>
__device__ __forceinline__ float2 row_sums(float2 v, int parts, int rank, int phase) {
    const int lane = threadIdx.x & 31;
    const bool upper = lane >= 16;
    float s = (upper ? v.y : v.x) + __shfl_xor_sync(0xffffffffu, upper ? v.x : v.y, 16);
    s = add_lanes(s, 8);
    if constexpr (OWNER != kWarp) {
        __shared__ float reds[2][2][32];
        auto& red = reds[phase & 1];
        const int warps = blockDim.x >> 5;
        if ((lane & 15) == 0) red[lane >> 4][threadIdx.x >> 5] = s;
        __syncthreads();
        const int l = lane & 15;
        s = (l < warps ? red[lane >> 4][l] : 0.0f) + (l + 16 < warps ? red[lane >> 4][l + 16] : 0.0f);
        s = add_lanes(s, 8);
    }
    v = make_float2(__shfl_sync(0xffffffffu, s, 0), __shfl_sync(0xffffffffu, s, 16));
    if constexpr (OWNER == kCluster) {
        __shared__ float2 shares[2][kMostParts];
        auto& share = shares[phase & 1];
        cg::cluster_group cluster = cg::this_cluster();
        if ((int)threadIdx.x < parts) *cluster.map_shared_rank(&share[rank], threadIdx.x) = v;
        cluster.sync();
        v = share[0];
        for (int p = 1; p < parts; ++p) { v.x += share[p].x; v.y += share[p].y; }
    }
    return v;
}

// Runs set() once for every device that is current at a call (done: a bit for each).
template <class F>
inline cudaError_t once_per_device(std::atomic<uint64_t>& done, F&& set) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    const uint64_t bit = uint64_t(1) << (dev & 63);
    if (e != cudaSuccess || (dev < 64 && (done.load(std::memory_order_relaxed) & bit))) return e;
    e = set();
    if (e == cudaSuccess && dev < 64) done.fetch_or(bit, std::memory_order_relaxed);
    return e;
}

// Clusters of `kernel` that run at the same time, asked for once and kept in `known` (all devices are alike).
template <class K>
inline cudaError_t active_clusters(std::atomic<int>& known, K kernel, const cudaLaunchConfig_t& cfg, int& clusters) {
    clusters = known.load(std::memory_order_relaxed);
    if (clusters > 0) return cudaSuccess;
    const cudaError_t e = cudaOccupancyMaxActiveClusters(&clusters, kernel, &cfg);
    clusters = std::max(clusters, 1);
    if (e == cudaSuccess) known.store(clusters, std::memory_order_relaxed);
    return e;
}

inline int round32(int v) { return (v + 31) / 32 * 32; }

// row_sum's `half` for a block of this many threads.
inline int half_of(int threads) {
    int half = 0;
    while (std::max(2 * half, 1) < threads / 32) half = std::max(2 * half, 1);
    return half;
}

template <int N> using Int = std::integral_constant<int, N>;

// Calls f with the constant `v` of LO .. HI.
template <int LO, int HI, class F>
cudaError_t with_int(int v, F&& f) {
    if constexpr (LO < HI) if (v > LO) return with_int<LO + 1, HI>(v, f);
    return f(Int<LO>());
}

}  // namespace norm
}  // namespace rocket
