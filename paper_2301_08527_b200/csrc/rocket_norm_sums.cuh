// Sums over the threads that own a row, shared by the layer norm kernels of both directions.
#pragma once

#include <algorithm>
#include <atomic>
#include <cstdint>
#include <type_traits>

#include "rocket_fast_dev.cuh"

namespace rocket {
namespace norm {

constexpr int kSms = 148;
constexpr int kMostParts = 16;            // blocks of a cluster

enum Owner { kWarp, kBlock, kCluster };

// A bounded wait that does not sleep at first: what it waits for is nearly always there, or about to be.
__device__ __forceinline__ bool wait_soon(uint32_t bar, uint32_t parity) {
    for (int i = 0; i < 8; ++i)
        if (fast::mbar_try(bar, parity)) return true;
    return fast::mbar_wait(bar, parity);
}

// Sums over the lanes whose numbers differ in the bits from `from` down, the same bits in each.
__device__ __forceinline__ float add_lanes(float v, int from) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        if (o <= from) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// Two values of every block of a cluster, handed to all of its blocks by stores that count on the receiver's barrier: nothing
// waits for the rows written meanwhile, as a cluster-wide barrier would.  One exchange per row; with two sets of buffers a block that is
// ahead writes where nobody reads any more: it has everybody's values of the row before, sent behind the block barrier that follows
// their reads.
struct Exchange {
    float2 share[2][kMostParts];
    uint64_t bar[2];

    // Behind it, all blocks of the cluster must meet before the first exchange.
    __device__ __forceinline__ void init() {
        if (threadIdx.x == 0) {
            fast::mbar_init(fast::smem_u32(&bar[0]), 1);
            fast::mbar_init(fast::smem_u32(&bar[1]), 1);
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
    }

    // All threads call it with the block's value v; returns the set of buffers that holds everybody's.  turn: 0, 1, 2 ..  false in ok: a wait
    // gave up, and nothing is waited for after that.
    __device__ __forceinline__ const float2* swap(float2 v, int parts, int rank, int turn, bool& ok) {
        const int set = turn & 1;
        if (threadIdx.x == 0) fast::mbar_arrive_expect_tx(fast::smem_u32(&bar[set]), (uint32_t)(parts * sizeof(float2)));
        if ((int)threadIdx.x < parts) {
            uint32_t to, on;
            asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(fast::smem_u32(&share[set][rank])), "r"((int)threadIdx.x));
            asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(on) : "r"(fast::smem_u32(&bar[set])), "r"((int)threadIdx.x));
            asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];"
                         ::"r"(to), "f"(v.x), "f"(v.y), "r"(on) : "memory");
        }
        ok = ok && wait_soon(fast::smem_u32(&bar[set]), (uint32_t)((turn >> 1) & 1));
        return share[set];
    }
};

// No block of a cluster ends while another may still write to its shared memory.
__device__ __forceinline__ void leave_cluster() {
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
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

// Lets `kernel` run in clusters of more than eight blocks.
template <class K>
inline cudaError_t allow_large_clusters(K kernel) { return cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1); }

// Clusters of `kernel` that run at the same time, asked for once and kept in `known` (all devices are alike).
template <class K>
inline cudaError_t active_clusters(std::atomic<int>& known, K kernel, const cudaLaunchConfig_t& cfg, int& clusters) {
    clusters = known.load(std::memory_order_relaxed);
    if (clusters > 0) return cudaSuccess;
    cudaError_t e = cudaOccupancyMaxActiveClusters(&clusters, kernel, &cfg);
    clusters = std::max(clusters, 1);
    if (e == cudaSuccess) known.store(clusters, std::memory_order_relaxed);
    return e;
}

inline int round32(int v) { return (v + 31) / 32 * 32; }

template <int N> using Int = std::integral_constant<int, N>;

// Calls f with the constant `v` of LO .. HI.
template <int LO, int HI, class F>
cudaError_t with_int(int v, F&& f) {
    if constexpr (LO < HI) if (v > LO) return with_int<LO + 1, HI>(v, f);
    return f(Int<LO>());
}

}  // namespace norm
}  // namespace rocket
