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

// How the words of a block's threads lie in its part of a row.  kFull: all threads have all their words.  kLast: all but the last for all.  Both with rows
// that bulk copies bring whole.  kEnd: as kLast, but a row may begin and end anywhere.  kAny: so, and threads may have fewer words.  Where a row comes
// from shared memory, a word beyond the end is then read as the last one, which keeps the loads of all words under way at once, and counts as
// nothing.
enum Fit { kAny, kEnd, kLast, kFull };

// A bounded wait that does not sleep at first: what it waits for is nearly always there, or about to be.
__device__ __forceinline__ bool wait_soon(uint32_t bar, uint32_t parity) {
    for (int i = 0; i < 8; ++i)
        if (fast::mbar_try(bar, parity)) return true;
    return fast::mbar_wait(bar, parity);
}

// Bytes of shared memory for a part of a row that may begin anywhere between two 16-byte borders.
__host__ __device__ constexpr int room_of(int part, int bytes) { return (part * bytes + 16 + 127) / 128 * 128; }

// A piece of a row, n values at p, on its way to shared memory.  Bulk copies bring the whole 16-byte units within it, to the same place relative to
// a 16-byte border; the up to 7 values before the first and behind the last border are stored there by a lane each.
template <class T>
struct Piece {
    int skew, head, tail;         // bytes from the last border to p; values before the first copied one; the first value behind the copied ones
    __device__ __forceinline__ Piece(const T* p, int n) {
        skew = (int)(reinterpret_cast<uintptr_t>(p) & 15);
        head = ((16 - skew) & 15) / (int)sizeof(T);
        tail = max(head, (int)(((unsigned)skew + (unsigned)n * (unsigned)sizeof(T)) / 16u * 16u - (unsigned)skew) / (int)sizeof(T));
    }
    __device__ __forceinline__ uint32_t copied() const { return (uint32_t)((tail - head) * (int)sizeof(T)); }
    __device__ __forceinline__ void copy(uint32_t dst, const T* p, uint32_t bar) const {
        if (tail > head) fast::bulk_g2s(dst + (uint32_t)(skew + head * (int)sizeof(T)), p + head, copied(), bar);
    }
};

// What one of 16 lanes has to bring of a piece: where to put it (bytes from the piece's place in shared memory; -1: nothing) and its bits.
template <class T>
struct Edge {
    int to = -1;
    std::conditional_t<sizeof(T) == 4, unsigned, unsigned short> bits = 0;
    __device__ __forceinline__ void fetch(const T* p, int n, int lane) {
        const Piece<T> piece(p, n);
        const int i = lane < 8 ? lane : piece.tail + lane - 8;
        to = -1;
        if (lane < 8 ? i < piece.head && i < n : i < n) {
            to = piece.skew + i * (int)sizeof(T);
            bits = __ldg(reinterpret_cast<const decltype(bits)*>(p + i));
        }
    }
    __device__ __forceinline__ void put(unsigned char* place) const {
        if (to >= 0) *reinterpret_cast<std::remove_const_t<decltype(bits)>*>(place + to) = bits;
    }
};

// Sums over the lanes whose numbers differ in the bits from `from` down, the same bits in each.
__device__ __forceinline__ float add_lanes(float v, int from) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        if (o <= from) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// Two or four values (V: float2, float4) of every block of a cluster, handed to all of its blocks by stores that count on the receiver's barrier: nothing
// waits for the rows written meanwhile, as a cluster-wide barrier would.  One exchange per row; with two sets of buffers a block that is
// ahead writes where nobody reads any more: it has everybody's values of the row before, sent behind the block barrier that follows
// their reads.
template <class V>
struct Exchange {
    V share[2][kMostParts];
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
    __device__ __forceinline__ const V* swap(V v, int parts, int rank, int turn, bool& ok) {
        const int set = turn & 1;
        if (threadIdx.x == 0) fast::mbar_arrive_expect_tx(fast::smem_u32(&bar[set]), (uint32_t)(parts * sizeof(V)));
        if ((int)threadIdx.x < parts) {
            uint32_t to, on;
            asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(fast::smem_u32(&share[set][rank])), "r"((int)threadIdx.x));
            asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(on) : "r"(fast::smem_u32(&bar[set])), "r"((int)threadIdx.x));
            if constexpr (sizeof(V) == 16)
                asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];"
                             ::"r"(to), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w), "r"(on) : "memory");
            else
                asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];"
                             ::"r"(to), "f"(v.x), "f"(v.y), "r"(on) : "memory");
        }
        ok = ok && wait_soon(fast::smem_u32(&bar[set]), (uint32_t)((turn >> 1) & 1));
        return share[set];
    }
};

// No block of a cluster ends while another may still write to its shared memory.  (Each has what was sent to it before it arrives; a block that
// still reads another's memory needs an arrival that releases.)
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
