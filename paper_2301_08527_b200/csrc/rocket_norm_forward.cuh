// Layer norm forward: m = mean(x), v = mean((x - m)^2), r = 1 / sqrt(v + eps), y = (x - m) r g + b for every row.
//
// Bound: memory.  A row is read once and stays in registers while its owner's next row is on its way.  A thread takes the mean of its values,
// as c + l with l a rounding of c (from the differences to its first value, which are exact where the row is far from zero), keeps the values as
// d = x - c, and takes the mean square q of d.  Where sets of values meet, with a share s of the whole, mean and q each, the whole has the mean
// sum s c and q = sum s (q + (c - whole's c)^2) (Chan, Golub and LeVeque); means are handed on as such pairs and added up as differences to the first set's.  So
// everything is held by its distance from a mean of some of the row's values, d + (c - mean) is y's numerator, and neither a row's distance from
// zero nor single values unlike the others cost the rest their digits; the threads of a block need one barrier, the blocks of a cluster one
// exchange per row.
//
// Who has a row: a warp where it is short, a block, or the blocks of a cluster where rows are few or longer than a block's
// registers.  The owners stay and go through the rows in turn.
//
// Measured: 16,384 x 4,096 bf16 50 us, 5.4 TB/s or 83 % of a copy (56 with two barriers a row and 16 values a thread, whose sums then are a third of the
// instructions; 79 with a block per row and no rows ahead); 677 x 20,000 fp32 to bf16 18 us (28 with a block of 1,024 threads per row that fetches gamma
// and beta again for each).
#pragma once

#include <algorithm>
#include <cfloat>

#include "rocket_float_types.cuh"
#include "rocket_internal.h"
#include "rocket_norm.h"
#include "rocket_norm_sums.cuh"

namespace rocket {
namespace norm {

// Where gamma and beta come from: registers, filled once (kHold); loads of a type known at compile time, both being there (kAsFloat,
// kAsInput: fp32, the input's); loads that ask (kAsk).
enum Weights { kAsk, kHold, kAsFloat, kAsInput };

constexpr int kMostStages = 8;
constexpr int kSmemSm = 227 * 1024;       // shared memory of an SM

// Threads that hold gamma and beta: 32 values of each, or 16 where they are loaded one by one; most threads of a block, and of one in a cluster.
constexpr int held_values(int W) { return W == 1 ? 16 : 32; }
__host__ __device__ constexpr int hold_threads(Owner owner, int values) { return values < 16 ? 1024 : (owner == kCluster ? 160 : 128) * (32 / values); }

__host__ __device__ constexpr int most_threads(Owner owner, Weights weights, int values) {
    return owner == kWarp ? 256 : weights == kHold ? hold_threads(owner, values) : 1024;
}

// Blocks of an SM that the registers are cut for.
constexpr int resident_blocks(Owner owner, Weights weights, int values) {
    return owner == kWarp ? (values <= 10 ? 4 : values <= 14 ? 3 : 2) : weights == kHold && values >= 16 ? (owner == kCluster ? (values == 32 ? 3 : 2) : values == 32 ? 4 : 3) : 1;
}

// W values per word, NV words per thread.  RING: a block's next rows come into shared memory by bulk copies, as many ahead as there are stages (a
// thread that gives up waiting counts as NaN, which makes the row NaN); else the threads hold the next one in registers.  LANES of a warp share a
// row; a warp has 32 / LANES rows at a time.
template <class T, int W, int NV, Owner OWNER, Weights WEIGHTS, Fit FIT, bool RING = false, int LANES = 32>
__global__ void __launch_bounds__(most_threads(OWNER, WEIGHTS, NV * W), resident_blocks(OWNER, WEIGHTS, NV * W))
rows_kernel(const Forward a, int parts, int stages, int stage_words) {
    extern __shared__ __align__(128) unsigned char ring[];
    __shared__ __align__(8) uint64_t arrived[RING ? kMostStages : 1];
    int64_t row, rows;
    int beg = 0, words = a.P / W, first, step, rank = 0;
    __shared__ Exchange<float4> exchange;
    if constexpr (OWNER == kWarp) {
        row = (int64_t)blockIdx.x * (blockDim.x / LANES) + (threadIdx.x >> 5) * (32 / LANES);      // the warp's first; its lanes' below
        rows = (int64_t)gridDim.x * (blockDim.x / LANES);
        first = threadIdx.x & (LANES - 1);
        step = LANES;
    } else {
        row = blockIdx.x / parts;
        rows = gridDim.x / parts;
        if constexpr (OWNER == kCluster) {
            exchange.init();
            rank = blockIdx.x % parts;
            const int all = words, from = (int)((int64_t)all * rank / parts);
            beg = from * W;
            words = (int)((int64_t)all * (rank + 1) / parts) - from;
            asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
        }
        first = threadIdx.x;
        step = blockDim.x;
    }
    const bool last = first + (NV - 1) * step < words;
    auto has = [&](int k) { return FIT == kFull || (FIT == kAny ? first + k * step < words : k < NV - 1 || last); };
    constexpr bool kEdges = RING && (FIT == kAny || FIT == kEnd);
    auto may_miss = [](int k) { return kEdges && (FIT == kAny || k == NV - 1); };      // read all the same, and counted as nothing
    const int at = beg + first * W;
    Packed<T, W> next[RING ? 1 : NV];
    const int ahead = OWNER == kWarp ? (threadIdx.x & 31) / LANES : 0;
    const T* source = static_cast<const T*>(a.x) + (row + ahead) * a.x_stride;
    const int64_t source_step = rows * a.x_stride;
    auto fetch = [&](int64_t n) {
        const T* from = source + at;
        if (LANES < 32 && n + ahead >= a.N) return;
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (has(k)) next[RING ? 0 : k] = load_packed_once<T, W>(from + k * step * W);
        source += source_step;
    };
    const uint32_t bars = fast::smem_u32(arrived), rings = fast::smem_u32(ring), stage_bytes = (uint32_t)room_of(stage_words * W, sizeof(T));
    const int columns = words * W;
    int64_t to_copy = row;
    auto copy = [&](int stage) {
        const uint32_t bar = bars + 8u * stage, dst = rings + (uint32_t)stage * stage_bytes;
        if constexpr (kEdges) {
            const Piece<T> piece(source + beg, columns);
            fast::mbar_arrive_expect_tx(bar, piece.copied());
            piece.copy(dst, source + beg, bar);
        } else {
            fast::mbar_arrive_expect_tx(bar, (uint32_t)(columns * (int)sizeof(T)));
            fast::bulk_g2s(dst, source + beg, (uint32_t)(columns * (int)sizeof(T)), bar);
        }
        source += source_step;
        to_copy += rows;
    };
    // the values that no bulk copy brings: the first lanes fetch them two rows ahead and store them one row ahead
    Edge<T> edge;
    auto fetch_edge = [&](int64_t n) {
        edge.to = -1;
        if (n < a.N && threadIdx.x < 16) edge.fetch(static_cast<const T*>(a.x) + n * a.x_stride + beg, columns, threadIdx.x);
    };
    int stage = 0;
    uint32_t parity = 0;
    if constexpr (RING) {
        if (threadIdx.x == 0) {
            for (int i = 0; i < stages; ++i) fast::mbar_init(bars + 8u * i, 1);
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
            for (int i = 0; i < stages && to_copy < a.N; ++i) copy(i);
        }
        if constexpr (kEdges) {
            fetch_edge(row);
            edge.put(ring);
            fetch_edge(row + rows);
        }
    } else {
        if (row < a.N) fetch(row);
    }
    float g[WEIGHTS == kHold ? NV : 1][W], b[WEIGHTS == kHold ? NV : 1][W];
    if constexpr (WEIGHTS == kHold)
#pragma unroll
        for (int k = 0; k < NV; ++k) {
#pragma unroll
            for (int j = 0; j < W; ++j) { g[k][j] = 1.0f; b[k][j] = 0.0f; }
            if (a.gamma && has(k)) load_typed<W>(a.gamma, a.w_type, at + k * step * W, g[k]);
            if (a.beta && has(k)) load_typed<W>(a.beta, a.w_type, at + k * step * W, b[k]);
        }
    // Values of this thread, its warp, its lane's warp, and the block.  Sets are joined by their shares of the whole, means and mean squares, not
    // sums, so that a row of large values leaves fp32's range only where the means themselves do.
    const int n_thread = ((words - first + step - 1) / step) * W;
    const float n = (float)(words > first ? n_thread : 0), over_n = n > 0.0f ? 1.0f / n : 0.0f;
    const float n_warp = add_lanes(n, LANES / 2), share = n_warp > 0.0f ? n / n_warp : 0.0f;
    constexpr int kMostWarps = most_threads(OWNER, WEIGHTS, NV * W) / 32;
    __shared__ float warp_n[kMostWarps];
    const int warps = blockDim.x >> 5;
    float share_warp = 0.0f;
    if constexpr (OWNER != kWarp) {
        if ((threadIdx.x & 31) == 0) warp_n[threadIdx.x >> 5] = n_warp;
        __syncthreads();
        share_warp = (threadIdx.x & 31) < warps ? warp_n[threadIdx.x & 31] / (float)(words * W) : 0.0f;
    }
    // the cluster's blocks, a lane for each in both halves of a warp
    const int part_lane = threadIdx.x & (kMostParts - 1);
    float share_part = 0.0f;
    if (OWNER == kCluster && part_lane < parts) {
        const int64_t all = a.P / W;
        share_part = (float)(((int)(all * (part_lane + 1) / parts) - (int)(all * part_lane / parts)) * W) / (float)a.P;
    }
    if constexpr (OWNER == kCluster) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    bool ok = true;
    for (int turn = 0; row < a.N; row += rows, ++turn) {
        float f[NV][W];
        if constexpr (RING) {
            ok = ok && wait_soon(bars + 8u * stage, parity);
            const unsigned char* in = ring + (size_t)stage * stage_bytes;
            const T* x = reinterpret_cast<const T*>(in);
            if constexpr (kEdges) {
                x = reinterpret_cast<const T*>(in + (reinterpret_cast<uintptr_t>(static_cast<const T*>(a.x) + row * a.x_stride + beg) & 15));
                edge.put(ring + (size_t)(stage + 1 == stages ? 0 : stage + 1) * stage_bytes);
                fetch_edge(row + 2 * rows);
            }
#pragma unroll
            for (int k = 0; k < NV; ++k)
                if (kEdges || has(k)) {
                    unpack<T, W>(load_packed<T, W>(x + (may_miss(k) ? min(first + k * step, words - 1) : first + k * step) * W), f[k]);
                    if (may_miss(k) && !has(k))
#pragma unroll
                        for (int j = 0; j < W; ++j) f[k][j] = f[0][0];
                }
        } else {
#pragma unroll
            for (int k = 0; k < NV; ++k)
                if (has(k)) unpack<T, W>(next[RING ? 0 : k], f[k]);
            if (row + rows < a.N) fetch(row + rows);
        }
        // the thread's mean c + l, from its first value on
        const float x0 = RING && !ok ? __int_as_float(0x7fc00000) : kEdges || has(0) ? f[0][0] : 0.0f;
        float s[2] = {0.0f, 0.0f}, q[2] = {0.0f, 0.0f};         // two chains each
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (kEdges || has(k))
#pragma unroll
                for (int j = 0; j < W; ++j) s[(k * W + j) & 1] = fmaf(f[k][j] - x0, over_n, s[(k * W + j) & 1]);
        const float from0 = s[0] + s[1], c = x0 + from0, l = (x0 - c) + from0;
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (kEdges || has(k))
#pragma unroll
                for (int j = 0; j < W; ++j) {
                    f[k][j] = may_miss(k) && !has(k) ? 0.0f : f[k][j] - c;
                    q[(k * W + j) & 1] = fmaf(f[k][j], f[k][j], q[(k * W + j) & 1]);
                }
        // the warp's: mean from a reference on, the first lane's c.  q / n is about c, so l^2 too large: e^2 - l^2 = h (h + 2 l) comes to it with
        // e = h + l, the distance of the thread's mean from the warp's (beyond fp32's range it stays infinite).
        float ref = __shfl_sync(0xffffffffu, c, 0, LANES), square = (q[0] + q[1]) * over_n;
        float mean = add_lanes(share * ((c - ref) + l), LANES / 2);
        const float h = (c - ref) - mean;
        square = add_lanes(square > FLT_MAX ? square : fmaf(share * h, h + 2.0f * l, share * square), LANES / 2);
        if constexpr (OWNER != kWarp) {
            __shared__ float4 sets[2][kMostWarps];                // mean's two parts and the mean square; taken in turn: one barrier a row is enough
            const int lane = threadIdx.x & 31;
            float high = ref + mean;
            if (lane == 0) sets[turn & 1][threadIdx.x >> 5] = make_float4(high, (ref - high) + mean, square, 0.0f);
            __syncthreads();
            if constexpr (RING) {
                // everybody has the row in registers: another may come into its place
                if (threadIdx.x == 0 && ok && to_copy < a.N) {
                    if constexpr (kEdges) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");      // behind the stores of the edges
                    copy(stage);
                }
                if (++stage == stages) { stage = 0; parity ^= 1u; }
            }
            ref = sets[turn & 1][0].x;
            const float4 of = lane < warps ? sets[turn & 1][lane] : make_float4(ref, 0.0f, 0.0f, 0.0f);
            float from = (of.x - ref) + of.y;
            mean = add_lanes(share_warp * from, 16);
            float e = from - mean;
            square = add_lanes(fmaf(share_warp * e, e, share_warp * of.z), 16);
            if constexpr (OWNER == kCluster) {
                high = ref + mean;
                const float4* all = exchange.swap(make_float4(high, (ref - high) + mean, square, 0.0f), parts, rank, turn, ok);
                ref = all[0].x;
                const float4 theirs = part_lane < parts ? all[part_lane] : make_float4(ref, 0.0f, 0.0f, 0.0f);
                from = (theirs.x - ref) + theirs.y;
                mean = add_lanes(share_part * from, kMostParts / 2);
                e = from - mean;
                square = add_lanes(fmaf(share_part * e, e, share_part * theirs.z), kMostParts / 2);
                if (!ok) square = __int_as_float(0x7fc00000);
            }
        }
        const float r = rsqrtf(square + a.eps), off = ((c - ref) - mean) * r;
        auto write = [&](auto* y) {
            y += (row + ahead) * a.y_stride + at;
#pragma unroll
            for (int k = 0; k < NV; ++k)
                if (has(k)) {
                    const int i = at + k * step * W, h = WEIGHTS == kHold ? k : 0;
                    float o[W];
                    if constexpr (WEIGHTS == kAsFloat) {
                        unpack<float, W>(load_packed_ro<float, W>(static_cast<const float*>(a.gamma) + i), g[0]);
                        unpack<float, W>(load_packed_ro<float, W>(static_cast<const float*>(a.beta) + i), b[0]);
                    } else if constexpr (WEIGHTS == kAsInput) {
                        unpack<T, W>(load_packed_ro<T, W>(static_cast<const T*>(a.gamma) + i), g[0]);
                        unpack<T, W>(load_packed_ro<T, W>(static_cast<const T*>(a.beta) + i), b[0]);
                    } else if constexpr (WEIGHTS == kAsk) {
#pragma unroll
                        for (int j = 0; j < W; ++j) { g[0][j] = 1.0f; b[0][j] = 0.0f; }
                        if (a.gamma) load_typed<W>(a.gamma, a.w_type, i, g[0]);
                        if (a.beta) load_typed<W>(a.beta, a.w_type, i, b[0]);
                    }
#pragma unroll
                    for (int j = 0; j < W; ++j) o[j] = fmaf(fmaf(f[k][j], r, off), g[h][j], b[h][j]);
                    store_packed(y + k * step * W, o);
                }
        };
        if (LANES < 32 && row + ahead >= a.N) break;              // the warp's last turn
        if (a.y_type == ROCKET_F32) write(static_cast<float*>(a.y));
        else if (a.y_type == ROCKET_F16) write(static_cast<__half*>(a.y));
        else write(static_cast<__nv_bfloat16*>(a.y));
        if (first == 0 && rank == 0) {
            if (a.mean) a.mean[row + ahead] = ref + mean;
            if (a.rstd) a.rstd[row + ahead] = r;
        }
    }
    // copies that a wait gave up on must not outlive the block
    if (RING && threadIdx.x == 0 && !ok)
        for (int i = 0; i < stages; ++i) {
            fast::mbar_wait(bars + 8u * stage, parity);
            if (++stage == stages) { stage = 0; parity ^= 1u; }
        }
    if constexpr (OWNER == kCluster) leave_cluster();
}

// Rows longer than the registers of a cluster: a block per row, the row read three times, its sums in double precision.
constexpr int kLongThreads = 1024;
__device__ __forceinline__ double2 block_sums(double2 s) {
    __shared__ double2 red[kLongThreads / 32];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        s.x += __shfl_xor_sync(0xffffffffu, s.x, o);
        s.y += __shfl_xor_sync(0xffffffffu, s.y, o);
    }
    __syncthreads();
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = s;
    __syncthreads();
    s = make_double2(0.0, 0.0);
#pragma unroll
    for (int w = 0; w < kLongThreads / 32; ++w) { s.x += red[w].x; s.y += red[w].y; }
    return s;
}

template <class T>
__global__ void __launch_bounds__(kLongThreads) long_rows_kernel(const Forward a) {
    const T* __restrict__ x = static_cast<const T*>(a.x) + (int64_t)blockIdx.x * a.x_stride;
    double2 s = make_double2(0.0, 0.0);
    for (int64_t i = threadIdx.x; i < a.P; i += kLongThreads) s.x += (double)to_float(x[i]);
    const float m = (float)(block_sums(s).x / (double)a.P);
    s = make_double2(0.0, 0.0);
    for (int64_t i = threadIdx.x; i < a.P; i += kLongThreads) {
        const double d = (double)to_float(x[i]) - (double)m;
        s.x += d;
        s.y += d * d;
    }
    s = block_sums(s);
    const double rest = s.x / (double)a.P;
    const double v = s.y / (double)a.P - rest * rest;
    const float r = (float)(1.0 / sqrt((v < 0.0 ? 0.0 : v) + (double)a.eps));
    for (int64_t i = threadIdx.x; i < a.P; i += kLongThreads) {
        float o[1] = {((to_float(x[i]) - m) - (float)rest) * r}, w[1];
        if (a.gamma) { load_typed<1>(a.gamma, a.w_type, i, w); o[0] *= w[0]; }
        if (a.beta) { load_typed<1>(a.beta, a.w_type, i, w); o[0] += w[0]; }
        store_typed<1>(a.y, a.y_type, (int64_t)blockIdx.x * a.y_stride + i, o);
    }
    if (threadIdx.x == 0) {
        if (a.mean) a.mean[blockIdx.x] = (float)((double)m + rest);
        if (a.rstd) a.rstd[blockIdx.x] = r;
    }
}

// Shared memory for a block's rows: 2 KB less than its share, for its other arrays and what the driver keeps.
inline int ring_bytes(int resident) { return kSmemSm / resident - 2048; }

template <class T, int W, int NV, Owner OWNER, Weights WEIGHTS, Fit FIT, int LANES = 32>
cudaError_t launch(const Forward& a, int threads, int parts, cudaStream_t stream) {
    auto kernel = rows_kernel<T, W, NV, OWNER, WEIGHTS, FIT, false, LANES>;
    static std::atomic<int> known[1024 / 32 + 1];                        // resident blocks of an SM, by warps; all devices are alike
    int resident = known[threads / 32].load(std::memory_order_relaxed);
    if (resident == 0) {
        const cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&resident, kernel, threads, 0);
        if (e != cudaSuccess) return e;
        known[threads / 32].store(resident, std::memory_order_relaxed);
    }
    const int64_t owners = OWNER == kWarp ? threads / LANES : 1;            // rows of a block
    const int64_t most = (int64_t)kSms * std::max(resident, 1) / parts;
    const int64_t blocks = std::min(((int64_t)a.N + owners - 1) / owners, std::max<int64_t>(most, 1)) * parts;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)parts;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = OWNER == kCluster ? 1 : 0;
    if constexpr (OWNER == kCluster) {
        // not every SM finds partners in its group of SMs: clusters that would have to wait for others to end cost a second round
        static std::atomic<uint64_t> allowed{0};
        static std::atomic<int> clusters[kMostParts + 1][1024 / 32 + 1];
        int at_once = 0;
        cudaError_t e = parts > 8 ? once_per_device(allowed, [&] { return allow_large_clusters(kernel); }) : cudaSuccess;
        if (e == cudaSuccess) e = active_clusters(clusters[parts][threads / 32], kernel, cfg, at_once);
        if (e != cudaSuccess) return e;
        cfg.gridDim = dim3((unsigned)std::min<int64_t>(blocks, (int64_t)at_once * parts));
    }
    count_launch();
    return cudaLaunchKernelEx(&cfg, kernel, a, parts, 0, 0);
}

// Blocks of `resident` per SM, each with as many stages as there is memory for.
template <class T, int W, int NV, Owner OWNER, Weights WEIGHTS, Fit FIT>
cudaError_t launch_ring(const Forward& a, int threads, int parts, int resident, cudaStream_t stream) {
    auto kernel = rows_kernel<T, W, NV, OWNER, WEIGHTS, FIT, true>;
    static std::atomic<uint64_t> done{0};
    cudaError_t e = once_per_device(done, [&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemSm - 4096); });
    if (e != cudaSuccess) return e;
    const int stage_words = (a.P / W + parts - 1) / parts, stage_bytes = room_of(stage_words * W, sizeof(T));
    const int stages = std::min(kMostStages, ring_bytes(resident) / stage_bytes);
    if (stages < 2) return cudaErrorInvalidConfiguration;                // the edges of a row are stored while the one before is read
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(std::min(a.N, kSms * resident / parts) * parts));
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = (size_t)stages * stage_bytes;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)parts;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = OWNER == kCluster ? 1 : 0;
    if constexpr (OWNER == kCluster) {
        static std::atomic<uint64_t> allowed{0};
        static std::atomic<int> clusters[kMostParts + 1][1024 / 32 + 1];
        int at_once = 0;
        if (parts > 8) e = once_per_device(allowed, [&] { return allow_large_clusters(kernel); });
        if (e == cudaSuccess) e = active_clusters(clusters[parts][threads / 32], kernel, cfg, at_once);
        if (e != cudaSuccess) return e;
        cfg.gridDim = dim3((unsigned)(std::min(a.N, at_once) * parts));
    }
    count_launch();
    return cudaLaunchKernelEx(&cfg, kernel, a, parts, stages, stage_words);
}

template <class T>
cudaError_t launch_long(const Forward& a, cudaStream_t stream) {
    long_rows_kernel<T><<<(unsigned)a.N, kLongThreads, 0, stream>>>(a);
    count_launch();
    return cudaGetLastError();
}

template <class T, int W>
cudaError_t launch_words(const Forward& a, cudaStream_t stream) {
    if (a.P > 1 << 20) return launch_long<T>(a, stream);            // more than any cluster's registers hold; sums of sizes below fit into 32 bits
    const int words = a.P / W;
    // Short rows: as few lanes of a warp as hold the row in up to 16 values each (up to 20 in 16 lanes, 32 in 32), since half of a warp's work
    // would else be the sums' shuffles: 100,003 rows of 257 binary16 values take 27 us with 16 lanes; with 32 they took 3 more.
    constexpr int kMost = W == 1 ? 16 : 32 / W, kFew = 16 / W, kMiddle = W == 1 ? 20 : 16 / W;
    if (words <= 8 * kFew)
        return with_int<1, kFew>((words + 7) / 8, [&](auto nv) { return launch<T, W, nv.value, kWarp, kHold, kLast, 8>(a, 256, 1, stream); });
    if (words <= 16 * kMiddle)
        return with_int<kFew / 2 + 1, kMiddle>((words + 15) / 16, [&](auto nv) { return launch<T, W, nv.value, kWarp, kHold, kLast, 16>(a, 256, 1, stream); });
    if (words <= 32 * kMost)
        return with_int<kMiddle / 2 + 1, kMost>((words + 31) / 32, [&](auto nv) {
            return launch<T, W, nv.value, kWarp, nv.value * W <= 16 ? kHold : kAsk, kLast>(a, 256, 1, stream);
        });
    // Enough rows, or none of whose words is of 16 bytes: gamma and beta stay in registers, in a block where they fit, else in a cluster
    // (677 x 20,000 20 us so and 25 with blocks that load them for every row; 8,000 x 2,001 27 us so and 56).  Two thirds of the odd lengths from 513 to
    // 4,095 have threads that miss more than their last word (kAny) and gain nothing so: 8,736 x 2,049 53 us.
    constexpr int kHeld = held_values(W) / W, kThreads = hold_threads(kBlock, held_values(W)), kPartThreads = hold_threads(kCluster, held_values(W));
    constexpr int kAtOnce = W == 1 ? 768 : 512;                      // threads of an SM, by the registers they are given
    constexpr bool kWide = W * sizeof(T) == 16;                      // every row begins and ends on a 16-byte border
    const int held = round32((words + kHeld - 1) / kHeld);
    // few rows of narrow words: one for a block or a cluster, whose threads load four values each at once (100 x 1,001 3.0 us; by bulk copies 6.4)
    if constexpr (!kWide) {
        int parts = 1;
        while (parts < kMostParts && (words > parts * 4096 / W || ((int64_t)parts * a.N <= kSms && a.P >= parts * 2048))) parts *= 2;
        const int part = (words + parts - 1) / parts;
        if (part <= 4096 / W && (int64_t)a.N * parts <= 2 * kSms) {
            constexpr int NV = 4 / W;
            const int threads = round32((part + NV - 1) / NV);
            return parts > 1 ? launch<T, W, NV, kCluster, kHold, kAny>(a, threads, parts, stream) : launch<T, W, NV, kBlock, kHold, kAny>(a, threads, 1, stream);
        }
    }
    if (held <= kThreads && (!kWide || a.N > 8 * kSms)) {
        const int resident = std::min(kAtOnce / held, 8);
        const bool most = (kHeld - 1) * held <= words;
        if constexpr (kWide) if (words == kHeld * held) return launch_ring<T, W, kHeld, kBlock, kHold, kFull>(a, held, 1, resident, stream);
        return most ? launch_ring<T, W, kHeld, kBlock, kHold, kWide ? kLast : kEnd>(a, held, 1, resident, stream)
                    : launch_ring<T, W, kHeld, kBlock, kHold, kAny>(a, held, 1, resident, stream);
    }
    const int blocks = std::max(2, (words + kHeld * kPartThreads - 1) / (kHeld * kPartThreads));
    if (held > kThreads && blocks <= kMostParts && (!kWide || (int64_t)a.N * blocks >= 2 * kSms)) {
        const int most = (words + blocks - 1) / blocks, fewest = words / blocks, threads = round32((most + kHeld - 1) / kHeld);
        const int resident = std::min((W == 1 ? 640 : 512) / threads, 4);
        const bool last_only = (kHeld - 1) * threads <= fewest;
        return last_only ? launch_ring<T, W, kHeld, kCluster, kHold, kWide ? kLast : kEnd>(a, threads, blocks, resident, stream)
                         : launch_ring<T, W, kHeld, kCluster, kHold, kAny>(a, threads, blocks, resident, stream);
    }
    if constexpr (!kWide) {
        return launch_long<T>(a, stream);
    } else {
        // few rows: every thread reads its part of a row at once
        constexpr int kBlockWords = W == 8 ? 3 : 5;                 // of a thread
        int parts = 1;
        while (parts < kMostParts && (words > parts * 1024 * kBlockWords || ((int64_t)parts * a.N <= kSms && a.P >= parts * 2048))) parts *= 2;
        const int part = (words + parts - 1) / parts, least = words / parts;      // words of the blocks
        if (part > 1024 * kBlockWords) return launch_long<T>(a, stream);
        int nv = (part + 1023) / 1024;
        while (nv < kBlockWords && (part + nv - 1) / nv > 256 && nv * W < 16) ++nv;
        while (nv > 1 && (nv - 1) * round32((part + nv - 1) / nv) > least) --nv;
        return with_int<1, kBlockWords>(nv, [&](auto n) {
            const int threads = round32((part + n.value - 1) / n.value);
            auto with = [&](auto w) {
                constexpr Weights WEIGHTS = decltype(w)::value;
                return parts > 1 ? launch<T, W, n.value, kCluster, WEIGHTS, kLast>(a, threads, parts, stream) : launch<T, W, n.value, kBlock, WEIGHTS, kLast>(a, threads, 1, stream);
            };
            const bool both = a.gamma && a.beta;
            if (both && a.w_type == ROCKET_F32) return with(std::integral_constant<Weights, kAsFloat>());
            if constexpr (sizeof(T) == 2) if (both && a.w_type == a.x_type) return with(std::integral_constant<Weights, kAsInput>());
            return with(std::integral_constant<Weights, kAsk>());
        });
    }
}

// The kernels of one type of x.
template <class T>
cudaError_t launch_rows(const Forward& a, cudaStream_t stream) {
    auto fits = [&](int W) {
        return a.P % W == 0 && packs(a.x, a.x_type, a.N > 1 ? a.x_stride : 0, W) && packs(a.y, a.y_type, a.N > 1 ? a.y_stride : 0, W) &&
               packs(a.gamma, a.w_type, 0, W) && packs(a.beta, a.w_type, 0, W);
    };
    if constexpr (sizeof(T) == 2) if (a.y_type != ROCKET_F32 && fits(8)) return launch_words<T, 8>(a, stream);
    if (fits(4)) return launch_words<T, 4>(a, stream);
    return launch_words<T, 1>(a, stream);
}

extern template cudaError_t launch_rows<float>(const Forward&, cudaStream_t);
extern template cudaError_t launch_rows<__half>(const Forward&, cudaStream_t);
extern template cudaError_t launch_rows<__nv_bfloat16>(const Forward&, cudaStream_t);

}  // namespace norm
}  // namespace rocket
