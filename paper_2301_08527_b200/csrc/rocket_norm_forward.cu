// Layer norm forward: m = mean(x), v = mean((x - m)^2), r = 1 / sqrt(v + eps), y = (x - m) r g + b for every row.
//
// Bound: memory.  A row is read once and stays in registers between its two reductions, while its owner's next row is on its
// way.  The sums are fp32 and safe at any scale.  The first gives a shift next to the mean, the second is of d = x - shift; what
// is left of the mean, mean(d), comes off the variance and off every value.  For 16-bit rows the shift is rounded to their type,
// so that d is exact and a constant row gives 0; for fp32 rows the first sum is taken of x - x[0], to the same end.
//
// Who has a row: a warp where it is short, a block, or the blocks of a cluster where rows are few or longer than a block's
// registers (each block sums its contiguous part, the sums meet in distributed shared memory).  The owners stay and go through
// the rows in turn.
#include <algorithm>

#include "rocket_float_types.cuh"
#include "rocket_internal.h"
#include "rocket_norm.h"
#include "rocket_norm_sums.cuh"

namespace rocket {
namespace norm {
namespace {

// W values per word, NV words per thread.  HOLD: a thread's values of gamma and beta stay in registers.
template <class T, int W, int NV, Owner OWNER, bool HOLD>
__global__ void __launch_bounds__(OWNER == kWarp || HOLD ? 256 : 1024)
rows_kernel(const Forward a, int parts, int half, float unit) {
    int64_t row, rows;
    int beg = 0, words = (a.P + W - 1) / W, first, step, rank = 0;
    if constexpr (OWNER == kWarp) {
        row = (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
        rows = (int64_t)gridDim.x * (blockDim.x >> 5);
        first = threadIdx.x & 31;
        step = 32;
    } else {
        row = blockIdx.x / parts;
        rows = gridDim.x / parts;
        if constexpr (OWNER == kCluster) {
            rank = blockIdx.x % parts;
            const int all = words, from = (int)((int64_t)all * rank / parts);
            beg = from * W;
            words = (int)((int64_t)all * (rank + 1) / parts) - from;
            cg::this_cluster().sync();             // nobody writes to another block's shared memory before that block runs
        }
        first = threadIdx.x;
        step = blockDim.x;
    }
    const int mine = (words - first + step - 1) / step;    // words of this thread: NV, or fewer (a warp's: NV or NV - 1)
    const int64_t at = beg + (int64_t)first * W;
    auto has = [&](int k) { return (OWNER == kWarp && k < NV - 1) || k < mine; };
    Packed<T, W> next[NV] = {};                            // words beyond the row's end stay zeros
    float next0 = 0.0f;
    auto fetch = [&](int64_t n) {
        const T* __restrict__ x = static_cast<const T*>(a.x) + n * a.x_stride;
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (has(k)) next[k] = load_packed_once<T, W>(x + at + (int64_t)k * step * W);
        if constexpr (sizeof(T) == 4) next0 = to_float(x[0]);
    };
    float g[HOLD ? NV : 1][W], b[HOLD ? NV : 1][W];
    auto weights = [&](int k, float (&gk)[W], float (&bk)[W]) {
#pragma unroll
        for (int j = 0; j < W; ++j) { gk[j] = 1.0f; bk[j] = 0.0f; }
        if (a.gamma) load_typed<W>(a.gamma, a.w_type, at + (int64_t)k * step * W, gk);
        if (a.beta) load_typed<W>(a.beta, a.w_type, at + (int64_t)k * step * W, bk);
    };
    if (row < a.N) fetch(row);
    if constexpr (HOLD)
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (has(k)) weights(k, g[k], b[k]);
    const float over_p = 1.0f / (float)a.P;
    for (; row < a.N; row += rows) {
        float f[NV][W];
        const float x0 = next0;
#pragma unroll
        for (int k = 0; k < NV; ++k) unpack<T, W>(next[k], f[k]);
        if (row + rows < a.N) fetch(row + rows);
        // unit: a power of two of at most 1 / P, so that no sum overflows
        float s1 = 0.0f;
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (sizeof(T) == 2 || has(k))
#pragma unroll
                for (int j = 0; j < W; ++j) s1 = fmaf(sizeof(T) == 4 ? f[k][j] - x0 : f[k][j], unit, s1);
        s1 = row_sum<OWNER>(s1, parts, rank, half);
        const float shift = to_float(from_float<T>(x0 + s1 * (over_p / unit)));
        float2 s2 = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (has(k))
#pragma unroll
                for (int j = 0; j < W; ++j) {
                    f[k][j] -= shift;
                    s2.x += f[k][j];
                    s2.y = fmaf(f[k][j], f[k][j], s2.y);
                }
        s2 = row_sums<OWNER>(s2, parts, rank, 0);
        const float rest = s2.x * over_p;
        const float v = fmaf(-rest, rest, s2.y * over_p), r = rsqrtf((v < 0.0f ? 0.0f : v) + a.eps);      // a NaN stays one
        const float off = -rest * r;
        const int64_t out = row * a.y_stride + at;
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (has(k)) {
                float o[W];
                if constexpr (HOLD) {
#pragma unroll
                    for (int j = 0; j < W; ++j) o[j] = fmaf(fmaf(f[k][j], r, off), g[k][j], b[k][j]);
                } else {
                    weights(k, g[0], b[0]);
#pragma unroll
                    for (int j = 0; j < W; ++j) o[j] = fmaf(fmaf(f[k][j], r, off), g[0][j], b[0][j]);
                }
                store_typed<W>(a.y, a.y_type, out + (int64_t)k * step * W, o);
            }
        if (first == 0 && rank == 0) {
            if (a.mean) a.mean[row] = shift + rest;
            if (a.rstd) a.rstd[row] = r;
        }
    }
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

// Sum's scale: the largest power of two that is at most 1 / P.
float unit_of(int P) {
    int bits = 0;
    while ((int64_t(1) << bits) < P) ++bits;
    return ldexpf(1.0f, -bits);
}
template <class T, int W, int NV, Owner OWNER, bool HOLD>
cudaError_t launch(const Forward& a, int threads, int parts, cudaStream_t stream) {
    auto kernel = rows_kernel<T, W, NV, OWNER, HOLD>;
    static std::atomic<int> known[1024 / 32 + 1];                        // resident blocks of an SM, by warps; all devices are alike
    int resident = known[threads / 32].load(std::memory_order_relaxed);
    if (resident == 0) {
        const cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&resident, kernel, threads, 0);
        if (e != cudaSuccess) return e;
        known[threads / 32].store(resident, std::memory_order_relaxed);
    }
    const int64_t owners = OWNER == kWarp ? threads / 32 : 1;            // rows of a block
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
        static std::atomic<int> clusters[kMostParts + 1][1024 / 32 + 1];
        int at_once = 0;
        const cudaError_t e = active_clusters(clusters[parts][threads / 32], kernel, cfg, at_once);
        if (e != cudaSuccess) return e;
        cfg.gridDim = dim3((unsigned)std::min<int64_t>(blocks, (int64_t)at_once * parts));
    }
    count_launch();
    return cudaLaunchKernelEx(&cfg, kernel, a, parts, half_of(threads), unit_of(a.P));
}

template <class T, int W>
cudaError_t launch_words(const Forward& a, cudaStream_t stream) {
    const int words = (a.P + W - 1) / W;
    constexpr int kWarpWords = W == 1 ? 16 : 32 / W;                // of a lane: rows of up to 512 values, 1,024 in wider words
    if (words <= 32 * kWarpWords)
        return with_int<1, kWarpWords>((words + 31) / 32, [&](auto nv) {
            return launch<T, W, nv.value, kWarp, nv.value * W <= 16>(a, 256, 1, stream);
        });
    constexpr int kBlockWords = W == 1 ? 16 : W == 8 ? 3 : 5;       // of a thread
    int parts = 1;
    while (parts < kMostParts && (words > parts * 1024 * kBlockWords || ((int64_t)parts * a.N <= kSms && a.P >= parts * 2048))) parts *= 2;
    const int part = (words + parts - 1) / parts;
    if (part > 1024 * kBlockWords) {
        long_rows_kernel<T><<<(unsigned)a.N, kLongThreads, 0, stream>>>(a);
        count_launch();
        return cudaGetLastError();
    }
    int nv = (part + 1023) / 1024;
    while (nv < kBlockWords && (part + nv - 1) / nv > 256 && nv * W < 16) ++nv;
    return with_int<1, kBlockWords>(nv, [&](auto n) {
        const int threads = round32((part + n.value - 1) / n.value);
        if constexpr (n.value * W <= 16) if (parts == 1 && threads <= 256 && a.N > 8 * kSms) return launch<T, W, n.value, kBlock, true>(a, threads, 1, stream);
        return parts > 1 ? launch<T, W, n.value, kCluster, false>(a, threads, parts, stream)
                         : launch<T, W, n.value, kBlock, false>(a, threads, 1, stream);
    });
}

}  // namespace

cudaError_t launch_forward(const Forward& a, cudaStream_t stream) {
    return with_float_type(a.x_type, [&](auto* tx) {
        using T = std::remove_pointer_t<decltype(tx)>;
        auto fits = [&](int W) {
            return a.P % W == 0 && packs(a.x, a.x_type, a.N > 1 ? a.x_stride : 0, W) && packs(a.y, a.y_type, a.N > 1 ? a.y_stride : 0, W) &&
                   packs(a.gamma, a.w_type, 0, W) && packs(a.beta, a.w_type, 0, W);
        };
        if constexpr (sizeof(T) == 2) if (fits(8)) return launch_words<T, 8>(a, stream);
        if (fits(4)) return launch_words<T, 4>(a, stream);
        return launch_words<T, 1>(a, stream);
    });
}

}  // namespace norm
}  // namespace rocket
