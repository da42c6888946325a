// The 2-norm of a gradient held in many tensors, and clipping by it: the step between the backward passes and the optimiser.
//
//   n = sqrt(sum over tensors and values of g^2)    c = min(1, max_norm / (n + 1e-6))    out = c g
//
// Squares and sums are kept in double precision: fp32 gradients of 1e-20 and 1e20 both have squares outside fp32.  The sums'
// order depends on sizes, types and alignments alone.
//
// Bound: memory.  Two kernels: the first leaves a sum per block, every block of the second adds those up for itself and scales.  Every
// block has a contiguous share of the tensors, taken as one long line, the same in both kernels.  Tensors may begin anywhere; a
// share's piece of one is taken in words of 16 bytes between its first and its last such border.
//
// Measured: the norm of 302 M bf16 values in 384 tensors 102 us, 5.9 TB/s or 92 % of a copy, of 302 M fp32 184 us, 6.6 TB/s (338 where each load asked
// whether it is within the tensor); 42.6 M binary16 values in 96 tensors clipped to fp32 72 us (341 MB with the second reading: 4.7 TB/s).
#include <cooperative_groups.h>

#include <algorithm>
#include <cmath>
#include <new>
#include <utility>
#include <vector>

#include "rocket_float_types.cuh"
#include "rocket_internal.h"
#include "rocket_norm_sums.cuh"

namespace rocket {
namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 256;
constexpr int kBlocks = 148 * 4;         // most blocks, and partial sums, of one launch
constexpr int kFewTensors = 64;          // of one launch: the table travels in its arguments, of which a short one is there sooner
constexpr int kTensors = 800;
constexpr int kPiece = 1 << 24;          // values of one tensor at a time, counted in 32 bits
constexpr int kLeast = 1024;             // values that a block is started for
// Values that one cluster deals with in one launch, without a workspace: 390,000 fp32 values are clipped in 9.4 us of device time so and in 6.8 by two
// kernels, whose second launch and workspace cost the caller 4.7 us; 22,000 take 6.2 and, by a cluster of eight, 7.2.
constexpr int kSmall = 512 * 1024;
constexpr int kSmallBlocks = 16, kSmallThreads = 512;

template <int N>
struct Table {
    const void* g[N];
    void* out[N];
    int64_t first[N + 1];                // values of the tensors before this one: all of them as one long line
    uint8_t g_type[N], out_type[N];
    int tensors;
};

template <int THREADS>
__device__ __forceinline__ double block_sum(double a) {
    constexpr int kWarps = THREADS / 32;
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

// The tensor that a value of the line belongs to.
template <int N>
__device__ __forceinline__ int tensor_of(const Table<N>& t, int64_t value) {
    int lo = 0, hi = t.tensors;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (t.first[mid] <= value) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Calls f(tensor, position in it, how many) for the pieces of this block's share of the line, a contiguous one.  Shares begin at multiples of
// 64 values, on 16-byte borders where the tensors begin and end on such.
template <int N, class F>
__device__ __forceinline__ void for_share(const Table<N>& t, int block, int blocks, F&& f) {
    const int64_t total = t.first[t.tensors], units = (total + 63) / 64;
    int64_t at = units * block / blocks * 64;
    const int64_t end = min(units * (block + 1) / blocks * 64, total);
    if (at >= end) return;
    for (int k = tensor_of(t, at); at < end; ++k) {
        const int64_t beg = t.first[k], stop = min(end, t.first[k + 1]);
        for (; at < stop; at += kPiece) f(k, at - beg, (int)min((int64_t)kPiece, stop - at));
        at = stop;
    }
}

// How p[0 .. n) falls into single values, words of W values on borders of a word, and single values again.
template <class T, int W>
struct Split {
    int head, words;
    __device__ __forceinline__ Split(const T* p, int n) {
        constexpr int kWord = W * (int)sizeof(T);
        head = min(n, (int)((kWord - (int)(reinterpret_cast<uintptr_t>(p) & (kWord - 1))) & (kWord - 1)) / (int)sizeof(T));
        words = (n - head) / W;
    }
    // The single value of this thread, or n.
    __device__ __forceinline__ int single(int n) const {
        const int t = (int)threadIdx.x;
        return t < head ? t : min(n, head + words * W + (t - head));
    }
};

// Calls f(word, number) for every word of this thread; the loads of U words are under way at a time.
template <int THREADS, int U, class T, int W, class F>
__device__ __forceinline__ void for_words(const T* body, int words, F&& f) {
    int i = (int)threadIdx.x;
    for (; i + (U - 1) * THREADS < words; i += U * THREADS) {
        Packed<T, W> v[U];
#pragma unroll
        for (int k = 0; k < U; ++k) v[k] = load_packed<T, W>(body + (int64_t)(i + k * THREADS) * W);
#pragma unroll
        for (int k = 0; k < U; ++k) f(v[k], i + k * THREADS);
    }
    for (; i < words; i += THREADS) f(load_packed<T, W>(body + (int64_t)i * W), i);
}

template <int THREADS, class T>
__device__ __noinline__ double sum_squares(const T* p, int n) {
    constexpr int W = 16 / (int)sizeof(T);
    const Split<T, W> split(p, n);
    double s[4] = {};
    for_words<THREADS, 4, T, W>(p + split.head, split.words, [&](const Packed<T, W>& v, int) {
        float x[W];
        unpack<T, W>(v, x);
#pragma unroll
        for (int j = 0; j < W; ++j) s[j & 3] = fma((double)x[j], (double)x[j], s[j & 3]);
    });
    const int at = split.single(n);
    if (at < n) s[0] = fma((double)to_float(p[at]), (double)to_float(p[at]), s[0]);
    return (s[0] + s[1]) + (s[2] + s[3]);
}

// Sum of squares of the block's share.
template <int THREADS, int N>
__device__ __forceinline__ double squares(const Table<N>& t, int block, int blocks) {
    double s = 0.0;
    for_share(t, block, blocks, [&](int k, int64_t beg, int n) {
        s += t.g_type[k] == ROCKET_F32 ? sum_squares<THREADS>(static_cast<const float*>(t.g[k]) + beg, n)
             : t.g_type[k] == ROCKET_F16 ? sum_squares<THREADS>(static_cast<const __half*>(t.g[k]) + beg, n)
                                         : sum_squares<THREADS>(static_cast<const __nv_bfloat16*>(t.g[k]) + beg, n);
    });
    return block_sum<THREADS>(s);
}

__device__ __forceinline__ float factor(float norm, float max_norm) {
    const float q = max_norm / (norm + 1e-6f);
    return q > 1.0f ? 1.0f : q;          // a NaN stays one
}

// Words of 16 bytes of the wider of the two types, so that a warp's loads and stores are both of one piece.  Not inlined: the registers would
// be asked for once for every pair of types.
template <int THREADS, class TG, class TO>
__device__ __noinline__ void scale_piece(const TG* g, TO* to, int n, float c) {
    constexpr int W = 16 / (int)(sizeof(TO) > sizeof(TG) ? sizeof(TO) : sizeof(TG)), U = 64 / (W * (int)sizeof(TG));
    const Split<TG, W> split(g, n);
    TO* body = to + split.head;
    auto scaled = [&](const Packed<TG, W>& v, float (&o)[W]) {
        unpack<TG, W>(v, o);
#pragma unroll
        for (int j = 0; j < W; ++j) o[j] *= c;
    };
    if (reinterpret_cast<uintptr_t>(body) % Packed<TO, W>::kWord == 0) {
        for_words<THREADS, U, TG, W>(g + split.head, split.words, [&](const Packed<TG, W>& v, int i) {
            float o[W];
            scaled(v, o);
            store_packed<TO, W>(body + (int64_t)i * W, o);
        });
    } else {
        for_words<THREADS, U, TG, W>(g + split.head, split.words, [&](const Packed<TG, W>& v, int i) {
            float o[W];
            scaled(v, o);
#pragma unroll
            for (int j = 0; j < W; ++j) body[(int64_t)i * W + j] = from_float<TO>(o[j]);
        });
    }
    const int at = split.single(n);
    if (at < n) to[at] = from_float<TO>(to_float(g[at]) * c);
}

template <int THREADS, class TG, int N>
__device__ __forceinline__ void scale_tensor(const Table<N>& t, int k, int64_t beg, int n, float c) {
    const TG* g = static_cast<const TG*>(t.g[k]) + beg;
    if constexpr (sizeof(TG) == 2)
        if (t.out_type[k] != ROCKET_F32) return scale_piece<THREADS>(g, static_cast<TG*>(t.out[k]) + beg, n, c);
    scale_piece<THREADS>(g, static_cast<float*>(t.out[k]) + beg, n, c);
}

template <int THREADS, int N>
__device__ __forceinline__ void scale(const Table<N>& t, int block, int blocks, float c) {
    for_share(t, block, blocks, [&](int k, int64_t beg, int n) {
        if (t.g_type[k] == ROCKET_F32) scale_tensor<THREADS, float>(t, k, beg, n, c);
        else if (t.g_type[k] == ROCKET_F16) scale_tensor<THREADS, __half>(t, k, beg, n, c);
        else scale_tensor<THREADS, __nv_bfloat16>(t, k, beg, n, c);
    });
}

template <int N>
__global__ void __launch_bounds__(kThreads, 4) squares_kernel(const __grid_constant__ Table<N> t, double* __restrict__ part) {
    const double sum = squares<kThreads>(t, blockIdx.x, gridDim.x);
    if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

__device__ __forceinline__ float norm_of(const double* __restrict__ part, int n) {
    double s = 0.0;
    for (int i = threadIdx.x; i < n; i += kThreads) s += part[i];
    return (float)sqrt(block_sum<kThreads>(s));
}

__global__ void __launch_bounds__(kThreads) norm_kernel(const double* __restrict__ part, int parts, float* __restrict__ norm) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const float n = norm_of(part, parts);
    if (threadIdx.x == 0) *norm = n;
}

// in_place: every output is its own gradient, and a gradient that is not clipped stays as it is.
template <int N>
__global__ void __launch_bounds__(kThreads, 4) scale_kernel(const __grid_constant__ Table<N> t, const double* __restrict__ part, int parts,
                                                            float* __restrict__ norm, float max_norm, bool in_place) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const float n = norm_of(part, parts), c = factor(n, max_norm);
    if (blockIdx.x == 0 && threadIdx.x == 0) *norm = n;
    if (!(in_place && c == 1.0f)) scale<kThreads>(t, blockIdx.x, gridDim.x, c);
}

// Both in one launch for a small gradient, by the blocks of one cluster, whose sums meet in distributed shared memory; nothing is
// written before the barrier behind which all of them have read everything.
__global__ void __launch_bounds__(kSmallThreads) small_kernel(const __grid_constant__ Table<kFewTensors> t, float* __restrict__ norm, float max_norm, bool clip,
                                                              bool in_place) {
    __shared__ double share[kSmallBlocks];
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = (int)cluster.block_rank();
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");       // nobody writes to a block that does not run yet
    const double sum = squares<kSmallThreads>(t, rank, kSmallBlocks);
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (threadIdx.x < kSmallBlocks) *cluster.map_shared_rank(&share[rank], threadIdx.x) = sum;
    cluster.sync();
    double s = share[0];
#pragma unroll
    for (int i = 1; i < kSmallBlocks; ++i) s += share[i];
    const float n = (float)sqrt(s), c = factor(n, max_norm);
    if (rank == 0 && threadIdx.x == 0) *norm = n;
    if (clip && !(in_place && c == 1.0f)) scale<kSmallThreads>(t, rank, kSmallBlocks, c);
}

int status_of(cudaError_t e) {
    if (e == cudaSuccess) return ROCKET_OK;
    cudaGetLastError();
    return e == cudaErrorMemoryAllocation ? ROCKET_ENOMEM : ROCKET_ECUDA;
}

using Span = std::pair<uintptr_t, uintptr_t>;

void sort_spans(std::vector<Span>& s) {
    if (!std::is_sorted(s.begin(), s.end())) std::sort(s.begin(), s.end());
}

// Whether one cluster deals with all of it, in one launch and without a workspace.
bool is_small(int count, int64_t total) { return count <= kFewTensors && total <= kSmall; }

// Of valid sizes.
int64_t workspace_bytes_for(int count, int64_t total) {
    return is_small(count, total) ? 0 : (int64_t)sizeof(double) * kBlocks * std::max<int64_t>(1, (count + (int64_t)kTensors - 1) / kTensors);
}

// All values, or -1 for a size out of range.
int64_t total_of(int count, const int64_t* sizes) {
    int64_t total = 0;
    for (int i = 0; i < count; ++i) {
        if (sizes[i] < 0 || sizes[i] > (int64_t(1) << 40)) return -1;
        total = std::min(total + sizes[i], int64_t(1) << 60);
    }
    return total;
}

// The arguments of both entry points; clip: whether gradients are written, to `out` or, where it is NULL, in place.
int check(int count, const void* const* grads, const int64_t* sizes, const int32_t* types, bool clip, void* const* out, const int32_t* out_types,
          const float* norm, const void* workspace, int64_t workspace_bytes) {
    if (count < 0 || !norm || (reinterpret_cast<uintptr_t>(norm) & 3u)) return ROCKET_EINVAL;
    if (count > 0 && (!grads || !sizes || !types || (out && !out_types))) return ROCKET_EINVAL;
    const int64_t total = total_of(count, sizes), need = workspace_bytes_for(count, total);
    if (total < 0 || workspace_bytes < need || (need > 0 && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 15u)))) return ROCKET_EINVAL;
    const uintptr_t ws = need > 0 ? (uintptr_t)workspace : 0;
    const Span own[] = {{(uintptr_t)norm, (uintptr_t)norm + 4}, {ws, ws + (uintptr_t)need}};
    auto meets = [](const Span& a, const Span& b) { return a.first < b.second && b.first < a.second; };
    if (meets(own[0], own[1])) return ROCKET_EINVAL;
    std::vector<Span> written, read;
    if (clip) written.reserve((size_t)count);
    if (out) read.reserve((size_t)count);
    for (int i = 0; i < count; ++i) {
        if (!is_float_type(types[i])) return ROCKET_EINVAL;
        if (out && (!is_float_type(out_types[i]) || (out_types[i] != types[i] && out_types[i] != ROCKET_F32))) return ROCKET_EINVAL;
        if (sizes[i] == 0) continue;
        const uintptr_t g = (uintptr_t)grads[i], o = out ? (uintptr_t)out[i] : g;
        const unsigned gb = (unsigned)float_type_bytes(types[i]), ob = out ? (unsigned)float_type_bytes(out_types[i]) : gb;
        if (!g || !o || (g & (gb - 1)) || (o & (ob - 1))) return ROCKET_EINVAL;
        const Span from = {g, g + (uintptr_t)sizes[i] * gb}, to = {o, o + (uintptr_t)sizes[i] * ob};
        if (meets(from, own[0]) || meets(from, own[1])) return ROCKET_EINVAL;
        if (!clip) continue;
        if (meets(to, own[0]) || meets(to, own[1])) return ROCKET_EINVAL;
        written.push_back(to);
        if (o != g || ob != gb) read.push_back(from);
    }
    if (total > (int64_t(1) << 46)) return ROCKET_EUNSUPPORTED;
    // what is written overlaps nothing; what is read may overlap itself (one tensor under two names counts twice)
    sort_spans(written);
    for (size_t i = 1; i < written.size(); ++i) if (written[i].first < written[i - 1].second) return ROCKET_EINVAL;
    sort_spans(read);
    size_t w = 0;
    for (const Span& r : read) {
        while (w < written.size() && written[w].second <= r.first) ++w;
        if (w < written.size() && written[w].first < r.second) return ROCKET_EINVAL;
    }
    return ROCKET_OK;
}

struct Call {
    int count;
    const void* const* grads;
    const int64_t* sizes;
    const int32_t* types;
    void* const* out;                    // nullptr: in place
    const int32_t* out_types;
};

template <int N>
void fill(Table<N>& t, const Call& c, int beg, int end) {
    t.tensors = 0;
    t.first[0] = 0;
    for (int i = beg; i < end; ++i) {
        if (c.sizes[i] == 0) continue;
        const int k = t.tensors++;
        t.g[k] = c.grads[i];
        t.out[k] = c.out ? c.out[i] : const_cast<void*>(c.grads[i]);
        t.g_type[k] = (uint8_t)c.types[i];
        t.out_type[k] = (uint8_t)(c.out ? c.out_types[i] : c.types[i]);
        t.first[k + 1] = t.first[k] + c.sizes[i];
    }
}

// A kernel that begins before its predecessor has ended, and waits for it by griddepcontrol.wait.
template <class... A, class... B>
cudaError_t launch_behind(void (*kernel)(A...), int blocks, cudaStream_t stream, B&&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(kThreads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    count_launch();
    return cudaLaunchKernelEx(&cfg, kernel, std::forward<B>(args)...);
}

template <int N>
cudaError_t run(const Call& c, bool clip, float max_norm, float* norm, double* part, cudaStream_t stream) {
    Table<N> t;
    int parts = 0;
    auto blocks_of = [&] { return (int)std::min<int64_t>((t.first[t.tensors] + kLeast - 1) / kLeast, kBlocks); };
    if constexpr (N == kFewTensors)
        if (is_small(c.count, total_of(c.count, c.sizes))) {
            fill(t, c, 0, c.count);
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3(kSmallBlocks);
            cfg.blockDim = dim3(kSmallThreads);
            cfg.stream = stream;
            cudaLaunchAttribute attr[1];
            attr[0].id = cudaLaunchAttributeClusterDimension;
            attr[0].val.clusterDim.x = kSmallBlocks;
            attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
            cfg.attrs = attr;
            cfg.numAttrs = 1;
            static std::atomic<uint64_t> allowed{0};
            const cudaError_t e = norm::once_per_device(allowed, [] { return norm::allow_large_clusters(small_kernel); });
            if (e != cudaSuccess) return e;
            count_launch();
            return cudaLaunchKernelEx(&cfg, small_kernel, t, norm, max_norm, clip, c.out == nullptr);
        }
    for (int beg = 0; beg < c.count; beg += N) {
        fill(t, c, beg, std::min(c.count, beg + N));
        const int blocks = blocks_of();
        if (!blocks) continue;
        squares_kernel<N><<<blocks, kThreads, 0, stream>>>(t, part + parts);
        count_launch();
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
        parts += blocks;
    }
    if (!clip || parts == 0) return launch_behind(norm_kernel, 1, stream, (const double*)part, parts, norm);
    for (int beg = (c.count - 1) / N * N; beg >= 0; beg -= N) {
        if (c.count > N) fill(t, c, beg, std::min(c.count, beg + N));
        const int blocks = blocks_of();
        if (!blocks) continue;
        const cudaError_t e = launch_behind(scale_kernel<N>, blocks, stream, t, (const double*)part, parts, norm, max_norm, c.out == nullptr);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

int call(const Call& c, bool clip, float max_norm, float* norm, void* workspace, int64_t workspace_bytes, void* cuda_stream) {
    try {
        const int st = check(c.count, c.grads, c.sizes, c.types, clip, c.out, c.out_types, norm, workspace, workspace_bytes);
        if (st != ROCKET_OK) return st;
    } catch (const std::bad_alloc&) {
        return ROCKET_ENOMEM;
    }
    auto* part = static_cast<double*>(workspace);
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    return status_of(c.count <= kFewTensors ? run<kFewTensors>(c, clip, max_norm, norm, part, stream) : run<kTensors>(c, clip, max_norm, norm, part, stream));
}

}  // namespace
}  // namespace rocket

using namespace rocket;

extern "C" int64_t rocket_grad_norm_workspace(int count, const int64_t* sizes) {
    if (count < 0 || (count > 0 && !sizes)) return ROCKET_EINVAL;
    const int64_t total = total_of(count, sizes);
    return total < 0 ? ROCKET_EINVAL : workspace_bytes_for(count, total);
}

extern "C" int rocket_grad_norm(int count, const void* const* grads_dev, const int64_t* sizes, const int32_t* types, float* norm_dev,
                                void* workspace_dev, int64_t workspace_bytes, void* cuda_stream) {
    return call({count, grads_dev, sizes, types, nullptr, nullptr}, false, 0.0f, norm_dev, workspace_dev, workspace_bytes, cuda_stream);
}

extern "C" int rocket_clip_grad_norm(int count, const void* const* grads_dev, const int64_t* sizes, const int32_t* types,
                                     void* const* out_dev, const int32_t* out_types, float max_norm, float* norm_dev,
                                     void* workspace_dev, int64_t workspace_bytes, void* cuda_stream) {
    if (!(max_norm >= 0.0f)) return ROCKET_EINVAL;
    return call({count, grads_dev, sizes, types, out_dev, out_types}, true, max_norm, norm_dev, workspace_dev, workspace_bytes, cuda_stream);
}
