// Layer norm backward: xh = (x - m) r, u = dy g, dx = r (u - mean(u) - xh mean(u xh)), dg = sum_n dy xh, db = sum_n dy.
//
// Bound: memory.  x and dy are read once.  A thread keeps its columns for all rows that its owner (a warp, a block, or the blocks
// of a cluster, by the length of a row) goes through: gamma and the sums of dg and db over those rows stay in registers, xh and u between
// a row's reduction and its dx.  The owners' sums go to the workspace, [owner][2][P], and a second kernel adds them up in the
// owners' order, which depends on the sizes alone: the same call gives the same bits.
//
// Rows on 16-byte borders come into shared memory by bulk copies, several rows ahead (a warp's rows, which are short, and rows of
// any other alignment are loaded by the threads).  Every wait is bounded; a thread that gives up counts as NaN, which makes the row's dx
// and the thread's sums NaN.
#include "rocket_fast_dev.cuh"
#include "rocket_float_types.cuh"
#include "rocket_internal.h"
#include "rocket_norm.h"
#include "rocket_norm_sums.cuh"

namespace rocket {
namespace norm {
namespace {

constexpr int kColumns = 16;              // of a thread
constexpr int kThreads = 256;             // most of a block; 128 registers each, so that 512 threads share an SM
constexpr int kMostStages = 8;
constexpr int kWarpColumns = 32 * kColumns;
constexpr int kSmemSm = 227 * 1024;       // shared memory of an SM

bool is_short(int P) { return P <= kWarpColumns; }
int parts_of(int P) { return (P + kThreads * kColumns - 1) / (kThreads * kColumns); }
// Columns of a block: a multiple of 8, which keeps every part of a row on a 16-byte border.
int part_of(int P) { const int parts = parts_of(P); return ((P + parts - 1) / parts + 7) / 8 * 8; }
int threads_of(int P) { return round32((part_of(P) + kColumns - 1) / kColumns); }
int resident_of(int P) { return is_short(P) ? 2 : std::min(512 / threads_of(P), 16); }
bool is_long(int P) { return parts_of(P) > kMostParts; }

// Owners whose sums go to the workspace (a block of warps adds its own up first).
int owners_of(int N, int P) {
    if (is_long(P)) return 0;
    if (N <= (is_short(P) ? 64 : 2)) return 1;           // no second launch: an owner by itself writes the gradients
    const int rows = is_short(P) ? kThreads / 32 : 1;
    return std::max(1, (int)std::min<int64_t>(((int64_t)N + rows - 1) / rows, (int64_t)kSms * resident_of(P) / (is_short(P) ? 1 : parts_of(P))));
}

// Sums of two values over the threads that own a row, the same bits in each.  Each half of a warp goes on with one of the values, which saves
// nearly half of the shuffles.  Two sets of buffers, taken in turn, make one barrier a row enough.
template <Owner OWNER>
__device__ __forceinline__ float2 row_sums(float2 v, int turn) {
    const int lane = threadIdx.x & 31;
    const bool upper = lane >= 16;
    float s = (upper ? v.y : v.x) + __shfl_xor_sync(0xffffffffu, upper ? v.x : v.y, 16);
    s = add_lanes(s, 8);
    if constexpr (OWNER != kWarp) {
        __shared__ float sets[2][2][kThreads / 32];
        auto& red = sets[turn & 1];
        const int warps = blockDim.x >> 5, l = lane & 15;
        if (l == 0) red[lane >> 4][threadIdx.x >> 5] = s;
        __syncthreads();
        s = add_lanes(l < warps ? red[lane >> 4][l & (kThreads / 32 - 1)] : 0.0f, 4);
    }
    return make_float2(__shfl_sync(0xffffffffu, s, 0), __shfl_sync(0xffffffffu, s, 16));
}

// One row's work of a thread: xh and u from x and dy, the sums over the row, the sums over the rows.
template <int W>
__device__ __forceinline__ void take(const float (&x)[W], const float (&dy)[W], const float (&g)[W], float m, float r, float (&xh)[W], float (&u)[W],
                                     float (&dg)[W], float (&db)[W], float2& s) {
#pragma unroll
    for (int j = 0; j < W; ++j) {
        xh[j] = (x[j] - m) * r;
        u[j] = dy[j] * g[j];
        s.x += u[j];
        s.y = fmaf(u[j], xh[j], s.y);
        dg[j] = fmaf(dy[j], xh[j], dg[j]);
        db[j] += dy[j];
    }
}

template <class TX, class TY, int W, int NV>
__global__ void __launch_bounds__(kThreads) warp_rows_kernel(const Backward a) {
    extern __shared__ float sums[];       // [2][P]
    const int lane = threadIdx.x & 31, words = a.P / W;
    const bool last = lane + 32 * (NV - 1) < words;
    auto has = [&](int k) { return k < NV - 1 || last; };
    float g[NV][W], dg[NV][W] = {}, db[NV][W] = {};
    Packed<TX, W> next_x[NV];
    Packed<TY, W> next_y[NV];
    float next_m = 0.0f, next_r = 0.0f;
    auto fetch = [&](int64_t n) {
        const TX* __restrict__ x = static_cast<const TX*>(a.x) + n * a.x_stride + lane * W;
        const TY* __restrict__ dy = static_cast<const TY*>(a.dy) + n * a.dy_stride + lane * W;
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (has(k)) {
                next_x[k] = load_packed_once<TX, W>(x + 32 * k * W);
                next_y[k] = load_packed_once<TY, W>(dy + 32 * k * W);
            }
        next_m = __ldg(a.mean + n);
        next_r = __ldg(a.rstd + n);
    };
    const int64_t rows = (int64_t)gridDim.x * (kThreads / 32);
    int64_t row = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    if (row < a.N) fetch(row);
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int j = 0; j < W; ++j) g[k][j] = 1.0f;
    if (a.gamma)
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (has(k)) load_typed<W>(a.gamma, a.w_type, (lane + 32 * k) * W, g[k]);
    const float over_p = 1.0f / (float)a.P;
    for (; row < a.N; row += rows) {
        float xh[NV][W], u[NV][W];
        float2 s = make_float2(0.0f, 0.0f);
        const float m = next_m, r = next_r;
        Packed<TX, W> cx[NV];
        Packed<TY, W> cy[NV];
#pragma unroll
        for (int k = 0; k < NV; ++k) { cx[k] = next_x[k]; cy[k] = next_y[k]; }
        if (row + rows < a.N) fetch(row + rows);
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (has(k)) {
                float x[W], dy[W];
                unpack<TX, W>(cx[k], x);
                unpack<TY, W>(cy[k], dy);
                take<W>(x, dy, g[k], m, r, xh[k], u[k], dg[k], db[k], s);
            }
        s = row_sums<kWarp>(s, 0);
        if (a.dx) {
            const float c1 = s.x * over_p * r, c2 = s.y * over_p * r;
            TX* __restrict__ dx = static_cast<TX*>(a.dx) + row * a.dx_stride + lane * W;
#pragma unroll
            for (int k = 0; k < NV; ++k)
                if (has(k)) {
                    float o[W];
#pragma unroll
                    for (int j = 0; j < W; ++j) o[j] = fmaf(u[k][j], r, -fmaf(xh[k][j], c2, c1));
                    store_packed<TX, W>(dx + 32 * k * W, o);
                }
        }
    }
    asm volatile("griddepcontrol.launch_dependents;");      // the kernel that adds up the sums waits for this one's end
    if (!a.dgamma && !a.dbeta) return;
    // the warps add their sums in turn
    for (int w = 0; w < kThreads / 32; ++w) {
        if ((int)(threadIdx.x >> 5) == w) {
#pragma unroll
            for (int k = 0; k < NV; ++k)
                if (has(k))
#pragma unroll
                    for (int j = 0; j < W; ++j) {
                        const int p = (lane + 32 * k) * W + j;
                        sums[p] = w == 0 ? dg[k][j] : sums[p] + dg[k][j];
                        sums[a.P + p] = w == 0 ? db[k][j] : sums[a.P + p] + db[k][j];
                    }
        }
        __syncthreads();
    }
    if (gridDim.x == 1) {
        for (int i = threadIdx.x; i < a.P; i += kThreads) {
            if (a.dgamma) store_typed<1>(a.dgamma, a.w_type, i, {sums[i]});
            if (a.dbeta) store_typed<1>(a.dbeta, a.w_type, i, {sums[a.P + i]});
        }
        return;
    }
    float* out = a.partial + (int64_t)blockIdx.x * 2 * a.P;
    for (int i = threadIdx.x; i < 2 * a.P; i += kThreads) out[i] = sums[i];
}

// RING: the rows come by bulk copies, as many ahead as there are stages; else the threads load them.  FIT: which words of a thread are within the
// row needs asking for none of them (2), for its last one (1), for all of them (0).
template <class TX, class TY, int W, int NV, bool RING, Owner OWNER, int FIT>
__global__ void __launch_bounds__(kThreads, 2) block_rows_kernel(const Backward a, int parts, int part, int stages) {
    extern __shared__ __align__(16) unsigned char ring[];
    __shared__ __align__(8) uint64_t arrived[kMostStages];
    __shared__ Exchange exchange;
    const int rank = OWNER == kCluster ? blockIdx.x % parts : 0, owner = blockIdx.x / parts, owners = gridDim.x / parts;
    const int beg = rank * part, columns = min(part, a.P - beg), words = columns / W, first = threadIdx.x, step = blockDim.x;
    const bool last = first + (NV - 1) * step < words;
    auto has = [&](int k) { return FIT == 2 || (FIT == 1 ? k < NV - 1 || last : first + k * step < words); };
    const uint32_t bars = fast::smem_u32(arrived), rings = fast::smem_u32(ring);
    const int x_bytes = part * (int)sizeof(TX), stage_bytes = x_bytes + part * (int)sizeof(TY);
    const TX* x_from = static_cast<const TX*>(a.x) + beg;
    const TY* y_from = static_cast<const TY*>(a.dy) + beg;
    // a copy's size is a multiple of 16 bytes: the words behind the last such one are loaded by their threads
    const int x_whole = columns * (int)sizeof(TX) / 16 * 16, y_whole = columns * (int)sizeof(TY) / 16 * 16;
    auto copied = [&](int k, int end_bytes, int whole) { return FIT == 2 || (FIT == 1 && k < NV - 1) || end_bytes <= whole; };
    int64_t to_copy = owner;
    auto copy = [&](int stage) {
        const uint32_t bar = bars + 8u * stage, dst = rings + (uint32_t)(stage * stage_bytes);
        fast::mbar_arrive_expect_tx(bar, (uint32_t)(x_whole + y_whole));
        if (x_whole) fast::bulk_g2s(dst, x_from + to_copy * a.x_stride, (uint32_t)x_whole, bar);
        if (y_whole) fast::bulk_g2s(dst + (uint32_t)x_bytes, y_from + to_copy * a.dy_stride, (uint32_t)y_whole, bar);
        to_copy += owners;
    };
    if (RING && threadIdx.x == 0) {
        for (int s = 0; s < stages; ++s) fast::mbar_init(bars + 8u * s, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        for (int s = 0; s < stages && to_copy < a.N; ++s) copy(s);
    }
    float g[NV][W], dg[NV][W] = {}, db[NV][W] = {};
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int j = 0; j < W; ++j) g[k][j] = 1.0f;
    if (a.gamma)
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (has(k)) load_typed<W>(a.gamma, a.w_type, beg + (first + k * step) * W, g[k]);
    // nobody waits on a barrier, or writes to another block's shared memory, before it is there
    if constexpr (OWNER == kCluster) {
        exchange.init();
        asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    } else {
        __syncthreads();
    }
    const float over_p = 1.0f / (float)a.P;
    int stage = 0, turn = 0;
    uint32_t parity = 0;
    bool ok = true;
    float m = 0.0f, r = 0.0f;
    if (owner < a.N) { m = __ldg(a.mean + owner); r = __ldg(a.rstd + owner); }
    for (int64_t row = owner; row < a.N; row += owners, ++turn) {
        float xh[NV][W], u[NV][W];
        float next_m = 0.0f, next_r = 0.0f;
        if (row + owners < a.N) { next_m = __ldg(a.mean + row + owners); next_r = __ldg(a.rstd + row + owners); }
        const TX* xs = x_from + row * a.x_stride;
        const TY* ys = y_from + row * a.dy_stride;
        if constexpr (RING) {
            ok = ok && wait_soon(bars + 8u * stage, parity);
        }
        float2 s = make_float2(ok ? 0.0f : __int_as_float(0x7fc00000), 0.0f);
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (has(k)) {
                const int i = (first + k * step) * W;
                float x[W], dy[W];
                if constexpr (RING) {
                    const unsigned char* in = ring + (size_t)stage * stage_bytes;
                    if (copied(k, (i + W) * (int)sizeof(TX), x_whole)) unpack<TX, W>(load_packed<TX, W>(reinterpret_cast<const TX*>(in) + i), x);
                    else unpack<TX, W>(load_packed_ro<TX, W>(xs + i), x);
                    if (copied(k, (i + W) * (int)sizeof(TY), y_whole)) unpack<TY, W>(load_packed<TY, W>(reinterpret_cast<const TY*>(in + x_bytes) + i), dy);
                    else unpack<TY, W>(load_packed_ro<TY, W>(ys + i), dy);
                } else {
                    unpack<TX, W>(load_packed_once<TX, W>(xs + i), x);
                    unpack<TY, W>(load_packed_once<TY, W>(ys + i), dy);
                }
                take<W>(x, dy, g[k], m, r, xh[k], u[k], dg[k], db[k], s);
            }
        if (!ok) dg[0][0] = db[0][0] = s.x;
        // behind the reduction's first barrier everybody has read the row: the next one may come into its place
        s = row_sums<OWNER>(s, turn);
        if constexpr (RING) {
            if (threadIdx.x == 0 && ok && to_copy < a.N) copy(stage);
            if (++stage == stages) { stage = 0; parity ^= 1u; }
        }
        if constexpr (OWNER == kCluster) {
            const float2* all = exchange.swap(s, parts, rank, turn, ok);
            s = all[0];
            for (int p = 1; p < parts; ++p) { s.x += all[p].x; s.y += all[p].y; }
            if (!ok) s.x = __int_as_float(0x7fc00000);
        }
        if (a.dx) {
            const float c1 = s.x * over_p * r, c2 = s.y * over_p * r;
            TX* __restrict__ dx = static_cast<TX*>(a.dx) + row * a.dx_stride + beg;
#pragma unroll
            for (int k = 0; k < NV; ++k)
                if (has(k)) {
                    float o[W];
#pragma unroll
                    for (int j = 0; j < W; ++j) o[j] = fmaf(u[k][j], r, -fmaf(xh[k][j], c2, c1));
                    store_packed<TX, W>(dx + (first + k * step) * W, o);
                }
        }
        m = next_m;
        r = next_r;
    }
    // copies that a wait gave up on must not outlive the block
    if (RING && threadIdx.x == 0 && !ok)
        for (int s = 0; s < stages; ++s) {
            fast::mbar_wait(bars + 8u * stage, parity);
            if (++stage == stages) { stage = 0; parity ^= 1u; }
        }
    if constexpr (OWNER == kCluster) leave_cluster();
    asm volatile("griddepcontrol.launch_dependents;");
    if (!a.dgamma && !a.dbeta) return;
    if (owners == 1) {
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (has(k)) {
                if (a.dgamma) store_typed<W>(a.dgamma, a.w_type, beg + (first + k * step) * W, dg[k]);
                if (a.dbeta) store_typed<W>(a.dbeta, a.w_type, beg + (first + k * step) * W, db[k]);
            }
        return;
    }
    float* out = a.partial + (int64_t)owner * 2 * a.P + beg;
#pragma unroll
    for (int k = 0; k < NV; ++k)
        if (has(k))
#pragma unroll
            for (int j = 0; j < W; ++j) {
                const int p = (first + k * step) * W + j;
                out[p] = dg[k][j];
                out[a.P + p] = db[k][j];
            }
}

// dg and db from the owners' sums: a lane has C columns, a block 32 C, its warps share the owners.
template <int C, int WARPS>
__global__ void __launch_bounds__(WARPS * 32) sum_owners_kernel(const float* __restrict__ partial, int owners, int P, void* dgamma, void* dbeta, int w_type) {
    __shared__ float red[2][WARPS][32 * C];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t p = ((int64_t)blockIdx.x * 32 + lane) * C;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    float s[C] = {}, q[C] = {};
    if (p < P)
#pragma unroll 4
        for (int o = warp; o < owners; o += WARPS) {
            const float* from = partial + (int64_t)o * 2 * P + p;
            const Packed<float, C> a = load_packed<float, C>(from), b = load_packed<float, C>(from + P);
            float x[C];
            unpack<float, C>(a, x);
#pragma unroll
            for (int j = 0; j < C; ++j) q[j] += x[j];
            unpack<float, C>(b, x);
#pragma unroll
            for (int j = 0; j < C; ++j) s[j] += x[j];
        }
#pragma unroll
    for (int j = 0; j < C; ++j) {
        red[0][warp][lane * C + j] = q[j];
        red[1][warp][lane * C + j] = s[j];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * 32 * C; i += WARPS * 32) {
        const int which = i / (32 * C), c = i % (32 * C);
        const int64_t column = (int64_t)blockIdx.x * 32 * C + c;
        void* out = which == 0 ? dgamma : dbeta;
        if (!out || column >= P) continue;
        float v[1] = {0.0f};
#pragma unroll
        for (int w = 0; w < WARPS; ++w) v[0] += red[which][w][c];
        store_typed<1>(out, w_type, column, v);
    }
}

// ---- rows longer than a cluster's registers: a block per row, then a block per 32 columns, sums in double precision ------------------

constexpr int kLongThreads = 256, kLongWarps = kLongThreads / 32;

template <class TX, class TY>
__global__ void __launch_bounds__(kLongThreads) long_rows_kernel(const Backward a) {
    __shared__ double2 red[kLongWarps];
    auto weight = [&](int64_t i) {
        float w[1] = {1.0f};
        if (a.gamma) load_typed<1>(a.gamma, a.w_type, i, w);
        return w[0];
    };
    for (int64_t n = blockIdx.x; n < a.N; n += gridDim.x) {
        const TX* __restrict__ x = static_cast<const TX*>(a.x) + n * a.x_stride;
        const TY* __restrict__ dy = static_cast<const TY*>(a.dy) + n * a.dy_stride;
        const float m = a.mean[n], r = a.rstd[n];
        double2 s = make_double2(0.0, 0.0);
        for (int64_t i = threadIdx.x; i < a.P; i += kLongThreads) {
            const float u = to_float(dy[i]) * weight(i), xh = (to_float(x[i]) - m) * r;
            s.x += (double)u;
            s.y += (double)u * (double)xh;
        }
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
        for (int w = 0; w < kLongWarps; ++w) { s.x += red[w].x; s.y += red[w].y; }
        const float c1 = (float)(s.x / (double)a.P), c2 = (float)(s.y / (double)a.P);
        TX* __restrict__ dx = static_cast<TX*>(a.dx) + n * a.dx_stride;
        for (int64_t i = threadIdx.x; i < a.P; i += kLongThreads) {
            const float u = to_float(dy[i]) * weight(i), xh = (to_float(x[i]) - m) * r;
            dx[i] = from_float<TX>(r * (u - c1 - xh * c2));
        }
    }
}

template <class TX, class TY>
__global__ void __launch_bounds__(kLongThreads) long_weights_kernel(const Backward a) {
    __shared__ double red[2][kLongWarps][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t p = (int64_t)blockIdx.x * 32 + lane;
    double s = 0.0, q = 0.0;
    if (p < a.P)
        for (int64_t n = warp; n < a.N; n += kLongWarps) {
            const float d = to_float(static_cast<const TY*>(a.dy)[n * a.dy_stride + p]);
            const float xh = (to_float(static_cast<const TX*>(a.x)[n * a.x_stride + p]) - a.mean[n]) * a.rstd[n];
            s += (double)d;
            q += (double)d * (double)xh;
        }
    red[0][warp][lane] = q;
    red[1][warp][lane] = s;
    __syncthreads();
    if (warp < 2 && p < a.P) {
        s = 0.0;
#pragma unroll
        for (int w = 0; w < kLongWarps; ++w) s += red[warp][w][lane];
        const float v[1] = {(float)s};
        void* out = warp == 0 ? a.dgamma : a.dbeta;
        if (out) store_typed<1>(out, a.w_type, p, v);
    }
}

// ---- launches ---------------------------------------------------------------------------------------------------------------------------

template <class TX, class TY, int W>
cudaError_t launch_short(const Backward& a, cudaStream_t stream) {
    return with_int<1, kColumns / W>((a.P / W + 31) / 32, [&](auto nv) {
        warp_rows_kernel<TX, TY, W, nv.value><<<owners_of(a.N, a.P), kThreads, 2 * a.P * sizeof(float), stream>>>(a);
        count_launch();
        return cudaGetLastError();
    });
}

// owners: of at most so many, how many there are is put here.
template <class TX, class TY, int W, int NV, bool RING, Owner OWNER, int FIT>
cudaError_t launch_owners(const Backward& a, int& owners, cudaStream_t stream) {
    const int parts = parts_of(a.P), part = part_of(a.P), threads = threads_of(a.P);
    auto kernel = block_rows_kernel<TX, TY, W, NV, RING, OWNER, FIT>;
    int stages = 0, bytes = 0;
    if (RING) {
        static std::atomic<uint64_t> done{0};
        const cudaError_t e = once_per_device(done, [&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemSm - 4096); });
        if (e != cudaSuccess) return e;
        const int stage = part * (int)(sizeof(TX) + sizeof(TY));
        stages = std::min(kMostStages, (kSmemSm / resident_of(a.P) - 2048) / stage);      // 2 KB: the block's other arrays, and what the driver keeps
        bytes = stages * stage;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(owners * parts));
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = (size_t)bytes;
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
        static std::atomic<int> known[kMostParts + 1][kThreads / 32 + 1];
        int most = 0;
        cudaError_t e = parts > 8 ? once_per_device(allowed, [&] { return allow_large_clusters(kernel); }) : cudaSuccess;
        if (e == cudaSuccess) e = active_clusters(known[parts][threads / 32], kernel, cfg, most);
        if (e != cudaSuccess) return e;
        owners = std::min(owners, most);
        cfg.gridDim = dim3((unsigned)(owners * parts));
    }
    count_launch();
    return cudaLaunchKernelEx(&cfg, kernel, a, parts, part, stages);
}

template <class TX, class TY, int W, int NV, bool RING>
cudaError_t launch_blocks(const Backward& a, int& owners, cudaStream_t stream) {
    const int parts = parts_of(a.P), part = part_of(a.P), least = a.P - (parts - 1) * part, threads = threads_of(a.P);      // least: the last block's columns
    auto with_fit = [&](auto fit) {
        constexpr int FIT = decltype(fit)::value;
        return parts > 1 ? launch_owners<TX, TY, W, NV, RING, kCluster, FIT>(a, owners, stream) : launch_owners<TX, TY, W, NV, RING, kBlock, FIT>(a, owners, stream);
    };
    if constexpr (RING) {
        const bool whole = least * (int)sizeof(TX) % 16 == 0 && least * (int)sizeof(TY) % 16 == 0;
        if (least == NV * W * threads && part == least && whole) return with_fit(Int<2>());
        if (least >= (NV - 1) * W * threads + (whole ? 0 : W)) return with_fit(Int<1>());
    }
    return with_fit(Int<0>());
}

template <class TX, class TY>
cudaError_t launch_long(const Backward& a, cudaStream_t stream) {
    cudaError_t e = cudaSuccess;
    if (a.dx && a.N > 0) {
        long_rows_kernel<TX, TY><<<std::min(a.N, kSms * 8), kLongThreads, 0, stream>>>(a);
        count_launch();
        e = cudaGetLastError();
    }
    if (e == cudaSuccess && (a.dgamma || a.dbeta)) {
        long_weights_kernel<TX, TY><<<(unsigned)(((int64_t)a.P + 31) / 32), kLongThreads, 0, stream>>>(a);
        count_launch();
        e = cudaGetLastError();
    }
    return e;
}

}  // namespace

int64_t backward_workspace(int N, int P) {
    const int owners = owners_of(N, P);
    return owners > 1 ? (int64_t)owners * 2 * P * (int64_t)sizeof(float) : 0;
}

cudaError_t launch_backward(const Backward& a, cudaStream_t stream) {
    if (a.N == 0 && !a.dgamma && !a.dbeta) return cudaSuccess;
    auto fits = [&](int W) {
        return a.P % W == 0 && packs(a.x, a.x_type, a.N > 1 ? a.x_stride : 0, W) && packs(a.dy, a.y_type, a.N > 1 ? a.dy_stride : 0, W) &&
               packs(a.dx, a.x_type, a.dx && a.N > 1 ? a.dx_stride : 0, W) && packs(a.gamma, a.w_type, 0, W) && packs(a.dgamma, a.w_type, 0, W) && packs(a.dbeta, a.w_type, 0, W);
    };
    // bulk copies begin on 16-byte borders
    const bool ring = packs(a.x, ROCKET_F32, 0, 4) && packs(a.dy, ROCKET_F32, 0, 4) &&
                      (a.N <= 1 || (packs(nullptr, a.x_type, a.x_stride, 16 / float_type_bytes(a.x_type)) && packs(nullptr, a.y_type, a.dy_stride, 16 / float_type_bytes(a.y_type))));
    int owners = owners_of(a.N, a.P);
    const cudaError_t e = with_float_type(a.x_type, [&](auto* px) {
        return with_float_type(a.y_type, [&](auto* py) {
            using TX = std::remove_pointer_t<decltype(px)>;
            using TY = std::remove_pointer_t<decltype(py)>;
            if (is_long(a.P)) return launch_long<TX, TY>(a, stream);
            if (is_short(a.P)) {
                if constexpr (sizeof(TX) == 2 && sizeof(TY) == 2) if (fits(8)) return launch_short<TX, TY, 8>(a, stream);
                return fits(4) ? launch_short<TX, TY, 4>(a, stream) : launch_short<TX, TY, 1>(a, stream);
            }
            if constexpr (sizeof(TX) == 2 && sizeof(TY) == 2) if (ring && fits(8)) return launch_blocks<TX, TY, 8, kColumns / 8, true>(a, owners, stream);
            if (ring && fits(4)) return launch_blocks<TX, TY, 4, kColumns / 4, true>(a, owners, stream);
            return launch_blocks<TX, TY, 1, kColumns, false>(a, owners, stream);
        });
    });
    if (e != cudaSuccess || owners <= 1 || (!a.dgamma && !a.dbeta)) return e;
    auto sum = [&](auto kernel, int columns, int warps) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)((a.P + columns - 1) / columns));
        cfg.blockDim = dim3((unsigned)(warps * 32));
        cfg.stream = stream;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        count_launch();
        return cudaLaunchKernelEx(&cfg, kernel, (const float*)a.partial, owners, a.P, a.dgamma, a.dbeta, a.w_type);
    };
    // Long rows fill the SMs with four columns a lane, and with as many warps as there are owners to share.
    if (a.P % 4 == 0 && a.P >= 8192) return owners > 64 ? sum(sum_owners_kernel<4, 16>, 128, 16) : sum(sum_owners_kernel<4, 8>, 128, 8);
    return sum(sum_owners_kernel<1, 32>, 32, 32);
}

}  // namespace norm
}  // namespace rocket
