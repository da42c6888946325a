// Layer norm backward: xh = (x - m) r, u = dy g, dx = r (u - mean(u) - xh mean(u xh)), dg = sum_n dy xh, db = sum_n dy.
//
// Bound: memory.  x and dy are read once.  A thread keeps its columns for all rows that its owner (a warp, a block, or the blocks
// of a cluster, by the length of a row) goes through: gamma and the sums of dg and db over those rows stay in registers, xh and u between
// a row's reduction and its dx.  The owners' sums go to the workspace, [owner][2][P], and a second kernel adds them up in the
// owners' order: the same call gives the same bits.
//
// A block's rows come into shared memory by bulk copies, several rows ahead (a warp's, which are short, are loaded by its lanes).
// Every wait is bounded; a thread that gives up counts as NaN, which makes the row's dx and the thread's sums NaN.
//
// Measured with the second kernel: 16,384 x 4,096 bf16 79 us, 5.1 TB/s or 79 % of a copy (1,135 with a pass per output); 677 x 9,996 fp32 and bf16
// 28 us (43 with more clusters than run at once, 31 with a cluster barrier per row); 8,000 x 2,001 fp32 41 us, where loads by the threads took 150.
#pragma once

#include "rocket_fast_dev.cuh"
#include "rocket_float_types.cuh"
#include "rocket_internal.h"
#include "rocket_norm.h"
#include "rocket_norm_sums.cuh"

namespace rocket {
namespace norm {

constexpr int kColumns = 16;              // of a thread
// Most of a block.  Rows of blocks and clusters: 128 registers each, so that 512 threads share an SM.  Short rows: as many as they ask for, up to 184;
// above 128 an SM has one block of the two that the grid counts on, and the grid runs in two rounds.  Cut to 128, 100,000 x 256 fp32 takes 68 us for
// 59 and 100,000 x 255 bf16 154 for 57 (60,000 x 512 fp32 64 for 70).
constexpr int kThreads = 256;
constexpr int kMostStages = 8;
constexpr int kWarpColumns = 32 * kColumns;
constexpr int kSmemSm = 227 * 1024;       // shared memory of an SM

inline bool is_short(int P) { return P <= kWarpColumns; }
// Lanes of a short row: the fewest, since half of a warp's work would else be the sums' shuffles.
inline int lanes_of(int P) { return P <= 8 * kColumns ? 8 : P <= 16 * kColumns ? 16 : 32; }
// Blocks of a row: one or two more than the columns ask for where that gives all threads all words but the last (narrow words, of an odd P, are the harder to
// divide).
inline int parts_of(int P) {
    if (P > kMostParts * kThreads * kColumns) return kMostParts + 1;
    const int fewest = (P + kThreads * kColumns - 1) / (kThreads * kColumns);
    if (fewest == 1) return 1;
    for (int parts = fewest; parts < fewest + 3 && parts <= kMostParts; ++parts) {
        const int part = ((P + parts - 1) / parts + 7) / 8 * 8, threads = round32((part + kColumns - 1) / kColumns);
        if (P - (parts - 1) * part >= (P % 4 ? kColumns - 1 : kColumns - 4) * threads) return parts;
    }
    return fewest;
}
// Columns of a block: a multiple of 8, which keeps every part of a row on a 16-byte border.
inline int part_of(int P) { const int parts = parts_of(P); return ((P + parts - 1) / parts + 7) / 8 * 8; }
inline int threads_of(int P) { return round32((part_of(P) + kColumns - 1) / kColumns); }
inline int resident_of(int P) { return is_short(P) ? 2 : std::min(512 / threads_of(P), 16); }
inline bool is_long(int P) { return parts_of(P) > kMostParts; }

// Rows that a block has at a time.
inline int block_rows(int P) { return is_short(P) ? kThreads / lanes_of(P) : 1; }
// Few rows: the blocks of one cluster are all owners, and add their sums up in distributed shared memory: no workspace, and no second launch.
// Up to so many turns of each.  A call costs 15 us so and 19 with a second kernel, its launch and its workspace, at every length; the device's own time,
// which counts in captured graphs, is 4.8 us so and 3.9 by a second kernel for 32 x 1,000 fp32, 8.6 and 4.1 for 128 x 1,000, 10.9 and 6.8 for
// 128 x 4,096, 8.7 and 4.8 for 4,096 x 128, and 14 and 5.3 at most (128 x 1,001).
constexpr int kJoinedTurns = 8;
inline bool is_joined(int N, int P) { return parts_of(P) == 1 && N <= (int64_t)kMostParts * block_rows(P) * kJoinedTurns; }

// Owners of rows (a block of warps adds its own sums up first).  weights: whether dgamma or dbeta is wanted; dx alone has nothing to join, and no
// reason to stay on the blocks of one cluster (128 x 1,001: 3.6 us of device time, 12.3 on 16 blocks).
inline int owners_of(int N, int P, bool weights) {
    if (is_long(P)) return 0;
    if (parts_of(P) > 1 && N <= 2) return 1;             // a cluster by itself writes the gradients
    const int64_t want = ((int64_t)N + block_rows(P) - 1) / block_rows(P);
    const int64_t most = weights && is_joined(N, P) ? kMostParts : kSms * resident_of(P) / (is_short(P) ? 1 : parts_of(P));
    return (int)std::max<int64_t>(1, std::min(want, most));
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

// dg and db from the sums [2][P] that every block of a cluster has in shared memory: each block adds up a share of the columns, in the blocks' order, in
// double precision.
__device__ __forceinline__ void join_owners(const float* sums, const Backward& a) {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    const int blocks = gridDim.x;
    for (int i = blockIdx.x * blockDim.x + threadIdx.x; i < 2 * a.P; i += blocks * blockDim.x) {
        void* out = i < a.P ? a.dgamma : a.dbeta;
        if (!out) continue;
        double sum = 0.0;
        for (int b = 0; b < blocks; ++b) {
            uint32_t from;
            float x;
            asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(from) : "r"(fast::smem_u32(sums + i)), "r"(b));
            asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x) : "r"(from) : "memory");
            sum += (double)x;
        }
        const float v[1] = {(float)sum};
        store_typed<1>(out, a.w_type, i < a.P ? i : i - a.P, v);
    }
    // no block ends while another still reads its sums: the arrival stands behind the reads
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
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

// LANES of a warp share a row; a warp has 32 / LANES rows at a time, and its lanes for the same columns meet at the end.
template <class TX, class TY, int W, int NV, int LANES>
__global__ void __launch_bounds__(kThreads) warp_rows_kernel(const Backward a) {
    extern __shared__ float sums[];       // of every warp, [2][P]
    const int lane = threadIdx.x & (LANES - 1), ahead = (threadIdx.x & 31) / LANES, words = a.P / W;
    const bool last = lane + LANES * (NV - 1) < words;
    auto has = [&](int k) { return k < NV - 1 || last; };
    float g[NV][W], dg[NV][W] = {}, db[NV][W] = {};
    Packed<TX, W> next_x[NV];
    Packed<TY, W> next_y[NV];
    float next_m = 0.0f, next_r = 0.0f;
    auto fetch = [&](int64_t n) {
        n += ahead;
        if (n >= a.N) return;
        const TX* __restrict__ x = static_cast<const TX*>(a.x) + n * a.x_stride + lane * W;
        const TY* __restrict__ dy = static_cast<const TY*>(a.dy) + n * a.dy_stride + lane * W;
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (has(k)) {
                next_x[k] = load_packed_once<TX, W>(x + LANES * k * W);
                next_y[k] = load_packed_once<TY, W>(dy + LANES * k * W);
            }
        next_m = __ldg(a.mean + n);
        next_r = __ldg(a.rstd + n);
    };
    const int64_t rows = (int64_t)gridDim.x * (kThreads / LANES);
    int64_t row = (int64_t)blockIdx.x * (kThreads / LANES) + (threadIdx.x >> 5) * (32 / LANES);      // the warp's first
    if (row < a.N) fetch(row);
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int j = 0; j < W; ++j) g[k][j] = 1.0f;
    if (a.gamma)
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (has(k)) load_typed<W>(a.gamma, a.w_type, (lane + LANES * k) * W, g[k]);
    const float over_p = 1.0f / (float)a.P;
    for (; row < a.N; row += rows) {
        float xh[NV][W], u[NV][W];
        float2 s = make_float2(0.0f, 0.0f);
        const float m = next_m, r = next_r;
        const bool mine = LANES == 32 || row + ahead < a.N;
        Packed<TX, W> cx[NV];
        Packed<TY, W> cy[NV];
#pragma unroll
        for (int k = 0; k < NV; ++k) { cx[k] = next_x[k]; cy[k] = next_y[k]; }
        if (row + rows < a.N) fetch(row + rows);
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (has(k) && mine) {
                float x[W], dy[W];
                unpack<TX, W>(cx[k], x);
                unpack<TY, W>(cy[k], dy);
                take<W>(x, dy, g[k], m, r, xh[k], u[k], dg[k], db[k], s);
            }
        s = LANES == 32 ? row_sums<kWarp>(s, 0) : make_float2(add_lanes(s.x, LANES / 2), add_lanes(s.y, LANES / 2));
        if (a.dx && mine) {
            const float c1 = s.x * over_p * r, c2 = s.y * over_p * r;
            TX* __restrict__ dx = static_cast<TX*>(a.dx) + (row + ahead) * a.dx_stride + lane * W;
#pragma unroll
            for (int k = 0; k < NV; ++k)
                if (has(k)) {
                    float o[W];
#pragma unroll
                    for (int j = 0; j < W; ++j) o[j] = fmaf(u[k][j], r, -fmaf(xh[k][j], c2, c1));
                    store_packed<TX, W>(dx + LANES * k * W, o);
                }
        }
    }
    asm volatile("griddepcontrol.launch_dependents;");      // the kernel that adds up the sums waits for this one's end
    if (!a.dgamma && !a.dbeta) return;
#pragma unroll
    for (int o = 16; o >= LANES; o /= 2)
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int j = 0; j < W; ++j) {
                dg[k][j] += __shfl_xor_sync(0xffffffffu, dg[k][j], o);
                db[k][j] += __shfl_xor_sync(0xffffffffu, db[k][j], o);
            }
    // every warp's sums, then those of the block in the first one's place
    float* own = sums + (threadIdx.x >> 5) * 2 * a.P;
#pragma unroll
    for (int k = 0; k < NV; ++k)
        if (has(k) && ahead == 0)
#pragma unroll
            for (int j = 0; j < W; ++j) {
                const int p = (lane + LANES * k) * W + j;
                own[p] = dg[k][j];
                own[a.P + p] = db[k][j];
            }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * a.P; i += kThreads) {
        float v = sums[i];
#pragma unroll
        for (int w = 1; w < kThreads / 32; ++w) v += sums[w * 2 * a.P + i];
        sums[i] = v;
    }
    if (a.joined) return join_owners(sums, a);
    float* out = a.partial + (int64_t)blockIdx.x * 2 * a.P;
    for (int i = threadIdx.x; i < 2 * a.P; i += kThreads) out[i] = sums[i];      // the thread's own
}

// A block's part of every row of its owner's; the rows come by bulk copies, as many ahead as there are stages.
template <class TX, class TY, int W, int NV, Owner OWNER, Fit FIT>
__global__ void __launch_bounds__(kThreads, 2) block_rows_kernel(const Backward a, int parts, int part, int stages) {
    extern __shared__ __align__(128) unsigned char ring[];
    __shared__ __align__(8) uint64_t arrived[kMostStages];
    __shared__ Exchange<float2> exchange;
    const int rank = OWNER == kCluster ? blockIdx.x % parts : 0, owner = blockIdx.x / parts, owners = gridDim.x / parts;
    const int beg = rank * part, columns = min(part, a.P - beg), words = columns / W, first = threadIdx.x, step = blockDim.x;
    const bool last = first + (NV - 1) * step < words;
    constexpr bool kEdges = FIT == kAny || FIT == kEnd;
    auto has = [&](int k) { return FIT == kFull || (FIT == kAny ? first + k * step < words : k < NV - 1 || last); };
    auto may_miss = [](int k) { return FIT == kAny || (FIT == kEnd && k == NV - 1); };
    const uint32_t bars = fast::smem_u32(arrived), rings = fast::smem_u32(ring);
    const int x_room = room_of(part, sizeof(TX)), stage_bytes = x_room + room_of(part, sizeof(TY));
    const TX* x_from = static_cast<const TX*>(a.x) + beg;
    const TY* y_from = static_cast<const TY*>(a.dy) + beg;
    const TX* x_next = x_from + owner * a.x_stride;                // the row to copy next
    const TY* y_next = y_from + owner * a.dy_stride;
    int64_t to_copy = owner;
    auto copy = [&](int stage) {
        const uint32_t bar = bars + 8u * stage, dst = rings + (uint32_t)(stage * stage_bytes);
        if constexpr (kEdges) {
            const Piece<TX> px(x_next, columns);
            const Piece<TY> py(y_next, columns);
            fast::mbar_arrive_expect_tx(bar, px.copied() + py.copied());
            px.copy(dst, x_next, bar);
            py.copy(dst + (uint32_t)x_room, y_next, bar);
        } else {
            const uint32_t x_bytes = (uint32_t)(columns * (int)sizeof(TX)), y_bytes = (uint32_t)(columns * (int)sizeof(TY));
            fast::mbar_arrive_expect_tx(bar, x_bytes + y_bytes);
            fast::bulk_g2s(dst, x_next, x_bytes, bar);
            fast::bulk_g2s(dst + (uint32_t)x_room, y_next, y_bytes, bar);
        }
        x_next += owners * a.x_stride;
        y_next += owners * a.dy_stride;
        to_copy += owners;
    };
    if (threadIdx.x == 0) {
        for (int s = 0; s < stages; ++s) fast::mbar_init(bars + 8u * s, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        for (int s = 0; s < stages && to_copy < a.N; ++s) copy(s);
    }
    // the values that no bulk copy brings: the first warp's lanes fetch them two rows ahead and store them one row ahead
    Edge<TX> x_edge;
    Edge<TY> y_edge;
    auto fetch_edges = [&](int64_t n) {
        x_edge.to = y_edge.to = -1;
        if (n >= a.N) return;
        if (threadIdx.x < 16) x_edge.fetch(x_from + n * a.x_stride, columns, threadIdx.x);
        else if (threadIdx.x < 32) y_edge.fetch(y_from + n * a.dy_stride, columns, threadIdx.x - 16);
    };
    auto put_edges = [&](int stage) {
        x_edge.put(ring + (size_t)stage * stage_bytes);
        y_edge.put(ring + (size_t)stage * stage_bytes + x_room);
    };
    if constexpr (kEdges) {
        fetch_edges(owner);
        put_edges(0);
        fetch_edges((int64_t)owner + owners);
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
    // Nobody waits on a barrier, or writes to another block's shared memory, before it is there, nor reads the first row before its edges are.  The
    // cluster's arrival is relaxed and orders no stores; one that releases cost 0.8 us a launch (32 x 20,000: 12.5 us for 11.7).
    if constexpr (OWNER == kCluster) {
        exchange.init();
        if constexpr (kEdges) __syncthreads();
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
        const unsigned char* in = ring + (size_t)stage * stage_bytes;
        const TX* xr = reinterpret_cast<const TX*>(in);
        const TY* yr = reinterpret_cast<const TY*>(in + x_room);
        if constexpr (kEdges) {
            xr = reinterpret_cast<const TX*>(in + (reinterpret_cast<uintptr_t>(x_from + row * a.x_stride) & 15));
            yr = reinterpret_cast<const TY*>(in + x_room + (reinterpret_cast<uintptr_t>(y_from + row * a.dy_stride) & 15));
            put_edges(stage + 1 == stages ? 0 : stage + 1);
            fetch_edges(row + 2 * (int64_t)owners);
        }
        ok = ok && wait_soon(bars + 8u * stage, parity);
        float2 s = make_float2(ok ? 0.0f : __int_as_float(0x7fc00000), 0.0f);
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (kEdges || has(k)) {
                const int i = (may_miss(k) ? min(first + k * step, words - 1) : first + k * step) * W;
                float x[W], dy[W];
                unpack<TX, W>(load_packed<TX, W>(xr + i), x);
                unpack<TY, W>(load_packed<TY, W>(yr + i), dy);
                if (may_miss(k) && !has(k))
#pragma unroll
                    for (int j = 0; j < W; ++j) { x[j] = m; dy[j] = 0.0f; }
                take<W>(x, dy, g[k], m, r, xh[k], u[k], dg[k], db[k], s);
            }
        // behind the reduction's first barrier everybody has read the row: the next one may come into its place
        s = row_sums<OWNER>(s, turn);
        if (threadIdx.x == 0 && ok && to_copy < a.N) {
            if constexpr (kEdges) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");      // behind the stores of the edges
            copy(stage);
        }
        if (++stage == stages) { stage = 0; parity ^= 1u; }
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
    if (!ok)
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int j = 0; j < W; ++j) dg[k][j] = db[k][j] = __int_as_float(0x7fc00000);
    // copies that a wait gave up on must not outlive the block
    if (threadIdx.x == 0 && !ok)
        for (int s = 0; s < stages; ++s) {
            fast::mbar_wait(bars + 8u * stage, parity);
            if (++stage == stages) { stage = 0; parity ^= 1u; }
        }
    if constexpr (OWNER == kCluster) leave_cluster();
    asm volatile("griddepcontrol.launch_dependents;");
    if (!a.dgamma && !a.dbeta) return;
    if (OWNER == kCluster && owners == 1) {
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (has(k)) {
                if (a.dgamma) store_typed<W>(a.dgamma, a.w_type, beg + (first + k * step) * W, dg[k]);
                if (a.dbeta) store_typed<W>(a.dbeta, a.w_type, beg + (first + k * step) * W, db[k]);
            }
        return;
    }
    // where the owners are joined, their sums take the place of the rows (which no thread reads any more, nor any copy writes)
    float* out = a.joined ? reinterpret_cast<float*>(ring) : a.partial + (int64_t)owner * 2 * a.P + beg;
#pragma unroll
    for (int k = 0; k < NV; ++k)
        if (has(k))
#pragma unroll
            for (int j = 0; j < W; ++j) {
                const int p = (first + k * step) * W + j;
                out[p] = dg[k][j];
                out[a.P + p] = db[k][j];
            }
    if (OWNER == kBlock && a.joined) join_owners(out, a);
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

// Launches a kernel of `owners` blocks, as one cluster where they are joined.
template <class... A, class... B>
cudaError_t launch_joined(void (*kernel)(A...), std::atomic<uint64_t>& done, int owners, int threads, size_t bytes, bool joined, cudaStream_t stream, B... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)owners);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)owners;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = joined ? 1 : 0;
    if (joined && owners > 8) {
        const cudaError_t e = once_per_device(done, [&] { return allow_large_clusters(kernel); });
        if (e != cudaSuccess) return e;
    }
    count_launch();
    return cudaLaunchKernelEx(&cfg, kernel, A(args)...);
}

template <class TX, class TY, int W>
cudaError_t launch_short(const Backward& a, cudaStream_t stream) {
    auto run = [&](auto lanes) {
        constexpr int LANES = decltype(lanes)::value, kMost = kColumns / W;
        return with_int<LANES == 8 ? 1 : kMost / 2 + 1, kMost>((a.P / W + LANES - 1) / LANES, [&](auto nv) {
            static std::atomic<uint64_t> done{0};
            return launch_joined(warp_rows_kernel<TX, TY, W, nv.value, LANES>, done, owners_of(a.N, a.P, a.dgamma || a.dbeta), kThreads, (size_t)(kThreads / 32) * 2 * a.P * sizeof(float), a.joined, stream, a);
        });
    };
    const int lanes = lanes_of(a.P);
    return lanes == 8 ? run(Int<8>()) : lanes == 16 ? run(Int<16>()) : run(Int<32>());
}

// owners: of at most so many, how many there are is put here.
template <class TX, class TY, int W, int NV, Owner OWNER, Fit FIT>
cudaError_t launch_owners(const Backward& a, int& owners, cudaStream_t stream) {
    const int parts = parts_of(a.P), part = part_of(a.P), threads = threads_of(a.P);
    auto kernel = block_rows_kernel<TX, TY, W, NV, OWNER, FIT>;
    static std::atomic<uint64_t> done{0};
    cudaError_t e = once_per_device(done, [&] {
        const cudaError_t set = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemSm - 4096);
        return set == cudaSuccess ? allow_large_clusters(kernel) : set;
    });
    if (e != cudaSuccess) return e;
    const int stage = room_of(part, sizeof(TX)) + room_of(part, sizeof(TY));
    const int stages = std::min(kMostStages, (kSmemSm / resident_of(a.P) - 2048) / stage);      // 2 KB: the block's other arrays, and what the driver keeps
    if (stages < 2) return cudaErrorInvalidConfiguration;      // the edges of a row are stored while the one before is read
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(owners * parts));
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = (size_t)stages * stage;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)(OWNER == kCluster ? parts : owners);
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = OWNER == kCluster || a.joined ? 1 : 0;
    if constexpr (OWNER == kCluster) {
        // not every SM finds partners in its group of SMs: clusters that would have to wait for others to end cost a second round
        static std::atomic<int> known[kMostParts + 1][kThreads / 32 + 1];
        int most = 0;
        e = active_clusters(known[parts][threads / 32], kernel, cfg, most);
        if (e != cudaSuccess) return e;
        owners = std::min(owners, most);
        cfg.gridDim = dim3((unsigned)(owners * parts));
    }
    count_launch();
    return cudaLaunchKernelEx(&cfg, kernel, a, parts, part, stages);
}

// aligned: every row begins on a 16-byte border.
template <class TX, class TY, int W, int NV>
cudaError_t launch_blocks(const Backward& a, bool aligned, int& owners, cudaStream_t stream) {
    const int parts = parts_of(a.P), part = part_of(a.P), least = a.P - (parts - 1) * part, threads = threads_of(a.P);      // least: the last block's columns
    auto with_fit = [&](auto fit) {
        constexpr Fit FIT = decltype(fit)::value;
        return parts > 1 ? launch_owners<TX, TY, W, NV, kCluster, FIT>(a, owners, stream) : launch_owners<TX, TY, W, NV, kBlock, FIT>(a, owners, stream);
    };
    const bool most = least >= (NV - 1) * W * threads;
    constexpr bool kWide = W * sizeof(TX) >= 16 && W * sizeof(TY) >= 16;      // every row begins and ends on a 16-byte border
    if constexpr (W > 1) {
        const bool whole = kWide || (aligned && least * (int)sizeof(TX) % 16 == 0 && least * (int)sizeof(TY) % 16 == 0);
        if (whole && part == least && least == NV * W * threads) return with_fit(std::integral_constant<Fit, kFull>());
        if (whole && most) return with_fit(std::integral_constant<Fit, kLast>());
    }
    if constexpr (!kWide) if (most) return with_fit(std::integral_constant<Fit, kEnd>());
    return with_fit(std::integral_constant<Fit, kAny>());
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

// The kernels of one type of x.
template <class TX>
cudaError_t launch_rows(const Backward& a, int& owners, cudaStream_t stream) {
    auto fits = [&](int W) {
        return a.P % W == 0 && packs(a.x, a.x_type, a.N > 1 ? a.x_stride : 0, W) && packs(a.dy, a.y_type, a.N > 1 ? a.dy_stride : 0, W) &&
               packs(a.dx, a.x_type, a.dx && a.N > 1 ? a.dx_stride : 0, W) && packs(a.gamma, a.w_type, 0, W) && packs(a.dgamma, a.w_type, 0, W) && packs(a.dbeta, a.w_type, 0, W);
    };
    const bool aligned = packs(a.x, ROCKET_F32, 0, 4) && packs(a.dy, ROCKET_F32, 0, 4) &&
                         (a.N <= 1 || (packs(nullptr, a.x_type, a.x_stride, 16 / float_type_bytes(a.x_type)) && packs(nullptr, a.y_type, a.dy_stride, 16 / float_type_bytes(a.y_type))));
    return with_float_type(a.y_type, [&](auto* py) {
        using TY = std::remove_pointer_t<decltype(py)>;
        if (is_long(a.P)) return launch_long<TX, TY>(a, stream);
        if (is_short(a.P)) {
            if constexpr (sizeof(TX) == 2 && sizeof(TY) == 2) if (fits(8)) return launch_short<TX, TY, 8>(a, stream);
            return fits(4) ? launch_short<TX, TY, 4>(a, stream) : launch_short<TX, TY, 1>(a, stream);
        }
        if constexpr (sizeof(TX) == 2 && sizeof(TY) == 2) if (fits(8)) return launch_blocks<TX, TY, 8, kColumns / 8>(a, aligned, owners, stream);
        if (fits(4)) return launch_blocks<TX, TY, 4, kColumns / 4>(a, aligned, owners, stream);
        return launch_blocks<TX, TY, 1, kColumns>(a, aligned, owners, stream);
    });
}

extern template cudaError_t launch_rows<float>(const Backward&, int&, cudaStream_t);
extern template cudaError_t launch_rows<__half>(const Backward&, int&, cudaStream_t);
extern template cudaError_t launch_rows<__nv_bfloat16>(const Backward&, int&, cudaStream_t);

}  // namespace norm
}  // namespace rocket
