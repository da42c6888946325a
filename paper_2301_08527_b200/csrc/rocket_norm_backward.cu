// Layer norm backward: which kernels a call takes, and the sum over the owners of rows.  The kernels for a type of x are compiled in a unit
// of their own (rocket_norm_backward_*.cu).
#include "rocket_norm_backward.cuh"

namespace rocket {
namespace norm {
namespace {

// dg and db from the owners' sums: a lane has C columns, a block 32 C, its warps share the owners.  The warps' sums, each at a good part of the whole's
// magnitude, are added in double precision; the owners' in fp32, as the rows before them (in double too, 32 x 20,000 takes 0.8 us more).
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
        double sum = 0.0;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) sum += (double)red[which][w][c];
        const float v[1] = {(float)sum};
        store_typed<1>(out, w_type, column, v);
    }
}

}  // namespace

int64_t backward_workspace(int N, int P) {
    const int owners = owners_of(N, P, true);
    return owners > 1 && !is_joined(N, P) ? (int64_t)owners * 2 * P * (int64_t)sizeof(float) : 0;
}

cudaError_t launch_backward(const Backward& args, cudaStream_t stream) {
    Backward a = args;
    if (a.N == 0 && !a.dgamma && !a.dbeta) return cudaSuccess;
    const bool weights = a.dgamma || a.dbeta;
    a.joined = weights && is_joined(a.N, a.P);
    int owners = owners_of(a.N, a.P, weights);
    const cudaError_t e = with_float_type(a.x_type, [&](auto* px) { return launch_rows<std::remove_pointer_t<decltype(px)>>(a, owners, stream); });
    if (e != cudaSuccess || owners <= 1 || a.joined || !weights) return e;
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
