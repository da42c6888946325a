// Layer norm of rows, forward and backward: the step between pooled features and a trained head, and back.  The entry points and
// their checks; the kernels are in rocket_norm_forward.cu and rocket_norm_backward.cu.
#include <cmath>

#include "rocket_float_types.cuh"
#include "rocket_internal.h"
#include "rocket_norm.h"

namespace rocket {
namespace {

// Rows [N][P] of `bytes` bytes a value, `stride` values apart.
struct Rows {
    uintptr_t base;
    int64_t N, P, stride;
    int bytes;
    uintptr_t end() const { return base + (uintptr_t)((N - 1) * stride + P) * bytes; }
};

// Whether an output shares a byte with another array.  Rows of equal distance may interleave (halves of one wider buffer).
bool overlap(const Rows& a, const Rows& b) {
    if (!a.base || !b.base || a.end() <= b.base || b.end() <= a.base) return false;
    const uintptr_t step = (uintptr_t)a.stride * a.bytes;
    if (a.N > 1 && step == (uintptr_t)b.stride * b.bytes && step > 0) {
        const uintptr_t wa = (uintptr_t)a.P * a.bytes, wb = (uintptr_t)b.P * b.bytes;
        const uintptr_t off = b.base >= a.base ? (b.base - a.base) % step : (step - (a.base - b.base) % step) % step;
        return !(off >= wa && off + wb <= step);
    }
    return true;
}

bool misaligned(const void* p, int type) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(float_type_bytes(type) - 1)) != 0; }

int status_of(cudaError_t e) {
    if (e == cudaSuccess) return ROCKET_OK;
    cudaGetLastError();
    return e == cudaErrorMemoryAllocation ? ROCKET_ENOMEM : ROCKET_ECUDA;
}

// Strides whose byte offsets stay far inside 64 bits; the rows of an output do not overlap.
bool stride_ok(int N, int P, int64_t stride, bool output) {
    return N <= 1 || (stride >= (output ? P : 0) && stride <= (int64_t(1) << 58) / N);
}

}  // namespace
}  // namespace rocket

using namespace rocket;

extern "C" int rocket_layer_norm(const void* x_dev, int x_type, int64_t x_stride, int N, int P, const void* gamma_dev,
                                 const void* beta_dev, int w_type, float eps, void* y_dev, int y_type, int64_t y_stride,
                                 float* mean_dev, float* rstd_dev, void* cuda_stream) {
    if (!is_float_type(x_type) || !is_float_type(y_type) || !is_float_type(w_type)) return ROCKET_EINVAL;
    if (N < 0 || P < 1 || !(eps >= 0.0f) || std::isinf(eps)) return ROCKET_EINVAL;
    if (N == 0) return ROCKET_OK;
    if (!x_dev || !y_dev || !stride_ok(N, P, x_stride, false) || !stride_ok(N, P, y_stride, true)) return ROCKET_EINVAL;
    if (misaligned(x_dev, x_type) || misaligned(y_dev, y_type) || misaligned(gamma_dev, w_type) || misaligned(beta_dev, w_type) ||
        misaligned(mean_dev, ROCKET_F32) || misaligned(rstd_dev, ROCKET_F32))
        return ROCKET_EINVAL;
    const Rows in[] = {{(uintptr_t)x_dev, N, P, N > 1 ? x_stride : P, float_type_bytes(x_type)},
                       {(uintptr_t)gamma_dev, 1, P, P, float_type_bytes(w_type)},
                       {(uintptr_t)beta_dev, 1, P, P, float_type_bytes(w_type)}};
    const Rows out[] = {{(uintptr_t)y_dev, N, P, N > 1 ? y_stride : P, float_type_bytes(y_type)},
                        {(uintptr_t)mean_dev, 1, N, N, 4},
                        {(uintptr_t)rstd_dev, 1, N, N, 4}};
    for (int o = 0; o < 3; ++o) {
        for (const Rows& i : in) if (overlap(out[o], i)) return ROCKET_EINVAL;
        for (int p = 0; p < o; ++p) if (overlap(out[o], out[p])) return ROCKET_EINVAL;
    }
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const norm::Forward a = {x_dev, y_dev, gamma_dev, beta_dev, mean_dev, rstd_dev, x_stride, y_stride, N, P, x_type, y_type, w_type, eps};
    return status_of(norm::launch_forward(a, stream));
}

extern "C" int64_t rocket_layer_norm_backward_workspace(int N, int P) {
    return N < 0 || P < 1 ? ROCKET_EINVAL : norm::backward_workspace(N, P);
}

extern "C" int rocket_layer_norm_backward(const void* dy_dev, int y_type, int64_t dy_stride, const void* x_dev, int x_type,
                                          int64_t x_stride, int N, int P, const void* gamma_dev, int w_type,
                                          const float* mean_dev, const float* rstd_dev, void* dx_dev, int64_t dx_stride,
                                          void* dgamma_dev, void* dbeta_dev, void* workspace_dev, int64_t workspace_bytes,
                                          void* cuda_stream) {
    if (!is_float_type(x_type) || !is_float_type(y_type) || !is_float_type(w_type)) return ROCKET_EINVAL;
    if (N < 0 || P < 1 || workspace_bytes < 0 || (!dx_dev && !dgamma_dev && !dbeta_dev)) return ROCKET_EINVAL;
    if (misaligned(dgamma_dev, w_type) || misaligned(dbeta_dev, w_type) || misaligned(gamma_dev, w_type) || misaligned(dy_dev, y_type) ||
        misaligned(x_dev, x_type) || misaligned(dx_dev, x_type) || misaligned(mean_dev, ROCKET_F32) || misaligned(rstd_dev, ROCKET_F32))
        return ROCKET_EINVAL;
    if (N > 0 && (!dy_dev || !x_dev || !mean_dev || !rstd_dev)) return ROCKET_EINVAL;
    if (!stride_ok(N, P, dy_stride, false) || !stride_ok(N, P, x_stride, false) || (dx_dev && !stride_ok(N, P, dx_stride, true))) return ROCKET_EINVAL;
    const int64_t need = dgamma_dev || dbeta_dev ? rocket_layer_norm_backward_workspace(N, P) : 0;
    if (workspace_bytes < need || (need > 0 && (!workspace_dev || (reinterpret_cast<uintptr_t>(workspace_dev) & 15u)))) return ROCKET_EINVAL;
    const int xb = float_type_bytes(x_type), wb = float_type_bytes(w_type);
    const Rows none = {0, 1, 1, 1, 1};
    const Rows in[] = {N ? Rows{(uintptr_t)dy_dev, N, P, N > 1 ? dy_stride : P, float_type_bytes(y_type)} : none,
                       N ? Rows{(uintptr_t)x_dev, N, P, N > 1 ? x_stride : P, xb} : none,
                       {(uintptr_t)gamma_dev, 1, P, P, wb},
                       N ? Rows{(uintptr_t)mean_dev, 1, N, N, 4} : none,
                       N ? Rows{(uintptr_t)rstd_dev, 1, N, N, 4} : none};
    const Rows out[] = {N ? Rows{(uintptr_t)dx_dev, N, P, N > 1 ? dx_stride : P, xb} : none,
                        {(uintptr_t)dgamma_dev, 1, P, P, wb},
                        {(uintptr_t)dbeta_dev, 1, P, P, wb},
                        need ? Rows{(uintptr_t)workspace_dev, 1, need, need, 1} : none};
    for (int o = 0; o < 4; ++o) {
        for (const Rows& i : in) if (overlap(out[o], i)) return ROCKET_EINVAL;
        for (int p = 0; p < o; ++p) if (overlap(out[o], out[p])) return ROCKET_EINVAL;
    }
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const norm::Backward a = {dy_dev, x_dev, gamma_dev, mean_dev, rstd_dev, dx_dev, dgamma_dev, dbeta_dev, static_cast<float*>(workspace_dev),
                              dy_stride, x_stride, dx_stride, N, P, y_type, x_type, w_type, false};
    return status_of(norm::launch_backward(a, stream));
}
