// Launchers of the layer norm kernels; the entry points (rocket_layer_norm.cu) have checked the arguments.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

namespace rocket {
namespace norm {

struct Forward {
    const void* x;
    void* y;
    const void* gamma;    // nullptr: ones
    const void* beta;     // nullptr: zeros
    float* mean;          // nullptr: not wanted
    float* rstd;
    int64_t x_stride, y_stride;
    int N, P, x_type, y_type, w_type;
    float eps;
};

cudaError_t launch_forward(const Forward& a, cudaStream_t stream);

struct Backward {
    const void* dy;
    const void* x;
    const void* gamma;    // nullptr: ones
    const float* mean;
    const float* rstd;
    void* dx;             // nullptr: not wanted, as dgamma and dbeta
    void* dgamma;
    void* dbeta;
    float* partial;       // workspace
    int64_t dy_stride, x_stride, dx_stride;
    int N, P, y_type, x_type, w_type;
    bool joined;          // the owners' sums meet in a cluster
};

// Bytes of workspace for the gradients of gamma and beta.
int64_t backward_workspace(int N, int P);
cudaError_t launch_backward(const Backward& a, cudaStream_t stream);

}  // namespace norm
}  // namespace rocket
