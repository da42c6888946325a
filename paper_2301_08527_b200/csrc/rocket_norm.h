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

}  // namespace norm
}  // namespace rocket
