// Layer norm backward, x of type __nv_bfloat16.
#include "rocket_norm_backward.cuh"

namespace rocket {
namespace norm {

template cudaError_t launch_rows<__nv_bfloat16>(const Backward&, int&, cudaStream_t);

}  // namespace norm
}  // namespace rocket
