// Layer norm forward, x of type __nv_bfloat16.
#include "rocket_norm_forward.cuh"

namespace rocket {
namespace norm {

template cudaError_t launch_rows<__nv_bfloat16>(const Forward&, cudaStream_t);

}  // namespace norm
}  // namespace rocket
