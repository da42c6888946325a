// Layer norm forward, x of type float.
#include "rocket_norm_forward.cuh"

namespace rocket {
namespace norm {

template cudaError_t launch_rows<float>(const Forward&, cudaStream_t);

}  // namespace norm
}  // namespace rocket
