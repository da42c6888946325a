// Layer norm backward, x of type float.
#include "rocket_norm_backward.cuh"

namespace rocket {
namespace norm {

template cudaError_t launch_rows<float>(const Backward&, int&, cudaStream_t);

}  // namespace norm
}  // namespace rocket
