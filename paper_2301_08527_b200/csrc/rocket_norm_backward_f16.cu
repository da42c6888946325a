// Layer norm backward, x of type __half.
#include "rocket_norm_backward.cuh"

namespace rocket {
namespace norm {

template cudaError_t launch_rows<__half>(const Backward&, int&, cudaStream_t);

}  // namespace norm
}  // namespace rocket
