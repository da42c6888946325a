// Layer norm forward, x of type __half.
#include "rocket_norm_forward.cuh"

namespace rocket {
namespace norm {

template cudaError_t launch_rows<__half>(const Forward&, cudaStream_t);

}  // namespace norm
}  // namespace rocket
