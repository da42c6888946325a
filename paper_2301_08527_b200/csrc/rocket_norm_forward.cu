// Layer norm forward: the call by the type of x.  The kernels for each are compiled in a unit of their own (rocket_norm_forward_*.cu).
#include "rocket_norm_forward.cuh"

namespace rocket {
namespace norm {

cudaError_t launch_forward(const Forward& a, cudaStream_t stream) {
    return with_float_type(a.x_type, [&](auto* tx) { return launch_rows<std::remove_pointer_t<decltype(tx)>>(a, stream); });
}

}  // namespace norm
}  // namespace rocket
