// act(x W^T + bias) + residual with a microscaled matrix.
#include "mx4_product.hpp"

namespace sun {

hipError_t launch_mx4_fused(const Mx4Linear& m, void* workspace, hipStream_t st) { return linear<FUSED>(m, workspace, st); }

}  // namespace sun
