// act(x Wg^T) * (x Wu^T) with microscaled matrices: the product of a pair whose tiles of 16 columns alternate, so that both sums of a column meet in a wave.
#include "mx4_product.hpp"

namespace sun {

hipError_t launch_mx4_gated(const Mx4Linear& m, void* workspace, hipStream_t st) { return linear<GATED>(m, workspace, st); }

}  // namespace sun
