// The gated block's products: both projections with the activation, and its gradient.
#include "matmul_launch.h"

namespace cmoe {

hipError_t launch_gated(Tile tile, int dtype, const MatArgs& p, hipStream_t s) {
  if (dtype == CMOE_BF16) return launch_product<false, true, EpiGated<bf16_t>>(tile, p, s);
  return launch_product<false, true, EpiGated<float>>(tile, p, s);
}

hipError_t launch_dgated(Tile tile, int dtype, const MatArgs& p, hipStream_t s) {
  if (dtype == CMOE_BF16) return launch_product<false, false, EpiDGated<bf16_t>>(tile, p, s);
  return launch_product<false, false, EpiDGated<float>>(tile, p, s);
}

}  // namespace cmoe
