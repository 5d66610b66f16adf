// Products over the tokens: gradients of weights.
#include "matmul_launch.h"

namespace cmoe {

hipError_t launch_dw(Tile tile, int dtype, const MatArgs& p, hipStream_t s) {
  if (dtype == CMOE_BF16) return launch_product<true, true, EpiStore<bf16_t, false, true>>(tile, p, s);
  return launch_product<true, true, EpiStore<float, false, true>>(tile, p, s);
}

}  // namespace cmoe
