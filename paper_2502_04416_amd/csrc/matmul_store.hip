// Products whose result is stored as it is: the down projection, the gradient of the block's input.
#include "matmul_launch.h"

namespace cmoe {

hipError_t launch_down(Tile tile, int dtype, const MatArgs& p, hipStream_t s) {
  if (dtype == CMOE_BF16) return launch_product<false, true, EpiStore<bf16_t, false, false>>(tile, p, s);
  return launch_product<false, true, EpiStore<float, false, false>>(tile, p, s);
}

hipError_t launch_dx(Tile tile, int dtype, const MatArgs& p, hipStream_t s) {
  if (dtype == CMOE_BF16) return launch_product<false, false, EpiStore<bf16_t, true, false>>(tile, p, s);
  return launch_product<false, false, EpiStore<float, true, false>>(tile, p, s);
}

}  // namespace cmoe
