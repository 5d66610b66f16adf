// The head's products: logits reduced to their largest and sum, their gradient, and what it sends to the input.
#include "matmul_launch.h"

namespace cmoe {

hipError_t launch_lse(Tile tile, int dtype, const MatArgs& p, hipStream_t s) {
  if (dtype == CMOE_BF16) return launch_product<false, false, EpiLse<bf16_t>>(tile, p, s);
  return launch_product<false, false, EpiLse<float>>(tile, p, s);
}

hipError_t launch_dlogits(Tile tile, int dtype, const MatArgs& p, hipStream_t s) {
  if (dtype == CMOE_BF16) return launch_product<false, false, EpiDLogits<bf16_t>>(tile, p, s);
  return launch_product<false, false, EpiDLogits<float>>(tile, p, s);
}

hipError_t launch_dhead(Tile tile, int dtype, const MatArgs& p, hipStream_t s) {
  if (dtype == CMOE_BF16) return launch_product<false, true, EpiDHead<bf16_t>>(tile, p, s);
  return launch_product<false, true, EpiDHead<float>>(tile, p, s);
}

}  // namespace cmoe
