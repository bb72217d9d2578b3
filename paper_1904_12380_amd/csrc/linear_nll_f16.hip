// Instances of the tile products of the loss over a vocabulary for fp16.
#include "sm_linear_nll_shapes.hpp"

namespace smx {

NllProduct nll_product_f16(int kind, int64_t m, int64_t n) {
  return nll_product_of<f16>(kind, m, n);
}

}  // namespace smx
