// Instances of the tile products of the loss over a vocabulary for bf16.
#include "sm_linear_nll_shapes.hpp"

namespace smx {

NllProduct nll_product_bf16(int kind, int64_t m, int64_t n) {
  return nll_product_of<bf16>(kind, m, n);
}

}  // namespace smx
