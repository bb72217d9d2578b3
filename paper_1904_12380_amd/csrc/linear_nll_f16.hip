// Instances of the tile products of the loss over a vocabulary for f16.
#include "sm_linear_nll_shapes.hpp"

namespace smx {

NllProduct nll_product_f16(int kind, int64_t tokens) { return nll_product_16<f16>(kind, tokens); }

}  // namespace smx
