// Instances of the tile products of the loss over a vocabulary for fp32.
#include "sm_linear_nll_shapes.hpp"

namespace smx {

NllProduct nll_product_f32(int kind, int64_t tokens) {
  const bool few = tokens <= 64;
  switch (kind) {
    case kLogits:
      return few ? nll_shape<float, kLogits, 128, 64, 4, 1, 3>()
                 : nll_shape<float, kLogits, 128, 128, 2, 2, 2>();
    case kProbs:
      return few ? nll_shape<float, kProbs, 128, 64, 4, 1, 3>()
                 : nll_shape<float, kProbs, 128, 128, 2, 2, 2>();
    case kInput:
      return few ? nll_shape<float, kInput, 128, 64, 4, 1, 3>()
                 : nll_shape<float, kInput, 128, 128, 2, 2, 2>();
    default:
      return nll_shape<float, kWeight, 128, 128, 2, 2, 2>();
  }
}

}  // namespace smx
