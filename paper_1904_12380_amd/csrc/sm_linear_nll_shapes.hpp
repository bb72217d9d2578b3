// Tile shapes of the products of 16-bit types.
#pragma once

#include "sm_linear_nll.hpp"
#include "sm_linear_nll_launch.hpp"

namespace smx {

template <typename T, int KIND, int BM, int BN, int WM, int WN, int STAGES>
NllProduct nll_shape() {
  return {reinterpret_cast<const void*>(&k_nll_product<T, KIND, BM, BN, WM, WN, STAGES>), BM, BN,
          64 * WM * WN};
}

template <typename T>
NllProduct nll_product_16(int kind, int64_t tokens) {
  const bool few = tokens <= 64;
  switch (kind) {
    case kLogits:
      return few ? nll_shape<T, kLogits, 128, 64, 4, 1, 3>()
                 : nll_shape<T, kLogits, 256, 256, 2, 4, 2>();
    case kProbs:
      return few ? nll_shape<T, kProbs, 128, 64, 4, 1, 3>()
                 : nll_shape<T, kProbs, 256, 256, 2, 4, 2>();
    case kInput:
      return few ? nll_shape<T, kInput, 128, 64, 4, 1, 3>()
                 : nll_shape<T, kInput, 256, 256, 2, 4, 2>();
    default:
      return nll_shape<T, kWeight, 256, 256, 2, 4, 2>();
  }
}

}  // namespace smx
