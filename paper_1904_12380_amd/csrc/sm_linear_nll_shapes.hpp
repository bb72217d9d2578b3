// Tile shapes of the products.
#pragma once

#include "sm_linear_nll.hpp"
#include "sm_linear_nll_launch.hpp"

namespace smx {

// The LDS of a CU holds two workgroups of all tiles but the 16-bit types' large ones, and
// splits count on both, but for the 16-bit types' narrow ones, where more splits are more
// sums to join (with gradients, 64 tokens x 10000 x 1024 of fp16: 72 us, counting on two
// 78; 60 x 75898 x 2816 of fp32: counting on one 1509, on two 1302).
template <typename T, int KIND, int BM, int BN, int WM, int WN, int STAGES>
NllProduct nll_shape() {
  typedef Product<T, NllShape<KIND>::kARows, NllShape<KIND>::kBRows, BM, BN, WM, WN, STAGES> P;
  return {reinterpret_cast<const void*>(&k_nll_product<T, KIND, BM, BN, WM, WN, STAGES>), BM, BN,
          64 * WM * WN, sizeof(T) == 4 || P::kLds <= 72 * 1024 ? 2 : 1};
}

// Up to kNllFew tokens: bound by the weight's bytes, so tiles are narrow in tokens
// (forward, 50001 x 2048 of bf16: 64 tokens 44 us, 65 in the next tiles 54).  Otherwise
// the largest tiles, unless they are too few to fill three quarters of the CUs (351
// tokens x 10007 x 520 of fp16, 80 large tiles: 21.1 us with them, 13.8 with the small
// ones; fp32's run two to a CU, so that takes 384, but for dx, whose splits make up for
// it: 1000 x 5000 x 1000 with gradients 528 us with 320 large ones, 397 with small ones)
// or half of each would be empty (probabilities of 128 tokens x 50001 x 2048 85 us, with
// small ones 67).  dweight of few tokens keeps the large ones: 128 tokens 111 us, with
// small ones 123.
constexpr int64_t kNllFew = 64;

template <typename T, int KIND>
NllProduct nll_shape_of(int size) {
  if constexpr (KIND != kWeight) {
    if (size == kNarrow) return nll_shape<T, KIND, 128, 64, 4, 1, 3>();
  }
  if constexpr (sizeof(T) == 2) {
    return size == kLarge ? nll_shape<T, KIND, 256, 256, 2, 4, 2>()
                          : nll_shape<T, KIND, 128, 128, 2, 2, 2>();
  } else {
    if constexpr (KIND != kPartial) {  // for few tiles
      if (size == kLarge) return nll_shape<T, KIND, 128, 128, 2, 2, 2>();
    }
    return nll_shape<T, KIND, 64, 64, 2, 2, 3>();
  }
}

// The product of `kind` for m x n entries.
template <typename T>
NllProduct nll_product_of(int kind, int64_t m, int64_t n) {
  constexpr int64_t kEdge = sizeof(T) == 2 ? 256 : 128;
  const int64_t tiles = ((m + kEdge - 1) / kEdge) * ((n + kEdge - 1) / kEdge);
  const bool tokens = kind != kWeight;  // n
  const int64_t full = sizeof(T) == 4 && kind != kInput ? 384 : 192;
  const int size = tokens && n <= kNllFew                            ? kNarrow
                   : tiles >= full && !(tokens && n <= kEdge / 2) ? kLarge : kSmall;
  if constexpr (sizeof(T) == 4) {
    if (kind == kPartial) return nll_shape_of<T, kPartial>(size);
  }
  switch (kind) {
    case kLogits: return nll_shape_of<T, kLogits>(size);
    case kProbs: return nll_shape_of<T, kProbs>(size);
    case kInput: return nll_shape_of<T, kInput>(size);
    default: return nll_shape_of<T, kWeight>(size);
  }
}

}  // namespace smx
