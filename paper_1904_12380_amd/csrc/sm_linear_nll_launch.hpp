// The compiled instances of the tile products behind the loss over a vocabulary,
// each type in a source file of its own.
#pragma once

#include <stdint.h>

namespace smx {

// One of the products (kLogits .. kPartial of sm_linear_nll.hpp) and its shape.
struct NllProduct {
  const void* fn;
  int bm, bn, threads;
  int resident;  // workgroups of a CU that a split counts on
};

constexpr int kNarrow = 0, kSmall = 1, kLarge = 2;

NllProduct nll_product_f32(int kind, int64_t m, int64_t n);
NllProduct nll_product_f16(int kind, int64_t m, int64_t n);
NllProduct nll_product_bf16(int kind, int64_t m, int64_t n);

}  // namespace smx
