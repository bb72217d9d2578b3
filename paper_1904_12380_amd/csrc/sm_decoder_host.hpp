// Host-side checks shared by the entry points of decoder_mi355x.h.
#pragma once

#include "../../include/decoder_mi355x.h"
#include "sm_heads_host.hpp"

namespace smx_host {

// Rows and tokens of a call: indices stay below 2^31, and a launch with four threads
// for each below 2^32.
constexpr int64_t kMaxRows = int64_t(1) << 29;

inline bool width_ok(int64_t d) { return d >= 8 && d <= SOFTMAX_MAX_WIDTH && d % 8 == 0; }

inline bool count_ok(int64_t n) { return n >= 0 && n <= kMaxRows; }

// The layout rules of rows [rows, d]; their extent in bytes (0 when empty).
inline bool rows_ok(const void* data, int64_t rows, int64_t stride, int64_t d, int size,
                    int64_t* bytes) {
  *bytes = 0;
  if (rows == 0) return true;
  int64_t extent = d;
  if (!aligned16(data) || stride % (16 / size) != 0 || !add_extent(rows, stride, &extent) ||
      extent > INT64_MAX / size)
    return false;
  *bytes = extent * size;
  return true;
}

inline int64_t up_to(int64_t x, int64_t whole) { return ceil_div(x, whole) * whole; }

}  // namespace smx_host
