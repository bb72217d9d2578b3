// Host-side checks shared by the entry points of attention_mi355x.h.
#pragma once

#include <algorithm>
#include <cmath>
#include <cstdlib>

#include "../../include/attention_mi355x.h"
#include "sm_host.hpp"

namespace smx_host {

inline int dtype_size(int dtype) {
  return dtype == SOFTMAX_F32 ? 4 : dtype == SOFTMAX_F16 || dtype == SOFTMAX_BF16 ? 2 : 0;
}

// log2 of a power of two up to 2^20, else -1.
inline int log2_of(int64_t x) {
  for (int i = 0; i <= 20; ++i)
    if (x == int64_t(1) << i) return i;
  return -1;
}

// extent += (count - 1) * stride without overflow; both not negative.
inline bool add_extent(int64_t count, int64_t stride, int64_t* extent) {
  int64_t x = 0;
  return stride >= 0 && !__builtin_mul_overflow(count - 1, stride, &x) &&
         !__builtin_add_overflow(*extent, x, extent);
}

// Positions and their sums with a tile's stay within 31 bits.
constexpr int64_t kMaxTokens = int64_t(1) << 30;

// The layout rules of a tensor [tokens, heads, d]; its extent in bytes (0
// when empty).
inline bool heads_ok(const softmax_heads_t* t, int size, int64_t* bytes) {
  *bytes = 0;
  if (t == nullptr || t->tokens < 0 || t->heads < 0 || t->tokens > kMaxTokens ||
      t->heads > INT32_MAX || t->d < 8 || t->d > SOFTMAX_HEADS_MAX_DIM || t->d % 8 != 0)
    return false;
  // A tile's offsets between its rows fit 31 bits.
  if (t->token_stride < 0 || t->token_stride > SOFTMAX_HEADS_MAX_STRIDE || t->head_stride < 0)
    return false;
  if (t->tokens == 0 || t->heads == 0) return true;
  const int64_t strip = 16 / size;
  if (!aligned16(t->data) || t->token_stride % strip != 0 || t->head_stride % strip != 0)
    return false;
  int64_t extent = t->d;
  if (!add_extent(t->tokens, t->token_stride, &extent) ||
      !add_extent(t->heads, t->head_stride, &extent) || extent > INT64_MAX / size)
    return false;
  *bytes = extent * size;
  return true;
}

inline bool cache_ok(const softmax_cache_t* t, int size, int64_t* bytes) {
  *bytes = 0;
  if (t == nullptr || t->blocks < 0 || t->blocks > INT32_MAX || log2_of(t->block_size) < 0 ||
      t->heads < 0 || t->heads > INT32_MAX || t->d < 8 || t->d > SOFTMAX_HEADS_MAX_DIM ||
      t->d % 8 != 0)
    return false;
  if (t->block_stride < 0 || t->token_stride < 0 || t->token_stride > SOFTMAX_HEADS_MAX_STRIDE ||
      t->head_stride < 0)
    return false;
  if (t->blocks == 0 || t->heads == 0) return true;
  const int64_t strip = 16 / size;
  if (!aligned16(t->data) || t->block_stride % strip != 0 || t->token_stride % strip != 0 ||
      t->head_stride % strip != 0)
    return false;
  int64_t extent = t->d;
  if (!add_extent(t->blocks, t->block_stride, &extent) ||
      !add_extent(t->block_size, t->token_stride, &extent) ||
      !add_extent(t->heads, t->head_stride, &extent) || extent > INT64_MAX / size)
    return false;
  *bytes = extent * size;
  return true;
}

inline bool same_cache(const softmax_cache_t* a, const softmax_cache_t* b) {
  return a->blocks == b->blocks && a->block_size == b->block_size && a->heads == b->heads &&
         a->d == b->d;
}

// Whether two caches of one shape have an element in common.  Their extents may
// overlap: a cache of both, with one's rows between the other's.  With the same
// strides two elements meet where the distance of the caches is a sum of index
// differences times strides; strides that do not overlap themselves leave two
// choices per axis, from the largest stride down, and a remainder within a row.
// Caches of different strides have no element in common if their extents have
// none, or else are taken to interleave unless they start at one place.
inline bool caches_meet(const softmax_cache_t* a, int64_t a_bytes, const softmax_cache_t* b,
                        int64_t b_bytes, int size) {
  const auto pa = reinterpret_cast<uintptr_t>(a->data), pb = reinterpret_cast<uintptr_t>(b->data);
  if (pa >= pb + b_bytes || pb >= pa + a_bytes) return false;
  if (pa == pb) return true;
  if (a->block_stride != b->block_stride || a->token_stride != b->token_stride ||
      a->head_stride != b->head_stride)
    return false;
  struct Axis {
    int64_t stride, count;
  } axes[3] = {{a->block_stride, a->blocks}, {a->token_stride, a->block_size},
               {a->head_stride, a->heads}};
  std::sort(axes, axes + 3, [](const Axis& x, const Axis& y) { return x.stride > y.stride; });
  int64_t left[8] = {static_cast<int64_t>(pa > pb ? pa - pb : pb - pa) / size};
  int n = 1;
  for (const Axis& x : axes) {
    if (x.stride == 0 || x.count <= 1) continue;
    for (int i = n; i-- > 0;) {  // the distance left over, or what the next step is too far
      const int64_t from = left[i], q = std::min(from / x.stride, x.count - 1);
      left[i] = from - q * x.stride;
      left[n + i] = q + 1 < x.count ? std::abs(from - (q + 1) * x.stride) : left[i];
    }
    n *= 2;
  }
  return std::any_of(left, left + n, [&](int64_t x) { return x < a->d; });
}

inline bool score_ok(const softmax_score_t* s) {
  return s != nullptr && std::isfinite(s->scale) && std::isfinite(s->cap) &&
         (s->cap == 0.0f || s->cap >= SOFTMAX_MIN_CAP) &&
         (s->causal == 0 || s->causal == 1) && (s->causal == 1 || s->prefix == nullptr);
}

struct Range {
  const void* p;
  int64_t bytes;
};

// The device allocation that a call's last checked range lies in: the small
// tensors of a call often share one, and a look-up costs 0.2 us.
struct Allocation {
  uintptr_t lo, hi;
};

inline int check_device_range(const Range& r, int dev, Allocation* last) {
  if (r.bytes <= 0) return SOFTMAX_OK;
  const uintptr_t p = reinterpret_cast<uintptr_t>(r.p);
  if (p >= last->lo && p < last->hi && static_cast<uintptr_t>(r.bytes) <= last->hi - p)
    return SOFTMAX_OK;
  if (const int rc = check_device_range(r.p, r.bytes, dev)) return rc;
  hipDeviceptr_t base = nullptr;
  size_t size = 0;
  if (hipMemGetAddressRange(&base, &size, const_cast<void*>(r.p)) == hipSuccess)
    *last = {reinterpret_cast<uintptr_t>(base), reinterpret_cast<uintptr_t>(base) + size};
  else
    (void)hipGetLastError();  // host memory: each range by itself
  return SOFTMAX_OK;
}

// Every range is memory that the current device can use, and no output
// overlaps an input or another output (`interleaved`: outputs may overlap
// each other).  Empty ranges may be null.
template <int NI, int NO>
int check_ranges(const Range (&in)[NI], const Range (&out)[NO], bool interleaved = false) {
  for (const Range& r : in)
    if (r.bytes > 0 && r.p == nullptr) return SOFTMAX_ERR_INVALID_ARG;
  for (int i = 0; i < NO; ++i) {
    if (out[i].bytes > 0 && out[i].p == nullptr) return SOFTMAX_ERR_INVALID_ARG;
    for (const Range& r : in)
      if (ranges_overlap(out[i].p, out[i].bytes, r.p, r.bytes)) return SOFTMAX_ERR_INVALID_ARG;
    for (int j = 0; j < i && !interleaved; ++j)
      if (ranges_overlap(out[i].p, out[i].bytes, out[j].p, out[j].bytes))
        return SOFTMAX_ERR_INVALID_ARG;
  }
  int dev = 0;
  const hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return fail_hip(e);
  Allocation last = {};
  for (const Range& r : in)
    if (const int rc = check_device_range(r, dev, &last)) return rc;
  for (const Range& r : out)
    if (const int rc = check_device_range(r, dev, &last)) return rc;
  return SOFTMAX_OK;
}

}  // namespace smx_host
