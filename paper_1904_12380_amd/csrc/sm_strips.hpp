// Rows in 16-byte strips, as the kernels around the attention read and write them.
#pragma once

#include "sm_heads.hpp"

namespace smx {

// A row's 16 bytes at a time.
template <typename T>
struct Strip {
  static constexpr int kN = 16 / sizeof(T);
  typedef T type __attribute__((ext_vector_type(16 / sizeof(T))));
  static __device__ __forceinline__ type load(const T* p) { return *reinterpret_cast<const type*>(p); }
  static __device__ __forceinline__ void store(T* p, const float (&v)[kN]) {
    type x;
#pragma unroll
    for (int i = 0; i < kN; ++i) x[i] = static_cast<T>(v[i]);
    *reinterpret_cast<type*>(p) = x;
  }
};

// i / per for i < all (64-bit divisions only where they are needed).
__device__ __forceinline__ int64_t row_of(int64_t i, unsigned per, int64_t all) {
  return all >> 32 == 0 ? static_cast<unsigned>(i) / per : i / per;
}

}  // namespace smx
