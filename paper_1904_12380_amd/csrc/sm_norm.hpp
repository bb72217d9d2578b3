// Norms of rows and their gradients (include/decoder_mi355x.h has the operations).
//
// Bound by memory: the forward pass reads and writes a row, the backward pass reads
// two and writes one.  A row is held in registers between its statistics and its
// output, by L lanes (part of a wavefront, one, or a workgroup) with S strips of 16
// bytes each, so every byte moves once; the variance is formed from differences from
// the mean.
//
//   k_norm_fwd   L lanes per row
//   k_norm_bwd   a fixed number of workgroups, each over rows of its own, which sum
//                their columns' shares of dweight and dbias in registers
//   k_norm_join  those sums over the workgroups, in order
//
// 16384 x 4096 of bf16: 50 us forward (5.4 TB/s), 87 + 7 backward (4.7 TB/s); 115200 x
// 200 of fp16: 19 and 28 + 4 us.
#pragma once

#include "sm_strips.hpp"

namespace smx {

struct NormArgs {
  const void* x;
  const void* dy;
  int64_t x_pitch, dy_pitch;  // elements
  const void* weight;         // may be null
  const void* bias;           // may be null
  void* out;                  // y, or dx (may be null)
  float* mean;                // null: without center
  float* rstd;
  void* dweight;              // may be null
  void* dbias;                // may be null
  float* part;                // [groups, 2, d]
  int rows, d, groups;
  float eps;
};

// Sums over the row's L lanes, the same bits in each; `lds` has a place for every
// wavefront and value.
template <int L, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float (*lds)[N]) {
  if constexpr (L <= 64) {
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = seg_sum<L>(v[n]);
  } else {
    const int wave = threadIdx.x / 64;
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = seg_sum<64>(v[n]);
    __syncthreads();  // the places have been read
    if (threadIdx.x % 64 == 0) {
#pragma unroll
      for (int n = 0; n < N; ++n) lds[wave][n] = v[n];
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n) {
      v[n] = 0.0f;
#pragma unroll
      for (int w = 0; w < L / 64; ++w) v[n] += lds[w][n];
    }
  }
}

// A lane's strips of a row (lane j: strips j, j + L, ..) in fp32; zeros past its end.
template <typename T, int L, int S>
__device__ __forceinline__ void load_row(float (&v)[S][Strip<T>::kN], const T* row, int j,
                                         int strips, bool live) {
  constexpr int kN = Strip<T>::kN;
  typename Strip<T>::type x[S];
#pragma unroll
  for (int s = 0; s < S; ++s) {
    x[s] = typename Strip<T>::type{};
    if (live && j + L * s < strips) x[s] = Strip<T>::load(row + (j + L * s) * kN);
  }
#pragma unroll
  for (int s = 0; s < S; ++s)
#pragma unroll
    for (int e = 0; e < kN; ++e) v[s][e] = static_cast<float>(x[s][e]);
}

template <int S, int N, typename F>
__device__ __forceinline__ float strip_sum(F f) {
  float t[N];
#pragma unroll
  for (int e = 0; e < N; ++e) {
    t[e] = 0.0f;
#pragma unroll
    for (int s = 0; s < S; ++s) t[e] += f(s, e);
  }
  return tree_sum(t);
}

template <typename T, int L, int S>
__global__ __launch_bounds__(L < 256 ? 256 : L) void k_norm_fwd(NormArgs a) {
  constexpr int kN = Strip<T>::kN, kRows = L < 256 ? 256 / L : 1;
  __shared__ float lds[L < 64 ? 1 : L / 64][1];
  const int j = threadIdx.x % L;
  const int strips = a.d / kN;
  const int64_t r = static_cast<int64_t>(blockIdx.x) * kRows + threadIdx.x / L;
  const bool live = r < a.rows;
  float v[S][kN];
  load_row<T, L, S>(v, static_cast<const T*>(a.x) + (live ? r : 0) * a.x_pitch, j, strips, live);
  const float inv = 1.0f / static_cast<float>(a.d);
  float sum[1] = {0.0f};
  if (a.mean != nullptr) {
    sum[0] = strip_sum<S, kN>([&](int s, int e) { return v[s][e]; });
    row_sums<L>(sum, lds);
    sum[0] *= inv;
  }
  const float mean = sum[0];
#pragma unroll
  for (int s = 0; s < S; ++s)
#pragma unroll
    for (int e = 0; e < kN; ++e) v[s][e] = j + L * s < strips ? v[s][e] - mean : 0.0f;
  sum[0] = strip_sum<S, kN>([&](int s, int e) { return v[s][e] * v[s][e]; });
  row_sums<L>(sum, lds);
  const float rstd = 1.0f / sqrtf(sum[0] * inv + a.eps);
  if (!live) return;
  if (j == 0) {
    if (a.mean != nullptr) a.mean[r] = mean;
    a.rstd[r] = rstd;
  }
#pragma unroll
  for (int s = 0; s < S; ++s) {
    const int at = (j + L * s) * kN;
    if (j + L * s >= strips) continue;
    float y[kN];
#pragma unroll
    for (int e = 0; e < kN; ++e) y[e] = v[s][e] * rstd;
    if (a.weight != nullptr) {
      const auto w = Strip<T>::load(static_cast<const T*>(a.weight) + at);
#pragma unroll
      for (int e = 0; e < kN; ++e) y[e] *= static_cast<float>(w[e]);
    }
    if (a.bias != nullptr) {
      const auto b = Strip<T>::load(static_cast<const T*>(a.bias) + at);
#pragma unroll
      for (int e = 0; e < kN; ++e) y[e] += static_cast<float>(b[e]);
    }
    Strip<T>::store(static_cast<T*>(a.out) + r * a.d + at, y);
  }
}

// Rows r, r + step, .. of each group of L lanes.
template <typename T, int L, int S>
__global__ __launch_bounds__(L < 256 ? 256 : L) void k_norm_bwd(NormArgs a) {
  constexpr int kN = Strip<T>::kN, kRows = L < 256 ? 256 / L : 1;
  __shared__ float lds[L < 64 ? 1 : L / 64][2];
  const int j = threadIdx.x % L;
  const int strips = a.d / kN;
  const float inv = 1.0f / static_cast<float>(a.d);
  const bool center = a.mean != nullptr;
  // A workgroup of 1024 has no registers to hold the weight from row to row.
  constexpr bool kHold = L < 1024;
  float w[S][kN], dw[S][kN], db[S][kN];
  auto load_weight = [&] {
    if (a.weight != nullptr) {
      load_row<T, L, S>(w, static_cast<const T*>(a.weight), j, strips, true);
      return;
    }
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int e = 0; e < kN; ++e) w[s][e] = 1.0f;
  };
  if constexpr (kHold) load_weight();
#pragma unroll
  for (int s = 0; s < S; ++s)
#pragma unroll
    for (int e = 0; e < kN; ++e) dw[s][e] = db[s][e] = 0.0f;
  // The same number of turns for every group: the sums of a workgroup's row meet at
  // barriers.
  const int64_t step = static_cast<int64_t>(gridDim.x) * kRows;
  for (int64_t r0 = static_cast<int64_t>(blockIdx.x) * kRows; r0 < a.rows; r0 += step) {
    const int64_t r = r0 + threadIdx.x / L;
    const bool live = r < a.rows;
    float h[S][kN], g[S][kN];
    load_row<T, L, S>(h, static_cast<const T*>(a.x) + (live ? r : 0) * a.x_pitch, j, strips, live);
    load_row<T, L, S>(g, static_cast<const T*>(a.dy) + (live ? r : 0) * a.dy_pitch, j, strips, live);
    const float mean = live && center ? a.mean[r] : 0.0f;
    const float rstd = live ? a.rstd[r] : 0.0f;
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int e = 0; e < kN; ++e) {
        h[s][e] = (h[s][e] - mean) * rstd;
        dw[s][e] += g[s][e] * h[s][e];
        db[s][e] += g[s][e];
      }
    if (a.out == nullptr) continue;
    if constexpr (!kHold) load_weight();
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int e = 0; e < kN; ++e) g[s][e] *= w[s][e];
    float sum[2];
    sum[0] = strip_sum<S, kN>([&](int s, int e) { return g[s][e]; });
    sum[1] = strip_sum<S, kN>([&](int s, int e) { return g[s][e] * h[s][e]; });
    row_sums<L>(sum, lds);
    const float c0 = center ? sum[0] * inv : 0.0f, c1 = sum[1] * inv;
    if (!live) continue;
#pragma unroll
    for (int s = 0; s < S; ++s) {
      if (j + L * s >= strips) continue;
      float y[kN];
#pragma unroll
      for (int e = 0; e < kN; ++e) y[e] = rstd * (g[s][e] - c0 - h[s][e] * c1);
      Strip<T>::store(static_cast<T*>(a.out) + r * a.d + (j + L * s) * kN, y);
    }
  }
  if (a.dweight == nullptr && a.dbias == nullptr) return;
  if constexpr (L < 64) {
    // The groups of a wavefront first: lanes of one column.
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int e = 0; e < kN; ++e) {
#pragma unroll
        for (int o = L; o < 64; o *= 2) {
          dw[s][e] += __shfl_xor(dw[s][e], o);
          db[s][e] += __shfl_xor(db[s][e], o);
        }
      }
  }
  float* const out = a.part + static_cast<int64_t>(blockIdx.x) * 2 * a.d;
  if constexpr (L <= 64) {
    // The workgroup's four wavefronts.
    __shared__ __attribute__((aligned(16))) float sums[4][2][L * S * kN];
    const int wave = threadIdx.x / 64;
    if (threadIdx.x % 64 < L) {
#pragma unroll
      for (int s = 0; s < S; ++s)
#pragma unroll
        for (int e = 0; e < kN; ++e) {
          sums[wave][0][(j + L * s) * kN + e] = dw[s][e];
          sums[wave][1][(j + L * s) * kN + e] = db[s][e];
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * a.d; i += 256) {
      const int k = i < a.d ? 0 : 1, c = i - k * a.d;
      out[i] = (sums[0][k][c] + sums[1][k][c]) + (sums[2][k][c] + sums[3][k][c]);
    }
  } else {
#pragma unroll
    for (int s = 0; s < S; ++s) {
      if (j + L * s >= strips) continue;
#pragma unroll
      for (int e = 0; e < kN; e += 4) {
        const int at = (j + L * s) * kN + e;
        *reinterpret_cast<f32x4*>(out + at) =
            f32x4{dw[s][e], dw[s][e + 1], dw[s][e + 2], dw[s][e + 3]};
        *reinterpret_cast<f32x4*>(out + a.d + at) =
            f32x4{db[s][e], db[s][e + 1], db[s][e + 2], db[s][e + 3]};
      }
    }
  }
}

// Columns over the groups: 32 lanes take a column each, the workgroup's 32 halves of
// wavefronts a share of the groups.  blockIdx.y: dweight, dbias.
constexpr int kJoinCols = 32;
constexpr int kJoinShares = 32;
template <typename T>
__global__ __launch_bounds__(kJoinCols* kJoinShares) void k_norm_join(NormArgs a) {
  __shared__ float lds[kJoinShares][kJoinCols];
  const int lane = threadIdx.x % kJoinCols, share = threadIdx.x / kJoinCols;
  const int c = blockIdx.x * kJoinCols + lane;
  void* const to = blockIdx.y == 0 ? a.dweight : a.dbias;
  if (to == nullptr) return;
  float sum = 0.0f;
  if (c < a.d) {
    const float* p = a.part + blockIdx.y * static_cast<int64_t>(a.d) + c;
#pragma unroll 16
    for (int i = share; i < a.groups; i += kJoinShares) sum += p[static_cast<int64_t>(i) * 2 * a.d];
  }
  lds[share][lane] = sum;
  __syncthreads();
#pragma unroll
  for (int s = kJoinShares / 2; s > 0; s /= 2) {
    if (share < s) lds[share][lane] += lds[share + s][lane];
    __syncthreads();
  }
  if (share == 0 && c < a.d) static_cast<T*>(to)[c] = static_cast<T>(lds[0][lane]);
}

}  // namespace smx
