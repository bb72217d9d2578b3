// C ABI of the norms of rows: argument checks, workspace and launches.
// Declarations and contract: include/decoder_mi355x.h.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "sm_decoder_host.hpp"
#include "sm_norm.hpp"

namespace {

using namespace smx;
using namespace smx_host;

constexpr int64_t kMostThreads = int64_t(1) << 31;  // of a launch

struct Shape {
  const void* fn;
  int lanes;
};

// The instance for rows of `strips` strips: lanes that hold a row, and strips of
// each lane.
template <bool BACK, typename T, int L, int S>
Shape instance() {
  if constexpr (BACK) return {reinterpret_cast<const void*>(&k_norm_bwd<T, L, S>), L};
  else return {reinterpret_cast<const void*>(&k_norm_fwd<T, L, S>), L};
}

// Rows of more than 8192 columns of fp32; those of 16-bit types have no more than
// 2048 strips.
template <bool BACK, typename T>
Shape wide() {
  if constexpr (sizeof(T) == 4) return instance<BACK, T, 1024, 4>();
  else return instance<BACK, T, 1024, 2>();
}

// Forward: a wavefront holds up to four strips per lane, a workgroup takes longer rows
// (16384 x 4096 of bf16: 64 us with a wavefront and eight strips per lane, 50 with 256
// threads and two), and rows that are too few to fill the device with a wavefront each.
template <typename T>
Shape forward_of(int64_t strips, int64_t rows) {
  constexpr bool B = false;
  if (strips <= 8) return instance<B, T, 8, 1>();
  if (strips <= 16) return instance<B, T, 16, 1>();
  if (strips <= 32) return instance<B, T, 32, 1>();
  if (strips <= 64) return instance<B, T, 64, 1>();
  if (rows > 1024 && strips <= 256) {
    if (strips <= 128) return instance<B, T, 64, 2>();
    return instance<B, T, 64, 4>();
  }
  if (strips <= 256) return instance<B, T, 256, 1>();
  if (strips <= 512) return instance<B, T, 256, 2>();
  if (strips <= 1024) return instance<B, T, 256, 4>();
  if (sizeof(T) == 2 || strips <= 2048) return instance<B, T, 1024, 2>();
  return wide<B, T>();
}

// Backward: x, dy, the weight and the sums of two columns' gradients are in
// registers, so a lane holds fewer strips.
template <typename T>
Shape backward_of(int64_t strips) {
  constexpr bool B = true;
  if (strips <= 8) return instance<B, T, 8, 1>();
  if (strips <= 16) return instance<B, T, 16, 1>();
  if (strips <= 32) return instance<B, T, 32, 1>();
  if (strips <= 64) return instance<B, T, 64, 1>();
  if (strips <= 128) return instance<B, T, 64, 2>();
  if (strips <= 256) return instance<B, T, 256, 1>();
  if (strips <= 512) return instance<B, T, 256, 2>();
  if (strips <= 1024) return instance<B, T, 1024, 1>();
  if (sizeof(T) == 2 || strips <= 2048) return instance<B, T, 1024, 2>();
  return wide<B, T>();
}

Shape forward_shape(int dtype, int64_t strips, int64_t rows) {
  return dtype == SOFTMAX_F32   ? forward_of<float>(strips, rows)
         : dtype == SOFTMAX_F16 ? forward_of<f16>(strips, rows) : forward_of<bf16>(strips, rows);
}
Shape backward_shape(int dtype, int64_t strips) {
  return dtype == SOFTMAX_F32   ? backward_of<float>(strips)
         : dtype == SOFTMAX_F16 ? backward_of<f16>(strips) : backward_of<bf16>(strips);
}

// The backward pass' workgroups, each of which leaves a row of sums: a fixed number
// whatever the device, since the order of the sums goes by it.
int64_t groups_of(int lanes, int64_t rows) {
  return std::min<int64_t>(ceil_div(rows, lanes < 256 ? 256 / lanes : 1), lanes == 1024 ? 512 : 1024);
}

bool sizes_ok(int64_t rows, int64_t d, int dtype) {
  return dtype_size(dtype) != 0 && count_ok(rows) && width_ok(d);
}

int64_t strips_of(int64_t d, int dtype) { return d * dtype_size(dtype) / 16; }

}  // namespace

extern "C" {

SOFTMAX_API int softmax_layer_norm_fwd(const void* x, int64_t x_stride, const void* weight,
                                       const void* bias, int64_t rows, int64_t d, float eps,
                                       int center, int dtype, void* y, float* mean, float* rstd,
                                       hipStream_t stream) {
  const int size = dtype_size(dtype);
  int64_t xb = 0;
  if (!sizes_ok(rows, d, dtype) || x_stride < 0 || !rows_ok(x, rows, x_stride, d, size, &xb) ||
      !std::isfinite(eps) || eps < 0.0f || (center != 0 && center != 1) || !aligned16(y) ||
      !aligned16(weight) || !aligned16(bias) || (center == 0 && mean != nullptr))
    return SOFTMAX_ERR_INVALID_ARG;
  if (rows == 0) return SOFTMAX_OK;
  const Range inputs[] = {{x, xb}, {weight, weight ? d * size : 0}, {bias, bias ? d * size : 0}};
  const Range outputs[] = {{y, rows * d * size}, {mean, center ? rows * 4 : 0}, {rstd, rows * 4}};
  const int rc = check_ranges(inputs, outputs);
  if (rc != SOFTMAX_OK) return rc;
  NormArgs a = {};
  a.x_pitch = x_stride;
  a.weight = weight;
  a.bias = bias;
  a.d = static_cast<int>(d);
  a.eps = eps;
  const Shape s = forward_shape(dtype, strips_of(d, dtype), rows);
  const int threads = std::max(s.lanes, 256);
  const int64_t each = threads / s.lanes;
  // A launch takes fewer than 2^32 threads.
  const int64_t most = kMostThreads / threads * each;
  hipError_t e = hipSuccess;
  for (int64_t from = 0; from < rows && e == hipSuccess; from += most) {
    const int64_t some = std::min(rows - from, most);
    a.x = static_cast<const char*>(x) + from * x_stride * size;
    a.out = static_cast<char*>(y) + from * d * size;
    a.mean = mean == nullptr ? nullptr : mean + from;
    a.rstd = rstd + from;
    a.rows = static_cast<int>(some);
    void* args[] = {&a};
    e = launch(s.fn, ceil_div(some, each), threads, args, stream);
  }
  return e == hipSuccess ? SOFTMAX_OK : fail_hip(e);
}

SOFTMAX_API int64_t softmax_layer_norm_bwd_workspace(int64_t rows, int64_t d, int dtype) {
  if (!sizes_ok(rows, d, dtype)) return -1;
  return groups_of(backward_shape(dtype, strips_of(d, dtype)).lanes, rows) * 2 * d * 4;
}

SOFTMAX_API int softmax_layer_norm_bwd(const void* dy, int64_t dy_stride, const void* x,
                                       int64_t x_stride, const void* weight, const float* mean,
                                       const float* rstd, int64_t rows, int64_t d, int dtype,
                                       void* dx, void* dweight, void* dbias, void* workspace,
                                       int64_t workspace_bytes, hipStream_t stream) {
  const int size = dtype_size(dtype);
  int64_t xb = 0, db = 0;
  if (!sizes_ok(rows, d, dtype) || x_stride < 0 || dy_stride < 0 ||
      !rows_ok(x, rows, x_stride, d, size, &xb) || !rows_ok(dy, rows, dy_stride, d, size, &db) ||
      !aligned16(weight) || !aligned16(dx) || !aligned16(workspace))
    return SOFTMAX_ERR_INVALID_ARG;
  const bool columns = dweight != nullptr || dbias != nullptr;
  if (!columns && (dx == nullptr || rows == 0)) return SOFTMAX_OK;
  const Shape s = backward_shape(dtype, strips_of(d, dtype));
  const int64_t groups = groups_of(s.lanes, rows);
  const int64_t need = columns ? groups * 2 * d * 4 : 0;
  if (workspace_bytes < need) return SOFTMAX_ERR_INVALID_ARG;
  const Range inputs[] = {{x, xb},
                          {dy, db},
                          {weight, weight ? d * size : 0},
                          {mean, mean ? rows * 4 : 0},
                          {rstd, rows * 4}};
  const Range outputs[] = {{dx, dx ? rows * d * size : 0},
                           {dweight, dweight ? d * size : 0},
                           {dbias, dbias ? d * size : 0},
                           {workspace, need}};
  const int rc = check_ranges(inputs, outputs);
  if (rc != SOFTMAX_OK) return rc;
  NormArgs a = {};
  a.x = x;
  a.x_pitch = x_stride;
  a.dy = dy;
  a.dy_pitch = dy_stride;
  a.weight = weight;
  a.out = dx;
  a.mean = const_cast<float*>(mean);
  a.rstd = const_cast<float*>(rstd);
  a.dweight = dweight;
  a.dbias = dbias;
  a.part = static_cast<float*>(workspace);
  a.rows = static_cast<int>(rows);
  a.d = static_cast<int>(d);
  a.groups = static_cast<int>(groups);
  void* args[] = {&a};
  hipError_t e = hipSuccess;
  if (rows > 0)
    e = launch(s.fn, groups, std::max(s.lanes, 256), args, stream);
  if (e == hipSuccess && columns) {
    const void* fn = dtype == SOFTMAX_F32   ? reinterpret_cast<const void*>(&k_norm_join<float>)
                     : dtype == SOFTMAX_F16 ? reinterpret_cast<const void*>(&k_norm_join<f16>)
                                            : reinterpret_cast<const void*>(&k_norm_join<bf16>);
    e = hipLaunchKernel(fn, dim3(static_cast<uint32_t>(ceil_div(d, kJoinCols)), 2),
                        dim3(kJoinCols * kJoinShares), args, 0, stream);
  }
  return e == hipSuccess ? SOFTMAX_OK : fail_hip(e);
}

}  // extern "C"
