// Multi-head attention with all products on the fp32 matrix cores.
//
// v_mfma_f32_16x16x4f32 takes A[16][4] and B[4][16]: lane l holds A at row
// l % 16, column l / 16, B at row l / 16, column l % 16, and D at column
// l % 16, rows 4 (l / 16) + i.  With scores transposed, S^T = K Q^T, a lane
// holds one query's scores of the keys 4 (l / 16) + i: the softmax is
// lane-local but for two exchanges, and S^T register i is the B operand of
// the value product O^T += V^T P^T at the keys {i, 4 + i, 8 + i, 12 + i},
// without a move.  The gradients work the same way: with S^T and dP^T = V
// dO^T, dQ^T += K^T dS^T; with keys as columns, S = Q K^T and dP = dO V^T,
// dV^T += dO^T P and dK^T += Q^T dS.
//
// A workgroup of four wavefronts takes 64 rows (16 each, operands in
// registers) against tiles of 32 keys (or 64 keys against tiles of 32 rows),
// staged as fp32 in LDS, whose rows are 4 floats longer than a row so that 16
// rows read at one column spread over the banks.  Bound by latency: a tile's product
// is one chain of dependent matrix ops.  4096 tokens of one document (16 heads of
// 128 on 4) take 0.81 ms forward, 85 of the 154 TFLOP/s that a large product
// reaches, and 4.7 ms back, 51; 64 single tokens over up to 8192 keys (32 heads on
// 8) 1.4 ms, 1.6 TB/s, since three of four wavefronts have no row; 101 tokens of
// four heads of 80 in short documents 9 us forward and 26 us back, a few tiles'
// latency each.
#pragma once

#include "sm_heads.hpp"

namespace smx {

constexpr int kF32Rows = 64;   // rows (or keys) of a workgroup
constexpr int kF32Step = 32;   // keys (or rows) of a staged tile
constexpr int kF32Threads = 256;

__device__ __forceinline__ f32x4 load4(const float* p) {
  return *reinterpret_cast<const f32x4*>(p);
}

template <typename T>
__device__ __forceinline__ void store4(T* p, f32x4 v) {
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<f32x4*>(p) = v;
  } else {
    typedef T t4 __attribute__((ext_vector_type(4)));
    *reinterpret_cast<t4*>(p) = t4{static_cast<T>(v[0]), static_cast<T>(v[1]),
                                   static_cast<T>(v[2]), static_cast<T>(v[3])};
  }
}

__device__ __forceinline__ f32x4 mfma4(float a, float b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

// The score of a dot product, and the derivative of its cap.
__device__ __forceinline__ float score_f32(const HeadsArgs& a, float dot, float slope, int dist,
                                           float* dcap) {
  float x = dot * a.scale;
  *dcap = 1.0f;
  if (a.cap > 0.0f) {
    const float t = tanhf(x / a.cap);
    x = a.cap * t;
    *dcap = 1.0f - t * t;
  }
  return x - slope * static_cast<float>(abs(dist));
}

// One row (of 16) of a register operand: element 4 t + j of the lane is
// column 16 t + 4 (l / 16) + j of the row, 0 past d.
template <int DP>
__device__ __forceinline__ void load_row(f32x4 (&r)[DP / 16], const float* row, bool valid, int g,
                                         int d) {
#pragma unroll
  for (int t = 0; t < DP / 16; ++t) {
    const int c = 16 * t + 4 * g;
    r[t] = valid && c < d ? load4(row + c) : f32x4{0, 0, 0, 0};
  }
}

// Rows of a staged tile against the lane's row: D[row of the tile][lane row].
template <int DP>
__device__ __forceinline__ f32x4 tile_dot(const float (*tile)[DP + 4], int row0,
                                          const f32x4 (&r)[DP / 16], int c, int g) {
  f32x4 s = {0, 0, 0, 0};
#pragma unroll
  for (int t = 0; t < DP / 16; ++t) {
    const f32x4 x = *reinterpret_cast<const f32x4*>(&tile[row0 + c][16 * t + 4 * g]);
#pragma unroll
    for (int j = 0; j < 4; ++j) s = mfma4(x[j], r[t][j], s);
  }
  return s;
}

// acc[column of the tile][lane row] += tile^T w, for the tile's rows row0 +
// 4 (l / 16) + i with the weights w[i].
template <int DP>
__device__ __forceinline__ void tile_accumulate(f32x4 (&acc)[DP / 16],
                                                const float (*tile)[DP + 4], int row0, f32x4 w,
                                                int c, int g) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int t = 0; t < DP / 16; ++t)
      acc[t] = mfma4(tile[row0 + 4 * g + i][16 * t + c], w[i], acc[t]);
  }
}

// A thread's share of the next tile's two tensors, loaded into registers
// during the products of this one: f(row, column, x, y) loads four columns
// of one row of each.
template <int DP>
struct NextTile {
  static constexpr int kShare = kF32Step * DP / 4 / kF32Threads;
  f32x4 x[kShare], y[kShare];

  template <typename F>
  __device__ __forceinline__ void load(F f) {
#pragma unroll
    for (int n = 0; n < kShare; ++n) {
      const int i = static_cast<int>(threadIdx.x) + n * kF32Threads;
      x[n] = y[n] = f32x4{0, 0, 0, 0};
      f(i / (DP / 4), 4 * (i % (DP / 4)), x[n], y[n]);
    }
  }
  __device__ __forceinline__ void store(float (*xs)[DP + 4], float (*ys)[DP + 4]) const {
#pragma unroll
    for (int n = 0; n < kShare; ++n) {
      const int i = static_cast<int>(threadIdx.x) + n * kF32Threads;
      *reinterpret_cast<f32x4*>(&xs[i / (DP / 4)][4 * (i % (DP / 4))]) = x[n];
      *reinterpret_cast<f32x4*>(&ys[i / (DP / 4)][4 * (i % (DP / 4))]) = y[n];
    }
  }
};

template <int DP, bool PAGED>
__global__ __launch_bounds__(kF32Threads) void k_heads_fwd_f32(HeadsArgs a) {
  __shared__ __attribute__((aligned(16))) float ks[kF32Step][DP + 4];
  __shared__ __attribute__((aligned(16))) float vs[kF32Step][DP + 4];
  __shared__ int held[kF32Step];
  const int hk = blockIdx.x % a.kv_heads;
  const int slot = static_cast<int>(gridDim.x / a.kv_heads - 1 - blockIdx.x / a.kv_heads);
  const int split = blockIdx.y;
  const DocLanes docs = load_docs<PAGED>(a, threadIdx.x % 64);
  const int chunk = PAGED ? split_chunk<kF32Rows>(a, docs) : 0;
  const DocTile w = find_tile<kF32Rows, PAGED, false>(a, docs, slot);
  const int rows = w.lq * a.group;
  if (w.tile * kF32Rows >= rows) return;

  const int tid = threadIdx.x, wave = tid / 64, lane = tid % 64;
  const int c = lane % 16, g = lane / 16;
  const int row = w.tile * kF32Rows + 16 * wave + c;
  const bool valid = row < rows;
  const int tok = valid ? row / a.group : w.lq - 1;
  const int head = hk * a.group + (valid ? row % a.group : 0);
  const int pos = tok + w.lk - w.lq;
  const int lim = valid ? keys_seen(a, w, tok) : 0;
  const int last_tok = (min(rows, (w.tile + 1) * kF32Rows) - 1) / a.group;
  const int seen = keys_seen(a, w, last_tok);
  int from, to;
  if (!split_range(seen, chunk, split, &from, &to)) return;
  const float slope = a.slopes != nullptr ? a.slopes[head] : 0.0f;
  const int64_t token = w.q0 + tok;

  f32x4 q[DP / 16];
  load_row<DP>(q, static_cast<const float*>(a.q.data) + token * a.q.ts + head * a.q.hs, valid, g,
                  a.d);
  f32x4 acc[DP / 16] = {};
  float m = -INFINITY, l = 0.0f;

  NextTile<DP> next;
  auto load = [&](int k0) {
    next.load([&](int r, int col, f32x4& x, f32x4& y) {
      const int j = k0 + r;
      if (j >= to || col >= a.d) return;
      int64_t kr, vr;
      if constexpr (PAGED) {
        kr = paged_row(a, w.b, j, a.k_bs, a.k.ts);
        vr = paged_row(a, w.b, j, a.v_bs, a.v.ts);
        if (kr < 0) return;
      } else {
        kr = static_cast<int64_t>(w.k0 + j) * a.k.ts;
        vr = static_cast<int64_t>(w.k0 + j) * a.v.ts;
      }
      x = load4(static_cast<const float*>(a.k.data) + kr + hk * a.k.hs + col);
      y = load4(static_cast<const float*>(a.v.data) + vr + hk * a.v.hs + col);
    });
  };
  load(from);
  for (int k0 = from; k0 < to; k0 += kF32Step) {
    __syncthreads();
    next.store(ks, vs);
    if (PAGED && tid < kF32Step)
      held[tid] = k0 + tid < to && paged_row(a, w.b, k0 + tid, a.k_bs, a.k.ts) >= 0;
    __syncthreads();
    load(k0 + kF32Step);
    f32x4 s[2];
    float top = -INFINITY;
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      s[kt] = tile_dot<DP>(ks, 16 * kt, q, c, g);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = 16 * kt + 4 * g + i, j = k0 + r;
        float dcap;
        const float x = score_f32(a, s[kt][i], slope, pos - j, &dcap);
        s[kt][i] = j < lim && (!PAGED || held[r]) ? x : -INFINITY;
        top = fmaxf(top, s[kt][i]);
      }
    }
    const float next = fmaxf(m, group4_max(top));
    const float base = next == -INFINITY ? 0.0f : next;
    const float alpha = __builtin_amdgcn_exp2f((m - base) * kLog2eF);
    m = next;
    float part = 0.0f;
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        // The argument's rounding is 2^-24 of it: 1e-6 of a weight of e^-16.
        s[kt][i] = __builtin_amdgcn_exp2f((s[kt][i] - base) * kLog2eF);
        part += s[kt][i];
      }
    }
    l = l * alpha + group4_sum(part);
#pragma unroll
    for (int t = 0; t < DP / 16; ++t) acc[t] *= alpha;
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) tile_accumulate<DP>(acc, vs, 16 * kt, s[kt], c, g);
  }

  if (!valid) return;
  const int64_t out = token * a.heads + head;
  if (chunk > 0) {
    const int64_t at = split * static_cast<int64_t>(a.tokens_q) * a.heads + out;
    if (g == 0) a.part_stat[at] = {m, l, split_count(seen, chunk), 0};
#pragma unroll
    for (int t = 0; t < DP / 16; ++t)
      if (16 * t + 4 * g < a.d)
        *reinterpret_cast<f32x4*>(a.part_o + at * a.d + 16 * t + 4 * g) = acc[t];
    return;
  }
  const float inv = m == -INFINITY ? 0.0f : 1.0f / l;
  if (g == 0 && a.lse != nullptr)
    a.lse[out] = m == -INFINITY ? lse_of_none(l) : m + __builtin_amdgcn_logf(l) * kLn2F;
#pragma unroll
  for (int t = 0; t < DP / 16; ++t)
    if (16 * t + 4 * g < a.d)
      store4(static_cast<float*>(a.out) + out * a.d + 16 * t + 4 * g, acc[t] * inv);
}

// D of every row and the gradient of the queries.
template <int DP>
__global__ __launch_bounds__(kF32Threads) void k_heads_dq_f32(HeadsArgs a) {
  __shared__ __attribute__((aligned(16))) float ks[kF32Step][DP + 4];
  __shared__ __attribute__((aligned(16))) float vs[kF32Step][DP + 4];
  const int hk = blockIdx.x % a.kv_heads;
  const int slot = static_cast<int>(gridDim.x / a.kv_heads - 1 - blockIdx.x / a.kv_heads);
  const DocTile w =
      find_tile<kF32Rows, false, false>(a, load_docs<false>(a, threadIdx.x % 64), slot);
  const int rows = w.lq * a.group;
  if (w.tile * kF32Rows >= rows) return;

  const int tid = threadIdx.x, wave = tid / 64, lane = tid % 64;
  const int c = lane % 16, g = lane / 16;
  const int row = w.tile * kF32Rows + 16 * wave + c;
  const bool valid = row < rows;
  const int tok = valid ? row / a.group : w.lq - 1;
  const int head = hk * a.group + (valid ? row % a.group : 0);
  const int pos = tok + w.lk - w.lq;
  const int lim = valid ? keys_seen(a, w, tok) : 0;
  const int to = keys_seen(a, w, (min(rows, (w.tile + 1) * kF32Rows) - 1) / a.group);
  const float slope = a.slopes != nullptr ? a.slopes[head] : 0.0f;
  const int64_t token = w.q0 + tok, out = token * a.heads + head;

  f32x4 q[DP / 16], dout[DP / 16];
  load_row<DP>(q, static_cast<const float*>(a.q.data) + token * a.q.ts + head * a.q.hs, valid, g,
                  a.d);
  load_row<DP>(dout, static_cast<const float*>(a.dout.data) + token * a.dout.ts + head * a.dout.hs,
                  valid, g, a.d);
  float delta = 0.0f;
  {
    f32x4 o[DP / 16];
    load_row<DP>(o, static_cast<const float*>(a.o.data) + token * a.o.ts + head * a.o.hs, valid, g,
                    a.d);
#pragma unroll
    for (int t = 0; t < DP / 16; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) delta = __builtin_fmaf(o[t][j], dout[t][j], delta);
    delta = group4_sum(delta);
  }
  const float lse = valid ? a.lse[out] : 0.0f;
  if (valid && g == 0) a.delta[out] = delta;
  f32x4 acc[DP / 16] = {};

  NextTile<DP> next;
  auto load = [&](int k0) {
    next.load([&](int r, int col, f32x4& x, f32x4& y) {
      if (k0 + r >= to || col >= a.d) return;
      const int64_t at = w.k0 + k0 + r;
      x = load4(static_cast<const float*>(a.k.data) + at * a.k.ts + hk * a.k.hs + col);
      y = load4(static_cast<const float*>(a.v.data) + at * a.v.ts + hk * a.v.hs + col);
    });
  };
  load(0);
  for (int k0 = 0; k0 < to; k0 += kF32Step) {
    __syncthreads();
    next.store(ks, vs);
    __syncthreads();
    load(k0 + kF32Step);
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      const f32x4 s = tile_dot<DP>(ks, 16 * kt, q, c, g);
      const f32x4 dp = tile_dot<DP>(vs, 16 * kt, dout, c, g);
      f32x4 ds;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int j = k0 + 16 * kt + 4 * g + i;
        float dcap;
        const float x = score_f32(a, s[i], slope, pos - j, &dcap);
        const float p = j < lim ? __builtin_amdgcn_exp2f((x - lse) * kLog2eF) : 0.0f;
        ds[i] = j < lim ? p * (dp[i] - delta) * dcap : 0.0f;
      }
      tile_accumulate<DP>(acc, ks, 16 * kt, ds, c, g);
    }
  }
  if (!valid) return;
#pragma unroll
  for (int t = 0; t < DP / 16; ++t)
    if (16 * t + 4 * g < a.d)
      store4(static_cast<float*>(a.out) + out * a.d + 16 * t + 4 * g, acc[t] * a.scale);
}

// The gradients of the keys and values: 64 keys per workgroup, against the
// rows of their document that see any of them.
template <int DP>
__global__ __launch_bounds__(kF32Threads) void k_heads_dkv_f32(HeadsArgs a) {
  __shared__ __attribute__((aligned(16))) float qs[kF32Step][DP + 4];
  __shared__ __attribute__((aligned(16))) float os[kF32Step][DP + 4];
  __shared__ float row_lse[kF32Step], row_delta[kF32Step], row_slope[kF32Step];
  const int hk = blockIdx.x % a.kv_heads;
  const DocTile w = find_tile<kF32Rows, false, true>(a, load_docs<false>(a, threadIdx.x % 64),
                                                     blockIdx.x / a.kv_heads);
  if (w.tile * kF32Rows >= w.lk) return;

  const int tid = threadIdx.x, wave = tid / 64, lane = tid % 64;
  const int c = lane % 16, g = lane / 16;
  const int first = w.tile * kF32Rows;
  const int key = first + 16 * wave + c;
  const bool valid = key < w.lk;
  const int64_t token = w.k0 + key;

  f32x4 k[DP / 16], v[DP / 16];
  load_row<DP>(k, static_cast<const float*>(a.k.data) + token * a.k.ts + hk * a.k.hs, valid, g,
                  a.d);
  load_row<DP>(v, static_cast<const float*>(a.v.data) + token * a.v.ts + hk * a.v.hs, valid, g,
                  a.d);
  f32x4 dk[DP / 16] = {}, dv[DP / 16] = {};

  // The first token that sees the tile's first key.
  const int tok0 = a.causal && first >= w.prefix ? max(first - (w.lk - w.lq), 0) : 0;
  const int rows = w.lq * a.group;
  NextTile<DP> next;
  float lse = 0.0f, delta = 0.0f, slope = 0.0f;  // of row r0 + tid
  auto load = [&](int r0) {
    next.load([&](int r, int col, f32x4& x, f32x4& y) {
      const int row = r0 + r;
      if (row >= rows || col >= a.d) return;
      const int64_t at = w.q0 + row / a.group;
      const int head = hk * a.group + row % a.group;
      x = load4(static_cast<const float*>(a.q.data) + at * a.q.ts + head * a.q.hs + col);
      y = load4(static_cast<const float*>(a.dout.data) + at * a.dout.ts + head * a.dout.hs + col);
    });
    const int row = r0 + tid;
    if (tid < kF32Step && row < rows) {
      const int head = hk * a.group + row % a.group;
      const int64_t at = static_cast<int64_t>(w.q0 + row / a.group) * a.heads + head;
      lse = a.lse[at];
      delta = a.delta[at];
      if (a.slopes != nullptr) slope = a.slopes[head];
    }
  };
  load(tok0 * a.group);
  for (int r0 = tok0 * a.group; r0 < rows; r0 += kF32Step) {
    __syncthreads();
    next.store(qs, os);
    if (tid < kF32Step) {
      row_lse[tid] = lse;
      row_delta[tid] = delta;
      row_slope[tid] = slope;
    }
    __syncthreads();
    load(r0 + kF32Step);
#pragma unroll
    for (int qt = 0; qt < 2; ++qt) {
      const f32x4 s = tile_dot<DP>(qs, 16 * qt, k, c, g);
      const f32x4 dp = tile_dot<DP>(os, 16 * qt, v, c, g);
      f32x4 p, ds;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = 16 * qt + 4 * g + i, row = r0 + r;
        const int tok = row / a.group;
        const bool seen = valid && row < rows && key < keys_seen(a, w, tok);
        float dcap;
        const float x = score_f32(a, s[i], row_slope[r], tok + w.lk - w.lq - key, &dcap);
        p[i] = seen ? __builtin_amdgcn_exp2f((x - row_lse[r]) * kLog2eF) : 0.0f;
        ds[i] = seen ? p[i] * (dp[i] - row_delta[r]) * dcap : 0.0f;
      }
      tile_accumulate<DP>(dv, os, 16 * qt, p, c, g);
      tile_accumulate<DP>(dk, qs, 16 * qt, ds, c, g);
    }
  }
  if (!valid) return;
  const int64_t out = (token * a.kv_heads + hk) * a.d;
#pragma unroll
  for (int t = 0; t < DP / 16; ++t) {
    const int col = 16 * t + 4 * g;
    if (col < a.d) {
      store4(static_cast<float*>(a.dk) + out + col, dk[t] * a.scale);
      store4(static_cast<float*>(a.dv) + out + col, dv[t]);
    }
  }
}

// Joins the splits of a row, one wavefront each, its lanes over the splits'
// statistics and then over the columns (up to 128 of them twice, for two splits
// at a time).  One token over 4001 keys (32 heads of 128, 16 splits) 6 us, mostly
// the launch and one load behind another; 2048 rows of 16 heads in up to eight
// splits 21 us, at memory's rate.
template <typename T>
__device__ __forceinline__ void join_row(const HeadsArgs& a, int64_t rows, int64_t row, int lane,
                                         SplitStat mine) {
  // Sums that do not ascend leave rows that no workgroup wrote: what their
  // places hold is no number of splits.
  const int count = clamp_i(__builtin_amdgcn_readfirstlane(mine.count), 0, a.splits);
  if (lane >= count) mine = {-INFINITY, 0.0f, 0, 0};
  const float m = seg_max<64>(mine.m);
  const float weight = __builtin_amdgcn_exp2f((mine.m - (m == -INFINITY ? 0.0f : m)) * kLog2eF);
  const float l = seg_sum<64>(mine.l * weight);
  const int pair = a.d <= 128 ? lane / 32 : 0, step = a.d <= 128 ? 2 : 1;
  const int col = 4 * (a.d <= 128 ? lane % 32 : lane);
  f32x4 acc = {0, 0, 0, 0};
  for (int s = 0; s < count; s += step) {
    const int at = s + pair;
    const float f = __shfl(weight, at);
    if (at < count && col < a.d)
      acc += *reinterpret_cast<const f32x4*>(a.part_o + (at * rows + row) * a.d + col) * f;
  }
  if (step == 2)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] += half32_partner(acc[j]);
  const float inv = m == -INFINITY ? 0.0f : 1.0f / l;
  if (lane == 0 && a.lse != nullptr)
    a.lse[row] = m == -INFINITY ? lse_of_none(l) : m + __builtin_amdgcn_logf(l) * kLn2F;
  if (pair == 0 && col < a.d) store4(static_cast<T*>(a.out) + row * a.d + col, acc * inv);
}

template <typename T>
__global__ __launch_bounds__(256) void k_heads_join(HeadsArgs a) {
  const int64_t rows = static_cast<int64_t>(a.tokens_q) * a.heads;
  const int lane = threadIdx.x % 64;
  const int chunk = a.part_head[0];
  for (int64_t row = static_cast<int64_t>(blockIdx.x) * 4 + threadIdx.x / 64; row < rows;
       row += static_cast<int64_t>(gridDim.x) * 4) {
    // All launched splits' places, before the row's own number is known.
    SplitStat mine = a.part_stat[min(lane, a.splits - 1) * rows + row];
    if (chunk == 0) return;
    join_row<T>(a, rows, row, lane, mine);
  }
}

}  // namespace smx
