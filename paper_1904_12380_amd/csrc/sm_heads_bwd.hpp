// Multi-head attention of 16-bit types: the gradients.
//
// The layout of sm_heads_mfma.hpp, twice.  The gradient of the queries goes
// by rows like the forward pass: S^T = K Q^T and dP^T = V dO^T with Q and dO in
// registers, and dS^T as it lies is the B operand of dQ^T += K^T dS^T.  The
// gradients of the keys and values go by keys: S = Q K^T and dP = dO V^T with K
// and V in registers, and P and dS are the B operands of dV^T += dO^T P and
// dK^T += Q^T dS.  Seven products instead of the five that one pass over both
// would take, but every sum has one owner: no atomics, the same bits each time.
//
// The first kernel writes what the second needs of every row as a pair (lse
// in powers of two, D), head by head, so that the second reads it by tokens.
#pragma once

#include "sm_heads_mfma.hpp"

namespace smx {

// Weights and score gradients are taken in two 16-bit parts for the first 64
// keys of a document where rows see at most this many keys.
constexpr int kTwoPartKeys = 128;

template <typename T, int DP>
__device__ __forceinline__ f32x16 rows_dot(const TileReader<DP>& rd, const char SMX_LDS* tile,
                                           int row0,
                                           const typename Vec8<T>::type (&b)[DP / 16]) {
  f32x16 s = {};
#pragma unroll
  for (int st = 0; st < DP / 16; ++st) s = mfma32(rd.template rows<T>(tile, row0, st), b[st], s);
  return s;
}

// acc[t] += (columns of the tile's rows row0 .. row0 + 31)^T x, x rounded to
// the type, or in two parts.
template <typename T, int DP>
__device__ __forceinline__ void cols_accumulate(const TileReader<DP>& rd,
                                                const char SMX_LDS* tile, int row0,
                                                const f32x16& x, bool two_parts,
                                                f32x16 (&acc)[DP / 32]) {
  typedef typename Vec8<T>::type V;
  V hi[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) hi[u] = pack8<T>(x, 8 * u);
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int t = 0; t < DP / 32; ++t)
      acc[t] = mfma32(rd.template cols<T>(tile, row0 + 16 * u, t), hi[u], acc[t]);
  if (two_parts) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const V lo = pack8_rest<T>(x, 8 * u, hi[u]);
#pragma unroll
      for (int t = 0; t < DP / 32; ++t)
        acc[t] = mfma32(rd.template cols<T>(tile, row0 + 16 * u, t), lo, acc[t]);
    }
  }
}

template <typename T, int DP>
__device__ __forceinline__ void store_columns(T* p, int d, int half, const f32x16 (&acc)[DP / 32],
                                              float f) {
  typedef T t4 __attribute__((ext_vector_type(4)));
#pragma unroll
  for (int t = 0; t < DP / 32; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int col = 32 * t + 8 * i + 4 * half;
      t4 x;
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = static_cast<T>(acc[t][4 * i + j] * f);
      if (col < d) *reinterpret_cast<t4*>(p + col) = x;
    }
}

template <typename T, int DP, bool SCORED>
__global__ __launch_bounds__(kTileThreads, DP <= 128 ? 2 : 1) void k_heads_dq(HeadsArgs a) {
  __shared__ __attribute__((aligned(16))) char lds_bytes[tile_lds_bytes<DP>()];
  char SMX_LDS* lds = (char SMX_LDS*)lds_bytes;
  const int hk = blockIdx.x % a.kv_heads;
  const int slot = static_cast<int>(gridDim.x / a.kv_heads - 1 - blockIdx.x / a.kv_heads);
  DocTile w;
  w.b = find_doc<kTileRows>(a.cu_q, a.n, a.tokens_q, a.group, slot, &w.tile);
  doc_queries(a, &w);
  doc_keys<false>(a, &w);
  const int rows = w.lq * a.group;
  const int row0 = w.tile * kTileRows;
  if (row0 >= rows) return;
  const int tile_rows = min(rows - row0, kTileRows);
  const int to = keys_seen(a, w, (row0 + tile_rows - 1) / a.group);

  const int lane = threadIdx.x % 64, half = lane / 32;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int local = 32 * wave + lane % 32;
  const bool valid = local < tile_rows;
  const int row = valid ? row0 + local : rows - 1;
  const int tok = row / a.group, head = hk * a.group + row % a.group;
  const int64_t token = w.q0 + tok, out = token * a.heads + head;
  const int pos = tok + w.lk - w.lq;
  const int lim = valid ? keys_seen(a, w, tok) : 0;
  int lim_all = 0, lim_any = 0;
  if (32 * wave < tile_rows) {
    lim_all = keys_seen(a, w, (row0 + 32 * wave) / a.group);
    lim_any = keys_seen(a, w, (min(rows, row0 + 32 * wave + 32) - 1) / a.group);
  }
  const float slope = SCORED && a.slopes != nullptr ? a.slopes[head] : 0.0f;
  const float c = SCORED ? 1.0f : fabsf(a.scale) * kLog2eF;

  typedef typename Vec8<T>::type V;
  V q[DP / 16], dout[DP / 16];
  load_operand<T, DP>(q, static_cast<const T*>(a.q.data) + token * a.q.ts + head * a.q.hs, valid,
                      half, a.d);
  load_operand<T, DP>(dout,
                      static_cast<const T*>(a.dout.data) + token * a.dout.ts + head * a.dout.hs,
                      valid, half, a.d);
  float delta = 0.0f;
  {
    V o[DP / 16];
    load_operand<T, DP>(o, static_cast<const T*>(a.o.data) + token * a.o.ts + head * a.o.hs,
                        valid, half, a.d);
#pragma unroll
    for (int s = 0; s < DP / 16; ++s)
#pragma unroll
      for (int j = 0; j < 8; ++j)
        delta = __builtin_fmaf(static_cast<float>(o[s][j]), static_cast<float>(dout[s][j]), delta);
    delta += half32_partner(delta);
  }
  // Rows that see no key: weights of zero from the finite scores.
  float lse2 = INFINITY;
  if (valid && lim > 0) {
    lse2 = a.lse[out] * kLog2eF;
    if (lse2 == -INFINITY) lse2 = INFINITY;
  }
  if (!SCORED && a.scale < 0.0f) {
#pragma unroll
    for (int i = 0; i < DP / 16; ++i) q[i] = -q[i];
  }
  f32x16 acc[DP / 32] = {};

  const Stager<DP, false> ks(a.k, 0, w.k0, hk), vs(a.v, 0, w.k0, hk);
  const TileReader<DP> rd;
  constexpr int kTile = kTileKeys * DP * 2;
  constexpr int N = kTileKeys / 4 / Stager<DP, false>::kRows;
  const int r0 = wave * (kTileKeys / 4), d2 = 2 * a.d;
  auto stage = [&](int k0, int buf) {
    char SMX_LDS* kt = lds + buf * 2 * kTile + r0 * DP * 2;
    stage_packed<DP, N>(ks, kt, k0, r0, to, d2);
    stage_packed<DP, N>(vs, kt + kTile, k0, r0, to, d2);
  };

  // Weights, and the scores' gradient over (dP - D), of 32 keys.
  auto weights = [&](f32x16& s, f32x16& dcap, int k0) {
    if constexpr (SCORED) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int j = k0 + 8 * (i / 4) + 4 * half + i % 4;
        float x;
        s[i] = score16(a, s[i], slope, pos - j, &x);
        dcap[i] = x;
      }
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], c, -lse2));
    if (k0 + 32 > lim_all) {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (k0 + 8 * (i / 4) + 4 * half + i % 4 >= lim) s[i] = 0.0f;
    }
  };

  if (to > 0) stage(0, 0);
  int buf = 0;
  for (int k0 = 0; k0 < to; k0 += kTileKeys, buf ^= 1) {
    staged();
    __syncthreads();
    if (k0 + kTileKeys < to) stage(k0 + kTileKeys, buf ^ 1);
    if (k0 >= lim_any) continue;
    const char SMX_LDS* kt = lds + buf * 2 * kTile;
    const char SMX_LDS* vt = kt + kTile;
    const bool two_parts = k0 == 0 && lim_all <= kTwoPartKeys;
    if (k0 == 0 && lim_all <= kTileKeys) {
      // Rows that see no key past this tile: D from the weights themselves,
      // which o's rounding would put off where few keys share them.
      float sum = 0.0f;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        f32x16 s = rows_dot<T, DP>(rd, kt, 32 * h, q), dcap;
        const f32x16 dp = rows_dot<T, DP>(rd, vt, 32 * h, dout);
        weights(s, dcap, 32 * h);
#pragma unroll
        for (int i = 0; i < 16; ++i) sum = __builtin_fmaf(s[i], dp[i], sum);
      }
      sum += half32_partner(sum);
      if (lim <= kTileKeys) delta = sum;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      f32x16 s = rows_dot<T, DP>(rd, kt, 32 * h, q), dcap;
      f32x16 dp = rows_dot<T, DP>(rd, vt, 32 * h, dout);
      weights(s, dcap, k0 + 32 * h);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        dp[i] = s[i] * (dp[i] - delta);
        if constexpr (SCORED) dp[i] *= dcap[i];
      }
      cols_accumulate<T, DP>(rd, kt, 32 * h, dp, two_parts, acc);
    }
  }
  if (!valid) return;
  if (half == 0)
    reinterpret_cast<float2*>(a.delta)[static_cast<int64_t>(head) * a.tokens_q + token] =
        make_float2(lse2, delta);
  store_columns<T, DP>(static_cast<T*>(a.out) + out * a.d, a.d, half, acc, a.scale);
}

template <typename T, int DP, bool SCORED>
__global__ __launch_bounds__(kTileThreads, DP <= 128 ? 2 : 1) void k_heads_dkv(HeadsArgs a) {
  __shared__ __attribute__((aligned(16))) char lds_bytes[tile_lds_bytes<DP>()];
  __shared__ __attribute__((aligned(16))) float stats[2][2][kTileKeys];  // [stage][lse, D][row]
  char SMX_LDS* lds = (char SMX_LDS*)lds_bytes;
  const int hk = blockIdx.x % a.kv_heads;
  DocTile w;
  w.b = find_doc<kTileRows>(a.cu_k, a.n, a.tokens_k, 1, blockIdx.x / a.kv_heads, &w.tile);
  doc_queries(a, &w);
  doc_keys<false>(a, &w);
  if (w.b >= a.n) {  // keys past the last document
    w.k0 = doc_start(a.cu_k, a.n, a.tokens_k);
    w.lk = a.tokens_k - w.k0;
    w.lq = 0;
  }
  const int first = w.tile * kTileRows;
  if (first >= w.lk) return;

  const int tid = threadIdx.x, lane = tid % 64, half = lane / 32;
  const int wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int key0 = first + 32 * wave;  // of the wavefront
  const int key = key0 + lane % 32;
  const bool valid = key < w.lk;
  const int64_t token = w.k0 + key;
  const float c = SCORED ? 1.0f : fabsf(a.scale) * kLog2eF;

  typedef typename Vec8<T>::type V;
  V k[DP / 16], v[DP / 16];
  load_operand<T, DP>(k, static_cast<const T*>(a.k.data) + token * a.k.ts + hk * a.k.hs, valid,
                      half, a.d);
  load_operand<T, DP>(v, static_cast<const T*>(a.v.data) + token * a.v.ts + hk * a.v.hs, valid,
                      half, a.d);
  if (!SCORED && a.scale < 0.0f) {
#pragma unroll
    for (int i = 0; i < DP / 16; ++i) k[i] = -k[i];
  }
  f32x16 dk[DP / 32] = {}, dv[DP / 32] = {};

  const TileReader<DP> rd;
  constexpr int kTile = kTileKeys * DP * 2;
  constexpr int N = kTileKeys / 4 / Stager<DP, false>::kRows;
  const int r0 = wave * (kTileKeys / 4), d2 = 2 * a.d;
  // The first token that sees the workgroup's first key.
  const int tok0 = a.causal && first >= w.prefix ? max(first - (w.lk - w.lq), 0) : 0;
  const int tiles = tok0 < w.lq ? (w.lq - tok0 + kTileKeys - 1) / kTileKeys : 0;
  const int turns = tiles * a.group;

  float2 stat = {INFINITY, 0.0f};
  auto stage = [&](int turn, int buf) {
    const int head = hk * a.group + turn / tiles;
    const int t0 = tok0 + turn % tiles * kTileKeys;
    const Stager<DP, false> qs(a.q, 0, w.q0, head), os(a.dout, 0, w.q0, head);
    char SMX_LDS* qt = lds + buf * 2 * kTile + r0 * DP * 2;
    stage_packed<DP, N>(qs, qt, t0, r0, w.lq, d2);
    stage_packed<DP, N>(os, qt + kTile, t0, r0, w.lq, d2);
    if (wave == 0) {
      stat = make_float2(INFINITY, 0.0f);
      if (t0 + lane < w.lq)
        stat = reinterpret_cast<const float2*>(
            a.delta)[static_cast<int64_t>(head) * a.tokens_q + w.q0 + t0 + lane];
    }
  };
  auto write_stats = [&](int buf) {
    if (wave == 0) {
      stats[buf][0][lane] = stat.x;
      stats[buf][1][lane] = stat.y;
    }
  };

  if (turns > 0) {
    stage(0, 0);
    write_stats(0);
  }
  int buf = 0;
  for (int turn = 0; turn < turns; ++turn, buf ^= 1) {
    staged();
    __syncthreads();
    if (turn + 1 < turns) stage(turn + 1, buf ^ 1);
    const int t0 = tok0 + turn % tiles * kTileKeys;
    const char SMX_LDS* qt = lds + buf * 2 * kTile;
    const char SMX_LDS* ot = qt + kTile;
    const float slope =
        SCORED && a.slopes != nullptr ? a.slopes[hk * a.group + turn / tiles] : 0.0f;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int t1 = t0 + 32 * h;
      if (t1 >= w.lq || keys_seen(a, w, min(t1 + 31, w.lq - 1)) <= key0) continue;
      const int lim_all = keys_seen(a, w, t1);
      f32x16 s = rows_dot<T, DP>(rd, qt, 32 * h, k), dcap;
      f32x16 dp = rows_dot<T, DP>(rd, ot, 32 * h, v);
      if constexpr (SCORED) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int tok = t1 + 8 * (i / 4) + 4 * half + i % 4;
          float x;
          s[i] = score16(a, s[i], slope, tok + w.lk - w.lq - key, &x);
          dcap[i] = x;
        }
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int r = 32 * h + 8 * (i / 4) + 4 * half + i % 4;
        s[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], c, -stats[buf][0][r]));
        dp[i] -= stats[buf][1][r];
      }
      if (lim_all < key0 + 32) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int tok = t1 + 8 * (i / 4) + 4 * half + i % 4;
          if (key >= keys_seen(a, w, tok)) s[i] = 0.0f;
        }
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        dp[i] *= s[i];
        if constexpr (SCORED) dp[i] *= dcap[i];
      }
      const bool two_parts = key0 < kTileKeys && lim_all <= kTwoPartKeys;
      cols_accumulate<T, DP>(rd, ot, 32 * h, s, two_parts, dv);
      cols_accumulate<T, DP>(rd, qt, 32 * h, dp, two_parts, dk);
    }
    write_stats(buf ^ 1);
  }
  if (!valid) return;
  const int64_t out = (token * a.kv_heads + hk) * a.d;
  store_columns<T, DP>(static_cast<T*>(a.dk) + out, a.d, half, dk, a.scale);
  store_columns<T, DP>(static_cast<T*>(a.dv) + out, a.d, half, dv, 1.0f);
}

}  // namespace smx
