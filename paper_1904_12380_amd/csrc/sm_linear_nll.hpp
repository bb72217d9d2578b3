// The loss of hidden states against the rows of a vocabulary, and its gradients
// (include/decoder_mi355x.h has the operation), without keeping the logits.
//
//   k_nll_pack      tokens that have a loss are taken together: x of token t
//                   goes to row place[t] of a matrix with rows of whole stages,
//                   so that tokens without a loss cost nothing in the products,
//                   whatever their x holds, and strides and row tails end here.
//   k_nll_product   products of tiles (sm_product.hpp):
//     kLogits   logits of a tile of the vocabulary by tokens; what stays of them
//               is each token's maximum and sum of exponentials over the tile
//     kProbs    the same logits again, turned into g = dl/dlogit, kept for a
//               piece of the vocabulary
//     kInput    sums over the piece's rows for dx, in splits, fp32
//     kWeight   sums over the tokens for the piece's rows of dweight, whole
//     kPartial  fp32: logits over a split of d, kept, where their tiles are few
//   k_nll_join      the tiles' statistics to lse and loss
//   k_nll_total     kPartial's sums to lse and loss
//   k_nll_grad      kPartial's sums to g
//   k_nll_input     the splits' sums to dx
//
// The products are bound by the matrix ops where there are thousands of tokens, by the
// weight's bytes for up to about a hundred (one token x 50001 x 2048 of bf16: 45 us,
// 4.5 TB/s); the other kernels move each of their bytes once.  8192 tokens (5% ignored)
// x 50001 x 2048 of bf16: pack 16 us, logits 1250, join 7; pack 29, probabilities 1415,
// dx 1210, dweight 1300, join of dx 24.  fp32, 4 tokens x 2500 x 4096, in 16 splits of d:
// pack 4, logits 14, k_nll_total 10; pack 5, logits 14, k_nll_grad 4, dx 15, dweight 20,
// join of dx 7.
//
// The logits are formed in both passes by the same operations in the same order, also
// where d is split.
// Of g the label's entry is taken from the loss, e^-loss - 1, which keeps it exact
// where the likelihood is near 1 and lse and the label's logit cancel.
//
// g is rounded to the type for the products on the matrix cores.  It is formed
// relative to the largest |dloss| of the call, in fp32, which enters the sums' last
// rounding: a loss that is a mean over tokens then leaves the label's entry e^-loss
// - 1 itself, not the product with 1 / tokens, whose rounding would be the same for
// all tokens and not average out.  For fp16 it is 2^14 times as large on top: fp16
// then holds 11 bits of it down to 2^-28 of the largest.
//
// A rounding of g averages out over the terms of a sum, unless one of them makes up
// most of it.  Of dx that is the label's, and k_nll_input adds what its rounding left.
// Of dweight any token's may be where there are few: up to kTwoParts tokens g is kept
// in two parts of the type, and both products take both.
#pragma once

#include "sm_product.hpp"

namespace smx {

typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr float kNoLogit = -__builtin_inff();
constexpr int kLogits = 0, kProbs = 1, kInput = 2, kWeight = 3, kPartial = 4;

// What the products know of a token: g = e^(logit - lse) * weight, and `label_g`
// at the label (-1: the label is no row of the vocabulary).
struct NllToken {
  float lse, weight, label_g;
  int label;
};

// What a call knows of its tokens, at the start of its workspace.
struct NllHead {
  int live;      // tokens that have a loss
  float unit;    // what the sums of g are multiplied with
  int pad[2];
};

struct NllArgs {
  const void* x;
  int64_t x_pitch;        // bytes
  const void* weight;
  int64_t w_pitch;        // bytes
  const int64_t* labels;
  int64_t ignore;
  int rows, vocab, d;
  int padded_rows;        // rows, in whole tiles
  int padded_d;           // d, in whole stages
  float* loss;            // written by the forward pass, read by the backward
  float* lse;
  const float* dloss;
  void* dx;               // may be null
  void* dweight;          // may be null
  // Workspace.
  NllHead* head;
  int* place;             // [rows]: a token's row among those that have a loss, or -1
  NllToken* token;        // [padded_rows]
  char* packed;           // [padded_rows, padded_d] of the type
  f32x2* part;            // forward: (max, sum) [tiles, padded_rows]
  float* at;              // forward: the label's logit [padded_rows]
  char* g;                // backward: [padded_rows, piece] of the type
  char* g_rest;           // [kTwoParts, piece]: what the rounding of g left
  float* logits;          // d_splits > 1: [d_splits, padded_rows, padded_vocab]
  float* sums;            // backward: [splits, padded_rows, padded_d]
  float* w_sums;          // backward, w_splits > 1: [w_splits, piece, d]
  int tiles;              // tiles of the vocabulary that `part` has
  int from, piece;        // backward: first row of the piece, and its padded length
  int padded_vocab;       // vocab, in whole tiles
  int d_splits;           // of d, for the logits
  int splits;             // of the piece's rows, for dx
  int w_splits;           // of the tokens, for dweight
};

// What the largest finite |dloss| becomes in g.
template <typename T>
constexpr float kUnitUp = __is_same(T, f16) ? 0x1p14f : 1.0f;

// Tokens with a loss up to which g of 16-bit types is kept in two parts: the backward
// pass of 256 tokens x 50001 x 2048 of bf16 takes 406 us with two, that of 257 tokens
// 344 with one.
constexpr int kTwoParts = 256;
template <typename T>
__device__ __forceinline__ int parts_of(int live) {
  return sizeof(T) == 2 && live <= kTwoParts ? 2 : 1;
}

constexpr int kPackTokens = 16;  // fewest tokens of a workgroup

// Tokens together.  Every workgroup counts the tokens before its own by itself:
// that reads the labels once per workgroup, from the L2, and saves a launch;
// `each` tokens per workgroup grow with their number.
template <typename T, bool BACK>
__global__ __launch_bounds__(256) void k_nll_pack(NllArgs a, int each) {
  __shared__ int count_lds[4];
  __shared__ float most_lds[4];
  const int tid = threadIdx.x, wave = tid / 64, lane = tid % 64;
  const int first = blockIdx.x * each, last = min(first + each, a.rows);
  int count = 0;
#pragma unroll 8
  for (int t = tid; t < first; t += 256) count += a.labels[t] != a.ignore;
  float most = 0.0f;
  if constexpr (BACK) {
#pragma unroll 8
    for (int t = tid; t < a.rows; t += 256) {
      const float w = fabsf(a.dloss[t]);
      if (w <= 3.402823466e38f && a.labels[t] != a.ignore) most = fmaxf(most, w);
    }
    most = seg_max<64>(most);
    if (lane == 0) most_lds[wave] = most;
  }
#pragma unroll
  for (int s = 1; s < 64; s *= 2) count += __shfl_xor(count, s);
  if (lane == 0) count_lds[wave] = count;
  __syncthreads();
  count = count_lds[0] + count_lds[1] + count_lds[2] + count_lds[3];
  float unit = 1.0f;
  if constexpr (BACK) {
    most = fmaxf(fmaxf(most_lds[0], most_lds[1]), fmaxf(most_lds[2], most_lds[3]));
    // A |dloss| far below the normal numbers is taken as it is.
    unit = most < 0x1p-100f ? 1.0f : most;
  }
  const int chunks = a.padded_d * static_cast<int>(sizeof(T)) / 16;
  const int whole = a.d * static_cast<int>(sizeof(T)) / 16;
  for (int t0 = first; t0 < last; t0 += 64) {
    const int t = t0 + lane;
    const int64_t label = t < last ? a.labels[t] : a.ignore;
    const bool live = t < last && label != a.ignore;
    const uint64_t mask = __ballot(live);
    const int row = count + __popcll(mask & ((uint64_t(1) << lane) - 1));
    if (t < last && wave == 0) {
      a.place[t] = live ? row : -1;
      if (live) {
        NllToken k = {0.0f, 0.0f, 0.0f, -1};
        if (label >= 0 && label < a.vocab) k.label = static_cast<int>(label);
        if constexpr (BACK) {
          const float loss = a.loss[t];
          k.lse = a.lse[t];
          k.weight = a.dloss[t] / unit * kUnitUp<T>;
          k.label_g = expm1f(-loss) * k.weight;
          if (k.label < 0) k.weight = __builtin_nanf("");
        }
        a.token[row] = k;
      }
    }
    // Each wavefront copies every fourth token of the 64.
    for (int i = wave; i < 64 && t0 + i < last; i += 4) {
      if (!(mask >> i & 1)) continue;
      const int64_t to = count + __popcll(mask & ((uint64_t(1) << i) - 1));
      const uint4* from = reinterpret_cast<const uint4*>(static_cast<const char*>(a.x) +
                                                         (t0 + i) * a.x_pitch);
      uint4* out = reinterpret_cast<uint4*>(a.packed) + to * chunks;
      for (int c0 = lane; c0 < chunks; c0 += 256) {
        uint4 v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          v[u] = uint4{0, 0, 0, 0};
          if (c0 + 64 * u < whole) v[u] = from[c0 + 64 * u];
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (c0 + 64 * u < chunks) out[c0 + 64 * u] = v[u];
      }
    }
    count += __popcll(mask);
  }
  // The last workgroup knows the number of tokens.
  if (last == a.rows && tid == 0) *a.head = {count, unit / kUnitUp<T>, {0, 0}};
}

// A lane's four values of two tiles side by side (m), to the type, as 16 bytes: the
// lanes l / 16 swap with their neighbours what the others' strip holds.  Even ones
// get m = 4 (l / 16) .. of the first tile, odd ones m = 4 (l / 16) - 4 .. of the
// second.
template <typename T>
__device__ __forceinline__ uint4 strip8(f32x4 first, f32x4 second) {
  typedef T T4 __attribute__((ext_vector_type(4)));
  T4 p, q;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    p[j] = static_cast<T>(first[j]);
    q[j] = static_cast<T>(second[j]);
  }
  const uint2 pu = __builtin_bit_cast(uint2, p), qu = __builtin_bit_cast(uint2, q);
  const auto x = __builtin_amdgcn_permlane16_swap(pu.x, qu.x, false, false);
  const auto y = __builtin_amdgcn_permlane16_swap(pu.y, qu.y, false, false);
  return {x[0], y[0], x[1], y[1]};
}

// What the rounding to the type leaves of four values.
template <typename T>
__device__ __forceinline__ f32x4 rest_of(f32x4 v) {
  f32x4 r;
#pragma unroll
  for (int j = 0; j < 4; ++j) r[j] = v[j] - static_cast<float>(static_cast<T>(v[j]));
  return r;
}

template <int KIND>
struct NllShape {
  // m by rows
  static constexpr bool kARows = KIND == kLogits || KIND == kProbs || KIND == kPartial;
  static constexpr bool kBRows = KIND != kWeight;
};

// One workgroup's tile of one of the products.  In each of them the entries that
// lie side by side in the result are the rows (m) of the tile:
//
//     kLogits, kProbs   m: vocabulary   n: tokens      k: d
//     kPartial          m: vocabulary   n: tokens      k: d (split)
//     kInput            m: d            n: tokens      k: vocabulary (piece, split)
//     kWeight           m: d            n: vocabulary  k: tokens
template <typename T, int KIND, int BM, int BN, int WM, int WN, int STAGES>
__global__ __launch_bounds__(64 * WM * WN) void k_nll_product(NllArgs a) {
  typedef Product<T, NllShape<KIND>::kARows, NllShape<KIND>::kBRows, BM, BN, WM, WN, STAGES> P;
  constexpr int kSize = sizeof(T);
  __shared__ __attribute__((aligned(16))) char raw_lds[P::kLds];
  char SMX_LDS* const lds = (char SMX_LDS*)raw_lds;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / 64);
  const int lane = static_cast<int>(__lane_id()), quarter = lane / 16;
  const int live = a.head->live;
  const int rows = (live + BN - 1) / BN;  // tiles of tokens
  const int left = min(a.vocab - a.from, a.piece);  // of the vocabulary
  int mt, nt;
  const int mtiles = KIND == kLogits || KIND == kPartial ? (a.vocab + BM - 1) / BM
                     : KIND == kProbs                    ? (left + BM - 1) / BM
                                                         : (a.d + BM - 1) / BM;
  const int ntiles = KIND == kWeight ? (left + BN - 1) / BN : rows;
  if (!tile_of(blockIdx.x, mtiles, ntiles, &mt, &nt)) return;
  const int m0 = mt * BM, n0 = nt * BN;
  const int64_t packed_pitch = static_cast<int64_t>(a.padded_d) * kSize;
  const int64_t g_pitch = static_cast<int64_t>(a.piece) * kSize;
  const char* const weight = static_cast<const char*>(a.weight) +
                             (KIND == kLogits ? 0 : a.from) * a.w_pitch;
  P p;
  p.clear();
  // Few tokens: fp32's matrix ops, not the weight's bytes, would bound the narrow tiles,
  // so columns past the tokens are left out, 16 at a time (forward, 50001 x 2048: 156 us
  // for all 64, one token 87, 4.7 TB/s).
  auto run = [&](auto& x, auto& y, int64_t k) {
    if constexpr (kSize == 4 && BN == 64 && WN == 1) {
      if (live - n0 <= 16) return p.template run<1>(x, y, lds, k, wave);
      if (live - n0 <= 32) return p.template run<2>(x, y, lds, k, wave);
    }
    p.run(x, y, lds, k, wave);
  };
  if constexpr (KIND == kLogits || KIND == kProbs) {
    typename P::A x(weight, a.w_pitch, m0, KIND == kLogits ? a.vocab : left, 0, wave);
    typename P::B y(a.packed, packed_pitch, n0, live, 0, wave);
    run(x, y, a.d);
  } else {
    // A split's share of the piece, of the tokens or of d, in whole stages.
    const int all = KIND == kInput ? left : KIND == kPartial ? a.d : live;
    const int stages = (all + P::A::kK - 1) / P::A::kK;
    const int splits = KIND == kInput ? a.splits : KIND == kPartial ? a.d_splits : a.w_splits;
    const int s0 = static_cast<int>(static_cast<int64_t>(stages) * blockIdx.y / splits);
    const int s1 = static_cast<int>(static_cast<int64_t>(stages) * (blockIdx.y + 1) / splits);
    const int64_t k0 = static_cast<int64_t>(s0) * P::A::kK;
    const int64_t k = max(min(static_cast<int64_t>(s1) * P::A::kK, static_cast<int64_t>(all)) - k0,
                          static_cast<int64_t>(0));
    for (int part = 0; part < (KIND == kPartial ? 1 : parts_of<T>(live)); ++part) {
      const char* g = part == 0 ? a.g : a.g_rest;
      if constexpr (KIND == kPartial) {
        typename P::A x(weight, a.w_pitch, m0, a.vocab, k0, wave);
        typename P::B y(a.packed, packed_pitch, n0, live, k0, wave);
        run(x, y, k);
      } else if constexpr (KIND == kInput) {
        typename P::A x(weight, a.w_pitch, m0, a.d, k0, wave);
        typename P::B y(g, g_pitch, n0, live, k0, wave);
        run(x, y, k);
      } else {
        typename P::A x(a.packed, packed_pitch, m0, a.padded_d, k0, wave);
        typename P::B y(g, g_pitch, n0, a.piece, k0, wave);
        run(x, y, k);
      }
    }
  }
  const int mw = m0 + wave % WM * (BM / WM);  // the wavefront's first row
  const int nw = n0 + wave / WM * (BN / WN) + lane % 16;
  const int m4 = mw + 4 * quarter;  // of register 0
  const int m8 = mw + 16 * (quarter % 2) + 4 * (quarter & 2);  // of strip8's bytes
  if constexpr (KIND == kLogits) {
    f32x2 SMX_LDS* const stat = (f32x2 SMX_LDS*)lds;
    // Rows past the vocabulary are no classes.
    if (m0 + BM > a.vocab) {
#pragma unroll
      for (int i = 0; i < P::kMT; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (m4 + 16 * i + r >= a.vocab) {
#pragma unroll
            for (int j = 0; j < P::kNT; ++j) p.acc[i][j][r] = kNoLogit;
          }
    }
#pragma unroll
    for (int j = 0; j < P::kNT; ++j) {
      const int row = nw + 16 * j;
      const int label = row < live ? a.token[row].label : -1;
      float m = kNoLogit;
#pragma unroll
      for (int i = 0; i < P::kMT; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) m = fmaxf(m, p.acc[i][j][r]);
      m = group4_max(m);
      const float ref = m == kNoLogit ? 0.0f : m;
      float t[8] = {};
#pragma unroll
      for (int i = 0; i < P::kMT; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          t[(4 * i + r) % 8] += __builtin_amdgcn_exp2f((p.acc[i][j][r] - ref) * kLog2eF);
      const float s = group4_sum(tree_sum(t));
      if (quarter == 0) stat[wave % WM * BN + row - n0] = f32x2{m, s};
      // The label's logit, where it is one of the wavefront's.
      const int rel = label - m4;
      if (__ballot(label >= mw && label < mw + BM / WM) != 0) {
#pragma unroll
        for (int i = 0; i < P::kMT; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (rel == 16 * i + r) a.at[row] = p.acc[i][j][r];
      }
    }
    __syncthreads();
    for (int n = threadIdx.x; n < BN; n += 64 * WM * WN) {
      f32x2 v = stat[n];
#pragma unroll
      for (int w = 1; w < WM; ++w) {
        const f32x2 u = stat[w * BN + n];
        const float m = fmaxf(v.x, u.x), ref = m == kNoLogit ? 0.0f : m;
        v.y = v.y * __builtin_amdgcn_exp2f((v.x - ref) * kLog2eF) +
              u.y * __builtin_amdgcn_exp2f((u.x - ref) * kLog2eF);
        v.x = m;
      }
      a.part[static_cast<int64_t>(mt) * a.padded_rows + n0 + n] = v;
    }
  } else if constexpr (KIND == kProbs) {
#pragma unroll
    for (int j = 0; j < P::kNT; ++j) {
      const int row = nw + 16 * j;
      const NllToken k = a.token[row];
      const int rel = k.label - a.from - m4;
      const int rest = left - m4;
      char* const out = a.g + row * g_pitch;
#pragma unroll
      for (int i = 0; i < P::kMT; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int at = 16 * i + r;
          float v = __builtin_amdgcn_exp2f((p.acc[i][j][r] - k.lse) * kLog2eF) * k.weight;
          v = rel == at ? k.label_g : v;
          p.acc[i][j][r] = at < rest ? v : 0.0f;
        }
      const bool two = parts_of<T>(live) == 2 && row < kTwoParts;
#pragma unroll
      for (int i = 0; i < P::kMT; i += kSize == 2 ? 2 : 1) {
        if constexpr (kSize == 2) {
          *reinterpret_cast<uint4*>(out + (m8 + 16 * i) * 2) =
              strip8<T>(p.acc[i][j], p.acc[i + 1][j]);
          if (__any(two)) {
            const uint4 rest = strip8<T>(rest_of<T>(p.acc[i][j]), rest_of<T>(p.acc[i + 1][j]));
            if (two) *reinterpret_cast<uint4*>(a.g_rest + row * g_pitch + (m8 + 16 * i) * 2) = rest;
          }
        }
        else
          *reinterpret_cast<f32x4*>(out + (m4 + 16 * i) * 4) = p.acc[i][j];
      }
    }
  } else if constexpr (KIND == kPartial) {
    float* const logits =
        a.logits + static_cast<int64_t>(blockIdx.y) * a.padded_rows * a.padded_vocab;
#pragma unroll
    for (int j = 0; j < P::kNT; ++j) {
      const int row = nw + 16 * j;
      if (row >= live) continue;
      float* const out = logits + static_cast<int64_t>(row) * a.padded_vocab + m4;
#pragma unroll
      for (int i = 0; i < P::kMT; ++i) *reinterpret_cast<f32x4*>(out + 16 * i) = p.acc[i][j];
    }
  } else if constexpr (KIND == kInput) {
    float* const sums = a.sums + static_cast<int64_t>(blockIdx.y) * a.padded_rows * a.padded_d;
#pragma unroll
    for (int j = 0; j < P::kNT; ++j) {
      float* const out = sums + static_cast<int64_t>(nw + 16 * j) * a.padded_d;
#pragma unroll
      for (int i = 0; i < P::kMT; ++i) {
        const int m = m4 + 16 * i;
        if (m >= a.d) continue;
        f32x4* const o = reinterpret_cast<f32x4*>(out + m);
        *o = a.from > 0 ? *o + p.acc[i][j] : p.acc[i][j];
      }
    }
  } else if (a.w_splits > 1) {
    float* const sums = a.w_sums + static_cast<int64_t>(blockIdx.y) * a.piece * a.d;
#pragma unroll
    for (int j = 0; j < P::kNT; ++j) {
      const int row = nw + 16 * j;
#pragma unroll
      for (int i = 0; i < P::kMT; ++i) {
        const int m = m4 + 16 * i;
        if (row < left && m < a.d)
          *reinterpret_cast<f32x4*>(sums + static_cast<int64_t>(row) * a.d + m) = p.acc[i][j];
      }
    }
  } else {
    const float unit = a.head->unit;
#pragma unroll
    for (int j = 0; j < P::kNT; ++j) {
      const int row = nw + 16 * j;
      char* const out = static_cast<char*>(a.dweight) +
                        (static_cast<int64_t>(a.from) + row) * a.d * kSize;
#pragma unroll
      for (int i = 0; i < P::kMT; i += kSize == 2 ? 2 : 1) {
        if constexpr (kSize == 2) {
          const uint4 strip = strip8<T>(p.acc[i][j] * unit, p.acc[i + 1][j] * unit);
          const int m = m8 + 16 * i;
          if (row < left && m < a.d) *reinterpret_cast<uint4*>(out + m * 2) = strip;
        } else {
          const int m = m4 + 16 * i;
          if (row < left && m < a.d) *reinterpret_cast<f32x4*>(out + m * 4) = p.acc[i][j] * unit;
        }
      }
    }
  }
}

// lse = M + ln S and loss = (M - x_label) + ln S from the tiles' statistics, summed in
// binary64: 16 tokens per workgroup, 16 threads over the tiles of each, which load
// eight tiles at a time.
constexpr int kJoinTokens = 16;
template <int SHARES>
__global__ __launch_bounds__(kJoinTokens* SHARES) void k_nll_join(NllArgs a) {
  __shared__ float m_lds[SHARES][kJoinTokens];
  __shared__ double s_lds[SHARES][kJoinTokens];
  const int lane = threadIdx.x % kJoinTokens, share = threadIdx.x / kJoinTokens;
  const int t = blockIdx.x * kJoinTokens + lane;
  const int row = t < a.rows ? a.place[t] : -1;
  float m = kNoLogit;
  double s = 0.0;
  if (row >= 0)
    for (int i0 = share; i0 < a.tiles; i0 += 8 * SHARES) {
      f32x2 v[8];
      float top = m;
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int i = i0 + u * SHARES;
        v[u] = f32x2{kNoLogit, 0.0f};
        if (i < a.tiles) v[u] = a.part[static_cast<int64_t>(i) * a.padded_rows + row];
        top = fmaxf(top, v[u].x);
      }
      const float ref = top == kNoLogit ? 0.0f : top;
      s *= static_cast<double>(__builtin_amdgcn_exp2f((m - ref) * kLog2eF));
#pragma unroll
      for (int u = 0; u < 8; ++u)
        s += static_cast<double>(v[u].y * __builtin_amdgcn_exp2f((v[u].x - ref) * kLog2eF));
      m = top;
    }
  m_lds[share][lane] = m;
  s_lds[share][lane] = s;
  __syncthreads();
  if (share != 0 || t >= a.rows) return;
#pragma unroll
  for (int w = 1; w < SHARES; ++w) m = fmaxf(m, m_lds[w][lane]);
  const float ref = m == kNoLogit ? 0.0f : m;
  s = 0.0;
#pragma unroll
  for (int w = 0; w < SHARES; ++w)
    s += s_lds[w][lane] *
         static_cast<double>(__builtin_amdgcn_exp2f((m_lds[w][lane] - ref) * kLog2eF));
  float loss = 0.0f, lse = 0.0f;
  if (row >= 0) {
    const double log_s = log(s);
    const bool bad = a.token[row].label < 0;
    lse = static_cast<float>(m + log_s);
    loss = bad ? __builtin_nanf("")
               : static_cast<float>(static_cast<double>(m) - a.at[row] + log_s);
  }
  a.lse[t] = lse;
  a.loss[t] = loss;
}

// Four logits of a token, v and on, from the splits of d.
__device__ __forceinline__ f32x4 logits_of(const NllArgs& a, int row, int v) {
  const float* p = a.logits + static_cast<int64_t>(row) * a.padded_vocab + v;
  const int64_t each = static_cast<int64_t>(a.padded_rows) * a.padded_vocab;
  f32x4 sum = *reinterpret_cast<const f32x4*>(p);
#pragma unroll 4
  for (int s = 1; s < a.d_splits; ++s) sum += *reinterpret_cast<const f32x4*>(p + s * each);
  return sum;
}

// lse and loss as k_nll_join has them, from the splits' logits: a workgroup for each
// token, whose threads take eight logits at a time.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void k_nll_total(NllArgs a) {
  __shared__ float m_lds[THREADS / 64];
  __shared__ double s_lds[THREADS / 64];
  const int t = blockIdx.x, tid = threadIdx.x;
  const int row = a.place[t];
  if (row < 0) {
    if (tid == 0) a.lse[t] = a.loss[t] = 0.0f;
    return;
  }
  float m = kNoLogit;
  double s = 0.0;
  for (int v0 = 4 * tid; v0 < a.vocab; v0 += 8 * THREADS) {
    float v[8];
    float top = m;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int at = v0 + u * 4 * THREADS;
      f32x4 l = {};
      if (at < a.vocab) l = logits_of(a, row, at);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[4 * u + j] = at + j < a.vocab ? l[j] : kNoLogit;
        top = fmaxf(top, v[4 * u + j]);
      }
    }
    const float ref = top == kNoLogit ? 0.0f : top;
    s *= static_cast<double>(__builtin_amdgcn_exp2f((m - ref) * kLog2eF));
#pragma unroll
    for (int j = 0; j < 8; ++j)
      s += static_cast<double>(__builtin_amdgcn_exp2f((v[j] - ref) * kLog2eF));
    m = top;
  }
  const float wave_m = seg_max<64>(m);
  float ref = wave_m == kNoLogit ? 0.0f : wave_m;
  s = wave_sum64(s * static_cast<double>(__builtin_amdgcn_exp2f((m - ref) * kLog2eF)));
  if (tid % 64 == 0) {
    m_lds[tid / 64] = wave_m;
    s_lds[tid / 64] = s;
  }
  __syncthreads();
  if (tid != 0) return;
  m = m_lds[0];
#pragma unroll
  for (int w = 1; w < THREADS / 64; ++w) m = fmaxf(m, m_lds[w]);
  ref = m == kNoLogit ? 0.0f : m;
  s = 0.0;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w)
    s += s_lds[w] * static_cast<double>(__builtin_amdgcn_exp2f((m_lds[w] - ref) * kLog2eF));
  const double log_s = log(s);
  const int label = a.token[row].label;
  a.lse[t] = static_cast<float>(m + log_s);
  a.loss[t] = label < 0 ? __builtin_nanf("")
                        : static_cast<float>(static_cast<double>(m) -
                                             logits_of(a, row, label & ~3)[label & 3] + log_s);
}

// g (fp32) of the tokens that have a loss, as kProbs leaves it, from the splits' logits.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void k_nll_grad(NllArgs a) {
  const int strips = (a.vocab + 3) / 4;
  const int64_t all = static_cast<int64_t>(a.head->live) * strips;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * THREADS + threadIdx.x; i < all;
       i += static_cast<int64_t>(gridDim.x) * THREADS) {
    const int row = static_cast<int>(i / strips), v = static_cast<int>(i % strips) * 4;
    const f32x4 l = logits_of(a, row, v);
    const NllToken k = a.token[row];
    f32x4 g;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float x = __builtin_amdgcn_exp2f((l[j] - k.lse) * kLog2eF) * k.weight;
      g[j] = v + j >= a.vocab ? 0.0f : v + j == k.label ? k.label_g : x;
    }
    *reinterpret_cast<f32x4*>(a.g + (static_cast<int64_t>(row) * a.piece + v) * 4) = g;
  }
}

// The piece's rows of dweight from the splits' sums.
template <typename T>
__global__ __launch_bounds__(256) void k_nll_weight(NllArgs a) {
  const int64_t strips = static_cast<int64_t>(min(a.vocab - a.from, a.piece)) * a.d / 4;
  const int64_t each = static_cast<int64_t>(a.piece) * a.d;
  const float unit = a.head->unit;
  typedef T T4 __attribute__((ext_vector_type(4)));
  T4* const out = reinterpret_cast<T4*>(static_cast<T*>(a.dweight) + static_cast<int64_t>(a.from) * a.d);
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < strips;
       i += static_cast<int64_t>(gridDim.x) * 256) {
    f32x4 sum = {};
#pragma unroll 8
    for (int s = 0; s < a.w_splits; ++s)
      sum += *reinterpret_cast<const f32x4*>(a.w_sums + s * each + 4 * i);
    sum *= unit;
    T4 v;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = static_cast<T>(sum[j]);
    out[i] = v;
  }
}

template <int UNUSED>
__global__ __launch_bounds__(256) void k_nll_clear(uint4* out, int64_t strips) {
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < strips;
       i += static_cast<int64_t>(gridDim.x) * 256)
    out[i] = uint4{0, 0, 0, 0};
}

// dx of every token from the splits' sums, and what the rounding of g left at the label:
// zeros for those without a loss.
template <typename T>
__global__ __launch_bounds__(256) void k_nll_input(NllArgs a) {
  const int strips = a.d / 8;
  const int64_t all = static_cast<int64_t>(a.rows) * strips;
  const float unit = a.head->unit;
  const bool one = sizeof(T) == 2 && parts_of<T>(a.head->live) == 1;
  typedef T T8 __attribute__((ext_vector_type(8)));
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < all;
       i += static_cast<int64_t>(gridDim.x) * 256) {
    const int t = static_cast<int>(i / strips), c = static_cast<int>(i % strips) * 8;
    const int row = a.place[t];
    f32x4 lo = {}, hi = {};
    if (row >= 0) {
      for (int s = 0; s < a.splits; ++s) {
        const float* p =
            a.sums + (static_cast<int64_t>(s) * a.padded_rows + row) * a.padded_d + c;
        lo += *reinterpret_cast<const f32x4*>(p);
        hi += *reinterpret_cast<const f32x4*>(p + 4);
      }
      const NllToken k = a.token[row];
      if (one && k.label >= 0) {
        const float rest = k.label_g - static_cast<float>(static_cast<T>(k.label_g));
        const T8 w = *reinterpret_cast<const T8*>(static_cast<const char*>(a.weight) +
                                                  k.label * a.w_pitch + c * sizeof(T));
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          lo[j] += rest * static_cast<float>(w[j]);
          hi[j] += rest * static_cast<float>(w[4 + j]);
        }
      }
    }
    lo *= unit;
    hi *= unit;
    T* const out = static_cast<T*>(a.dx) + static_cast<int64_t>(t) * a.d + c;
    T8 v;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[j] = static_cast<T>(lo[j]);
      v[4 + j] = static_cast<T>(hi[j]);
    }
    *reinterpret_cast<T8*>(out) = v;
  }
}

}  // namespace smx
