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
// The first kernel writes what the second needs of every row as a pair (-lse
// / c, -D) (fp16: with the lift of the weights, below), head by head, so that the
// second reads it by tokens: the values that its scores and dP start from, so that
// the shift and the difference cost no instruction.
#pragma once

#include "sm_heads_f32.hpp"
#include "sm_heads_mfma.hpp"

namespace smx {

// Weights and score gradients of a block of 32 rows and 32 keys are taken in
// two 16-bit parts where a weight of the block is larger than this: its
// rounding is then a part of the sums that no others average, and with D's
// would put gradients of rows with few keys (or a steep bias) off by 1.7 times
// their own rounding to 16 bits.
constexpr float kLargeWeight = 0.125f;

__device__ __forceinline__ bool any_large(const f32x16& p, float large) {
  float top = p[0];
#pragma unroll
  for (int i = 1; i < 16; ++i) top = fmaxf(top, p[i]);
  return __any(top > large);
}

// What is rounded to fp16 for a product is put into its range first, and its sums
// are taken back when they are stored; bf16 has the range of fp32 and needs
// neither.
//
// Weights for dV are at most 1 but for their scores' rounding, and a key that
// many rows see little of sums up many small ones: they are formed 2^kWeightLift
// times as large, in the exponent's argument, with 11 bits down to 2^-26.
template <typename T>
constexpr int kWeightLift = __is_same(T, f16) ? 12 : 0;

// Score gradients are of any size, with that of dO.  A lane pair's own (one row
// of dQ, one key of dK) are taken times a power of two, lowered when a value
// would pass 2^15, to leave it below 2^9, so that few blocks lower it; the sums so
// far go with it.  A value then loses bits to fp16's denormal numbers only where it
// is 2^22 times smaller than one that the sum already has.
template <typename T>
struct FitRange {
  template <int N>
  __device__ __forceinline__ void fit(f32x16&, f32x16 (&)[N]) {}
  __device__ __forceinline__ float back() const { return 1.0f; }
};
template <>
struct FitRange<f16> {
  float f = 0x1p100f;  // fp16's smallest dO, V and weights leave more than 2^-80

  // x is multiplied by f; acc holds sums of earlier such x.
  template <int N>
  __device__ __forceinline__ void fit(f32x16& x, f32x16 (&acc)[N]) {
    float top = fabsf(x[0]);
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, fabsf(x[i]));
    top = fmaxf(top, half32_partner(top));
    if (__any(top * f > 0x1p15f)) {
      // 2^8 <= top * next < 2^9, from top's exponent.
      const int now = __builtin_bit_cast(int, f);
      const int next = top * f > 0x1p15f
                           ? (127 + 127 + 8 - (__builtin_bit_cast(int, top) >> 23)) << 23 : now;
      const float ratio = __builtin_bit_cast(float, max(next - now + (127 << 23), 0));
#pragma unroll
      for (int t = 0; t < N; ++t) acc[t] *= ratio;
      f = __builtin_bit_cast(float, next);
    }
    x *= f;
  }
  // 1 / f.
  __device__ __forceinline__ float back() const {
    return __builtin_bit_cast(float, (254 << 23) - __builtin_bit_cast(int, f));
  }
};

template <typename T, int DP>
__device__ __forceinline__ f32x16 rows_dot(const TileReader<DP>& rd, const char SMX_LDS* tile,
                                           int row0,
                                           const typename Vec8<T>::type (&b)[DP / 16],
                                           f32x16 s = f32x16{}) {
#pragma unroll
  for (int st = 0; st < DP / 16; ++st) s = mfma32(rd.template rows<T>(tile, row0, st), b[st], s);
  interleave<DP / 16, 1>();
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
  interleave<2 * DP / 32, 2>();
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

// The lane's row, of fp32 sums, times f.
template <int DP>
__device__ __forceinline__ void store_sums(float* p, int d, int half,
                                           const f32x16 (&acc)[DP / 32], float f) {
#pragma unroll
  for (int t = 0; t < DP / 32; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int col = 32 * t + 8 * i + 4 * half;
      f32x4 x;
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = acc[t][4 * i + j] * f;
      if (col < d) *reinterpret_cast<f32x4*>(p + col) = x;
    }
}

// D's error that is left alone, as a part of the sum of the sizes of a row's score
// gradients: half of the type's unit roundoff.  Where one key's term opposes all
// others' it is half of that sum, and dQ's error then stays within the roundoff.
template <typename T>
constexpr float kMostOff = __is_same(T, f16) ? 0x1p-12f : 0x1p-9f;

// dQ and D, by rows: three products for each pair, in one pass over the keys, and
// where D's error counts (below) two more in a second.  16384 tokens of one document
// (16 heads of 128 on 2, bf16): 1.65 ms, 1000 TFLOP/s; 8192 tokens of documents of up
// to 2048 (32 heads on 8): 156 us, 510 TFLOP/s, since most of these are a few tiles
// long.  Bound by matrix ops and LDS reads: one operand of each product comes from
// LDS, 32 rows of it for 32 columns held in registers.  At a width of 128 the plain
// scores' instance holds all of its registers; a bias spills 22 of them, a cap 8 and
// both 88.
template <typename T, int DP, int MODE>
__global__ __launch_bounds__(kTileThreads, DP <= 128 ? 2 : 1) void k_heads_dq(HeadsArgs a) {
  __shared__ __attribute__((aligned(16))) char lds_bytes[tile_lds_bytes<DP>()];
  __shared__ int redo[4];
  char SMX_LDS* lds = (char SMX_LDS*)lds_bytes;
  const int hk = blockIdx.x % a.kv_heads;
  const int slot = static_cast<int>(gridDim.x / a.kv_heads - 1 - blockIdx.x / a.kv_heads);
  const DocTile w =
      find_tile<kTileRows, false, false>(a, load_docs<false>(a, threadIdx.x % 64), slot);
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
  const Scoring<MODE> sc(a, MODE != kPlain && a.slopes != nullptr ? a.slopes[head] : 0.0f);
  const float c = sc.unit();

  typedef typename Vec8<T>::type V;
  V q[DP / 16], dout[DP / 16];
  load_operand<T, DP>(q, static_cast<const T*>(a.q.data) + token * a.q.ts + head * a.q.hs, valid,
                      half, a.d);
  load_operand<T, DP>(dout,
                      static_cast<const T*>(a.dout.data) + token * a.dout.ts + head * a.dout.hs,
                      valid, half, a.d);
  float delta = 0.0f, around = 0.0f;  // D, and the sum of |do o|
  {
    V o[DP / 16];
    load_operand<T, DP>(o, static_cast<const T*>(a.o.data) + token * a.o.ts + head * a.o.hs,
                        valid, half, a.d);
#pragma unroll
    for (int s = 0; s < DP / 16; ++s)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float x = static_cast<float>(o[s][j]) * static_cast<float>(dout[s][j]);
        delta += x;
        around += fabsf(x);
      }
    delta += half32_partner(delta);
    around += half32_partner(around);
  }
  // Rows that see no key: weights of zero from the finite scores.
  float lse2 = INFINITY;
  if (valid && lim > 0) {
    lse2 = a.lse[out] * kLog2eF;
    if (lse2 == -INFINITY) lse2 = INFINITY;
  }
  if (MODE == kPlain && a.scale < 0.0f) {
#pragma unroll
    for (int i = 0; i < DP / 16; ++i) q[i] = -q[i];
  }
  f32x16 acc[DP / 32] = {};
  FitRange<T> range;
  // The sum of P (dP - D), which D's error alone keeps from 0 (the weights sum
  // to 1): what D is corrected by; and the sum of its terms' sizes.
  float rest[2] = {0.0f, 0.0f}, size = 0.0f;

  const TileReader<DP> rd;
  constexpr int kTile = kTileKeys * DP * 2;
  const int r0 = wave * kGroup;
  const KeySource<DP, kPacked, 1> keys(a, w, hk, to);
  auto stage = [&](int k0, int buf) {
    char SMX_LDS* kt = lds + buf * 2 * kTile + r0 * DP * 2;
    keys.stage(a, keys.k, kt, k0 + r0);
    keys.stage(a, keys.v, kt + kTile, k0 + r0);
  };

  // Weights of 32 keys from dot products; cap: what the cap's derivative takes.
  auto weights = [&](f32x16& s, f32x16& cap, int k0) {
    if constexpr (MODE != kPlain) {
      sc.scores(s, cap, static_cast<float>(pos - k0 - 4 * half), -1.0f);
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
    if (k0 == 0 && lim_all <= kTileKeys) {
      // Rows that see no key past this tile: D from the weights themselves,
      // which o's rounding would put off where few keys share them.
      float sum = 0.0f;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        f32x16 s = rows_dot<T, DP>(rd, kt, 32 * h, q), cap;
        const f32x16 dp = rows_dot<T, DP>(rd, vt, 32 * h, dout);
        weights(s, cap, 32 * h);
#pragma unroll
        for (int i = 0; i < 16; ++i) sum = __builtin_fmaf(s[i], dp[i], sum);
      }
      sum += half32_partner(sum);
      if (lim <= kTileKeys) delta = sum;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      f32x16 s = rows_dot<T, DP>(rd, kt, 32 * h, q), cap;
      f32x16 dp = rows_dot<T, DP>(rd, vt, 32 * h, dout);
      weights(s, cap, k0 + 32 * h);
      const bool two_parts = any_large(s, kLargeWeight);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        dp[i] = s[i] * (dp[i] - delta);
        rest[i % 2] += dp[i];
        size += fabsf(dp[i]);
        if constexpr (MODE >= kCap) dp[i] *= sc.derivative(cap[i]);
      }
      range.fit(dp, acc);
      cols_accumulate<T, DP>(rd, kt, 32 * h, dp, two_parts, acc);
    }
  }
  // D comes from o as it was rounded.  Where that error counts beside the row's
  // score gradients (weights of nearly one key, whose terms all but cancel; values
  // with a large common part), a second pass takes it out of dQ: it subtracts its
  // product with P K.  With scores of a deviation of 30, dQ was off by 4.4 times its
  // own rounding.  2^-19 of the sum of |do o| is what fp32 sums of D leave.
  const float off = (rest[0] + rest[1]) + half32_partner(rest[0] + rest[1]);
  size += half32_partner(size);
  const bool wrong = fabsf(off) > fmaxf(kMostOff<T> * size, 0x1p-19f * around);
  if (lane == 0) redo[wave] = __any(wrong);
  __syncthreads();  // the last tile has been read
  if (redo[0] || redo[1] || redo[2] || redo[3]) {
    // Blocks of weights this small count for nothing, all of them together.
    const float small = kMostOff<T> / 256.0f * size / (fabsf(off) * ((to + 31) / 32));
    auto stage_keys = [&](int k0, int buf) {
      keys.stage(a, keys.k, lds + buf * kTile + r0 * DP * 2, k0 + r0);
    };
    stage_keys(0, 0);
    buf = 0;
    for (int k0 = 0; k0 < to; k0 += kTileKeys, buf ^= 1) {
      staged();
      __syncthreads();
      if (k0 + kTileKeys < to) stage_keys(k0 + kTileKeys, buf ^ 1);
      if (k0 >= lim_any) continue;
      const char SMX_LDS* kt = lds + buf * kTile;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        f32x16 s = rows_dot<T, DP>(rd, kt, 32 * h, q), cap;
        weights(s, cap, k0 + 32 * h);
        if (!any_large(s, small)) continue;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          s[i] *= -off;
          if constexpr (MODE >= kCap) s[i] *= sc.derivative(cap[i]);
        }
        range.fit(s, acc);
        cols_accumulate<T, DP>(rd, kt, 32 * h, s, false, acc);
      }
    }
    __syncthreads();
  }
  delta += off;
  if (valid && half == 0)
    reinterpret_cast<float2*>(a.delta)[static_cast<int64_t>(head) * a.tokens_q + token] =
        make_float2((kWeightLift<T> - lse2) / c, -delta);
  store_rows<T, DP>(lds + wave * 32 * DP * 2, acc, a.scale * range.back(),
                    static_cast<T*>(a.out), valid ? static_cast<int>(out) : -1, a.d);
}

// The turns of a key tile: 32 tokens of one head each, head by head, each from
// the document's last tokens down to the first that sees the tile's first
// key.  Workgroups of different key tiles then read the same rows at the same
// time, and these come from the L2: in ascending order each would start at
// rows of its own.
constexpr int kTurnRows = 32;

struct KeyTurns {
  int last, tiles, turns;  // last token tile; token tiles of a head; turns
};

__device__ __forceinline__ KeyTurns key_turns(const HeadsArgs& a, const DocTile& w, int first) {
  KeyTurns k;
  const int tok0 = a.causal && first >= w.prefix ? max(first - (w.lk - w.lq), 0) : 0;
  k.last = (w.lq + kTurnRows - 1) / kTurnRows - 1;
  k.tiles = tok0 < w.lq ? k.last + 1 - tok0 / kTurnRows : 0;
  k.turns = k.tiles * a.group;
  return k;
}

// Turns per split, the same for the whole call: at least kMinTurns, such that
// the longest document fits the launched splits and the call makes about
// `target` workgroups.  0: not split.
constexpr int kMinTurns = 32;

__device__ __forceinline__ int split_turns(const HeadsArgs& a, const DocLanes& mine) {
  if (a.splits <= 1) return 0;
  auto turns = [&](const DocLanes& x) {
    return x.lk > 0 ? (x.lq + kTurnRows - 1) / kTurnRows * a.group : 0;
  };
  double sum;
  float longest;
  over_docs<false>(
      a, mine,
      [&](const DocLanes& x) {
        return static_cast<double>(turns(x)) * ((x.lk + kTileRows - 1) / kTileRows);
      },
      [&](const DocLanes& x) { return __int2float_ru(turns(x)); }, &sum, &longest);
  const int64_t all = static_cast<int64_t>(a.causal ? sum / 2 : sum) * a.kv_heads;
  const int64_t most = static_cast<int64_t>(longest);
  int64_t chunk = max((all + a.target - 1) / a.target, (most + a.splits - 1) / a.splits);
  chunk = max(chunk, static_cast<int64_t>(kMinTurns));
  return __builtin_amdgcn_readfirstlane(chunk >= most ? 0 : static_cast<int>(chunk));
}

// Splits of a tile's turns: enough for the chunk, and so many that they begin
// with heads (a divisor of the group, or a multiple of it), which keeps the
// tiles' workgroups at the same rows.
__device__ __forceinline__ int turn_splits(const HeadsArgs& a, int turns, int chunk) {
  if (chunk == 0 || turns <= chunk) return 1;
  int count = (turns + chunk - 1) / chunk;
  if (count >= a.group)
    count = (count + a.group - 1) / a.group * a.group;
  else
    while (a.group % count != 0) ++count;
  return min(count, a.splits);
}

// LDS of k_heads_dkv: V of the key tile, and two stages of kTurnRows rows of Q
// and dO.
template <int DP>
constexpr int kKeyLds = (kTileRows + 2 * 2 * kTurnRows) * DP * 2;

// dK and dV, by keys: four products for each pair.  16384 tokens of one
// document: 2.4 ms, 920 TFLOP/s; packed documents of 8192 tokens 190 us (sizes as
// above).  Bound by matrix ops and LDS reads, of which V's are a fifth.  Where a call
// has 64 documents or more every workgroup reads all of their lengths for its
// splits: 8192 tokens in 2048 documents of 4 take 3.8 ms forward and backward.
//
// A wavefront's K operand stays in registers, its V operand in LDS: with both in
// registers (64 at a width of 128, beside 128 of sums and 32 of scores) some
// were spilled, and a reload from scratch waits for the next stage's loads.  The
// instances with a bias, a cap or both still spill 29, 78 and 83 registers there, and
// all of width 256 do: packed documents of 8192 tokens take 717, 750 and 905 us
// forward and backward with them, and 515 without.
template <typename T, int DP, int MODE>
__global__ __launch_bounds__(kTileThreads, DP <= 128 ? 2 : 1) void k_heads_dkv(HeadsArgs a) {
  __shared__ __attribute__((aligned(16))) char lds_bytes[kKeyLds<DP>];
  // Of a stage's rows: -lse / c (what a row's scores start from; scored: -lse
  // in powers of two), and -D (what dP starts from).
  __shared__ __attribute__((aligned(16))) float stats[2][2][kTurnRows];
  char SMX_LDS* lds = (char SMX_LDS*)lds_bytes;
  const int hk = blockIdx.x % a.kv_heads;
  const DocLanes docs = load_docs<false>(a, threadIdx.x % 64);
  const DocTile w = find_tile<kTileRows, false, true>(a, docs, blockIdx.x / a.kv_heads);
  const int first = w.tile * kTileRows;
  if (first >= w.lk) return;
  const KeyTurns kt = key_turns(a, w, first);
  const int chunk = split_turns(a, docs);
  const int splits = turn_splits(a, kt.turns, chunk);
  const bool split = splits > 1;
  if (static_cast<int>(blockIdx.y) >= splits) return;
  const int per = (kt.turns + splits - 1) / splits;
  int turn = static_cast<int>(blockIdx.y) * per;
  const int turns = min(kt.turns, turn + per);

  const int tid = threadIdx.x, lane = tid % 64, half = lane / 32;
  const int wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int key0 = first + 32 * wave;  // of the wavefront
  const int key = key0 + lane % 32;
  const bool valid = key < w.lk;
  const int64_t token = w.k0 + key;
  const float c = Scoring<MODE>(a, 0.0f).unit();

  typedef typename Vec8<T>::type V;
  V k[DP / 16];
  load_operand<T, DP>(k, static_cast<const T*>(a.k.data) + token * a.k.ts + hk * a.k.hs, valid,
                      half, a.d);
  const int d2 = 2 * a.d;
  const char SMX_LDS* vt = lds + 32 * wave * DP * 2;
  Stager<DP>(a.v, 0, w.k0, hk)
      .template packed<32 / Stager<DP>::kRows>(lds + 32 * wave * DP * 2, key0, w.lk, d2);
  if (MODE == kPlain && a.scale < 0.0f) {
#pragma unroll
    for (int i = 0; i < DP / 16; ++i) k[i] = -k[i];
  }
  f32x16 dk[DP / 32] = {}, dv[DP / 32] = {};
  FitRange<T> range;
  constexpr float kRaise = 1 << kWeightLift<T>, kLower = 1.0f / kRaise;

  const TileReader<DP> reader;
  constexpr int kTile = kTurnRows * DP * 2;
  constexpr int N = kTurnRows / 4 / Stager<DP>::kRows;
  const int r0 = wave * (kTurnRows / 4);
  char SMX_LDS* stages = lds + kTileRows * DP * 2;

  float2 stat = {-INFINITY, 0.0f};
  // The head and the first token of the turn to stage next, and of this one.
  const int top = kt.last * kTurnRows, bottom = (kt.last + 1 - kt.tiles) * kTurnRows;
  int next_head = hk * a.group, next_t0 = top;
  if (turn < turns) {
    next_head += turn / kt.tiles;
    next_t0 -= turn % kt.tiles * kTurnRows;
  }
  auto stage = [&](int buf) {
    const int head = next_head, t0 = next_t0;
    next_t0 -= kTurnRows;
    if (next_t0 < bottom) {
      next_t0 = top;
      ++next_head;
    }
    if (wave == 0) {  // before the stage's loads: waiting for it waits for no other
      stat = make_float2(-INFINITY, 0.0f);
      if (lane < kTurnRows && t0 + lane < w.lq)
        stat = reinterpret_cast<const float2*>(
            a.delta)[static_cast<int64_t>(head) * a.tokens_q + w.q0 + t0 + lane];
    }
    char SMX_LDS* qt = stages + buf * 2 * kTile + r0 * DP * 2;
    Stager<DP>(a.q, 0, w.q0, head).template packed<N>(qt, t0 + r0, w.lq, d2, r0);
    Stager<DP>(a.dout, 0, w.q0, head).template packed<N>(qt + kTile, t0 + r0, w.lq, d2,
                                                                     r0);
  };
  auto write_stats = [&](int buf) {
    if (tid < kTurnRows) {
      stats[buf][0][lane] = stat.x;
      stats[buf][1][lane] = stat.y;
    }
  };
  // Four rows' statistics for the registers 4 q .. 4 q + 3.
  auto rows_stat = [&](const float (&x)[kTurnRows]) {
    f32x16 r;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const f32x4 y = *reinterpret_cast<const f32x4*>(&x[8 * q + 4 * half]);
#pragma unroll
      for (int j = 0; j < 4; ++j) r[4 * q + j] = y[j];
    }
    return r;
  };

  int this_head = next_head, this_t0 = next_t0;
  if (turn < turns) {
    stage(0);
    write_stats(0);
  }
  int buf = 0;
  for (; turn < turns; ++turn, buf ^= 1) {
    staged();
    __syncthreads();
    const int head = this_head, t0 = this_t0;
    this_head = next_head;
    this_t0 = next_t0;
    if (turn + 1 < turns) stage(buf ^ 1);
    const char SMX_LDS* qt = stages + buf * 2 * kTile;
    const char SMX_LDS* ot = qt + kTile;
    if (keys_seen(a, w, min(t0 + kTurnRows, w.lq) - 1) > key0) {
      const int lim_all = keys_seen(a, w, t0);
      const TileReader<DP> rd = reader.fresh();
      f32x16 s, cap;
      if constexpr (MODE != kPlain) {
        const Scoring<MODE> sc(a, a.slopes != nullptr ? a.slopes[head] : 0.0f);
        s = rows_dot<T, DP>(rd, qt, 0, k);
        sc.scores(s, cap, static_cast<float>(t0 + 4 * half + w.lk - w.lq - key), 1.0f);
        s += rows_stat(stats[buf][0]);
      } else {
        __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
        s = rows_dot<T, DP>(rd, qt, 0, k, rows_stat(stats[buf][0]));
      }
      f32x16 dp = rows_stat(stats[buf][1]);
#pragma unroll
      for (int st = 0; st < DP / 16; ++st)
        dp = mfma32(rd.template rows<T>(ot, 0, st), rd.template rows<T>(vt, 0, st), dp);
      interleave<DP / 16, 2, 2>();
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(s[i] * c);
      if (lim_all < key0 + 32) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int tok = t0 + 8 * (i / 4) + 4 * half + i % 4;
          if (key >= keys_seen(a, w, tok)) s[i] = 0.0f;
        }
      }
      const bool two_parts = any_large(s, kLargeWeight * kRaise);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        dp[i] *= s[i];
        if constexpr (MODE >= kCap) dp[i] *= Scoring<MODE>::derivative(cap[i]);
      }
      cols_accumulate<T, DP>(rd, ot, 0, s, two_parts, dv);
      range.fit(dp, dk);
      cols_accumulate<T, DP>(rd, qt, 0, dp, two_parts, dk);
    }
    write_stats(buf ^ 1);
  }
  const int64_t row = token * a.kv_heads + hk;
  if (split) {
    if (!valid) return;
    const int64_t rows = static_cast<int64_t>(a.tokens_k) * a.kv_heads;
    float* p = a.part_o + ((2 * static_cast<int64_t>(blockIdx.y)) * rows + row) * a.d;
    store_sums<DP>(p, a.d, half, dk, range.back() * kLower);
    store_sums<DP>(p + rows * a.d, a.d, half, dv, kLower);
    return;
  }
  // The wavefront's own V has landed (also without a turn) and been read: its
  // place turns the rows.
  staged();
  const int index = valid ? static_cast<int>(row) : -1;
  store_rows<T, DP>(lds + 32 * wave * DP * 2, dk, a.scale * range.back() * kLower,
                    static_cast<T*>(a.dk), index, a.d);
  store_rows<T, DP>(lds + 32 * wave * DP * 2, dv, kLower, static_cast<T*>(a.dv), index,
                    a.d);
}

// Sums the splits of a key tile's gradients, in their order: the same bits each
// time.  A tile's rows are shared out over the launch's second axis: by one
// workgroup each, 8192 tokens of 8 key/value heads of 128 in up to four splits
// took 41 us, 16384 tokens of two heads in eight 76; by four 29 and 41, by memory's
// rate.
template <typename T>
__global__ __launch_bounds__(256) void k_heads_sum(HeadsArgs a) {
  const int hk = blockIdx.x % a.kv_heads;
  const DocLanes docs = load_docs<false>(a, threadIdx.x % 64);
  const DocTile w = find_tile<kTileRows, false, true>(a, docs, blockIdx.x / a.kv_heads);
  const int first = w.tile * kTileRows;
  if (first >= w.lk) return;
  const KeyTurns kt = key_turns(a, w, first);
  const int count = turn_splits(a, kt.turns, split_turns(a, docs));
  if (count == 1) return;
  const int64_t rows = static_cast<int64_t>(a.tokens_k) * a.kv_heads;
  const int quads = a.d / 4, keys = min(w.lk - first, kTileRows);
  for (int i = threadIdx.x + 256 * blockIdx.y; i < keys * quads; i += 256 * gridDim.y) {
    const int64_t row = static_cast<int64_t>(w.k0 + first + i / quads) * a.kv_heads + hk;
    const int64_t at = row * a.d + i % quads * 4;
    f32x4 k = {0, 0, 0, 0}, v = {0, 0, 0, 0};
#pragma unroll 4
    for (int s = 0; s < count; ++s) {
      const float* p = a.part_o + 2 * static_cast<int64_t>(s) * rows * a.d + at;
      k += *reinterpret_cast<const f32x4*>(p);
      v += *reinterpret_cast<const f32x4*>(p + rows * a.d);
    }
    store4(static_cast<T*>(a.dk) + at, k * a.scale);
    store4(static_cast<T*>(a.dv) + at, v);
  }
}

}  // namespace smx
