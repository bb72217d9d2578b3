// What the kernels of multi-head attention share (include/attention_mi355x.h
// has the operation): their arguments, the map from workgroups to documents,
// addresses of rows, and the scores.
//
// Rows.  The query heads that share a key/value head are packed as rows: row
// r of a document is the token r / G and the head hk G + r % G of the group
// of G.  A tile of rows then reads each key and value once for the whole
// group, and single tokens still fill a part of a tile.
//
// Documents.  Their lengths are device data, so the host launches for the
// largest number of tiles that any lengths could need: with documents that
// start at the rows s(b), the tiles of T rows of document b take the
// workgroup slots from floor(s(b) / T) + b on.  Slots of different documents
// never meet: floor((s + l) / T) + 1 >= floor(s / T) + ceil(l / T).  A slot's
// document is the last whose first slot is not past it, found by 64-way
// search (one step for fewer than 64 documents).  Tokens past the last document
// are a document of their own, without keys.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sm_device.hpp"

namespace smx {

typedef _Float16 f16;
typedef __bf16 bf16;
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float kLog2eF = 0x1.715476p+0f;
constexpr float kLn2F = 0x1.62e430p-1f;

// Rows of a tensor [tokens, heads, d].
struct HeadsView {
  const void* data;
  int64_t ts, hs;  // strides in elements between tokens and heads
};

// A row's maximum (natural units) and sum over one split of its keys, and the
// number of its splits.
struct SplitStat {
  float m, l;
  int count, pad;
};

struct HeadsArgs {
  HeadsView q, k, v, o, dout;
  void* out;         // o of the forward pass, or dq
  void* dk;
  void* dv;
  float* lse;        // written by the forward pass (may be null), read by the backward
  float* delta;      // D of every query row (backward); 16-bit types: pairs
  const int* cu_q;   // [n + 1]
  const int* cu_k;   // [n + 1]; paged: key_lens [n]
  const float* slopes;
  const int* prefix;
  // Paged cache.
  const int* table;
  int64_t k_bs, v_bs;  // strides between blocks
  int64_t blocks;
  int64_t max_keys;    // table width times block size
  int width, log_block;
  // Splits of the keys (paged).
  int* part_head;        // keys per split, 0: not split
  SplitStat* part_stat;  // [splits, tokens, heads]
  float* part_o;         // [splits, tokens, heads, d]
  int splits;
  int target;          // workgroups that a call aims at
  int min_chunk;       // fewest keys of a split
  int n, tokens_q, tokens_k, heads, kv_heads, group, d;
  int causal;
  float scale, cap;
  float exp_cap;       // 2 log2 e / cap
};

__device__ __forceinline__ int clamp_i(int x, int lo, int hi) {
  return x < lo ? lo : (x > hi ? hi : x);
}

// First token of document b of n (sums in cu, clamped); b == n: the tokens
// past the last document.
__device__ __forceinline__ int doc_start(const int* cu, int b, int tokens) {
  return b == 0 ? 0 : clamp_i(cu[b], 0, tokens);
}

// A document and one of its tiles.
struct DocTile {
  int b;        // document, n for the tokens past the last
  int q0, lq;   // its queries
  int k0, lk;   // its keys (paged: k0 = 0)
  int prefix;   // keys that every query sees
  int tile;     // tile of the document
};

// The last of 0 .. n whose base is at most t (base(0) <= t, not falling).
template <typename F>
__device__ __forceinline__ int last_at_most(int n, int t, F base) {
  int lo = 0, hi = n;
  while (lo < hi) {
    const int step = (hi - lo) / 64 + 1;
    const int b = lo + static_cast<int>(__lane_id()) * step;
    const uint64_t at = __ballot(b <= hi && base(min(b, hi)) <= t);
    const int count = at == 0 ? 1 : 64 - __builtin_clzll(at);
    lo = lo + (count - 1) * step;
    if (step == 1) break;
    hi = min(hi, lo + step - 1);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// The documents that a wavefront's lanes hold, lane b document b: with fewer
// than 64 of them everything about a workgroup's own and about the whole call
// follows from one load of the sums, with no load behind another.
struct DocLanes {
  int q0, lq, k0, lk;
  bool live;  // a document (lane n: the tokens past the last one)
};

template <bool PAGED>
__device__ __forceinline__ DocLanes load_docs(const HeadsArgs& a, int b) {
  DocLanes x = {0, 0, 0, 0, b < a.n};
  if (b > a.n) return x;
  x.q0 = doc_start(a.cu_q, b, a.tokens_q);
  x.lq = max((x.live ? doc_start(a.cu_q, b + 1, a.tokens_q) : a.tokens_q) - x.q0, 0);
  if constexpr (PAGED) {
    if (x.live) x.lk = static_cast<int>(min(static_cast<int64_t>(max(a.cu_k[b], 0)), a.max_keys));
  } else if (x.live) {
    x.k0 = doc_start(a.cu_k, b, a.tokens_k);
    x.lk = max(doc_start(a.cu_k, b + 1, a.tokens_k) - x.k0, 0);
  }
  return x;
}

// The document and tile of workgroup slot t, for tiles of T rows (`group` per
// token) or, BY_KEYS, of T keys.  `mine`: the lanes' documents, where the call
// has fewer than 64.
template <int T, bool PAGED, bool BY_KEYS>
__device__ __forceinline__ DocTile find_tile(const HeadsArgs& a, const DocLanes& mine, int t) {
  const int* cu = BY_KEYS ? a.cu_k : a.cu_q;
  const int tokens = BY_KEYS ? a.tokens_k : a.tokens_q;
  const int group = BY_KEYS ? 1 : a.group;
  auto first = [&](int start, int b) {
    return static_cast<int>(static_cast<int64_t>(start) * group / T) + b;
  };
  DocTile w;
  if (a.n < 64) {
    const int lane = static_cast<int>(__lane_id());
    // The tokens past the last document have queries but no keys, and the
    // keys past it no queries.
    const int start = !BY_KEYS ? mine.q0 : lane < a.n ? mine.k0 : 0;
    int base = first(start, lane);
    if (BY_KEYS && lane == a.n) base = first(doc_start(cu, a.n, tokens), lane);
    const uint64_t at = __ballot(lane <= a.n && base <= t);
    w.b = at == 0 ? 0 : 63 - __builtin_clzll(at);
    w.q0 = __builtin_amdgcn_readlane(mine.q0, w.b);
    w.lq = __builtin_amdgcn_readlane(mine.lq, w.b);
    w.k0 = __builtin_amdgcn_readlane(mine.k0, w.b);
    w.lk = __builtin_amdgcn_readlane(mine.lk, w.b);
    w.tile = t - __builtin_amdgcn_readlane(base, w.b);
  } else {
    w.b = last_at_most(a.n, t, [&](int b) { return first(doc_start(cu, b, tokens), b); });
    const DocLanes x = load_docs<PAGED>(a, w.b);
    w.q0 = __builtin_amdgcn_readfirstlane(x.q0);
    w.lq = __builtin_amdgcn_readfirstlane(x.lq);
    w.k0 = __builtin_amdgcn_readfirstlane(x.k0);
    w.lk = __builtin_amdgcn_readfirstlane(x.lk);
    w.tile = t - first(doc_start(cu, w.b, tokens), w.b);
  }
  if (BY_KEYS && w.b >= a.n) {
    w.k0 = doc_start(a.cu_k, a.n, a.tokens_k);
    w.lk = a.tokens_k - w.k0;
    w.lq = 0;
  }
  w.prefix = a.prefix != nullptr && w.b < a.n ? clamp_i(a.prefix[w.b], 0, w.lk) : 0;
  return w;
}

// Sums f(document) over the call's documents, and takes the largest of g
// (both below 2^53 and 2^24; every wavefront of a call gets the same).
template <bool PAGED, typename F, typename G>
__device__ __forceinline__ void over_docs(const HeadsArgs& a, const DocLanes& mine, F f, G g,
                                          double* sum, float* most) {
  double s = 0.0;
  float m = 0.0f;
  const int lane = static_cast<int>(__lane_id());
  if (a.n < 64) {
    if (mine.live && mine.lq > 0) {
      s = f(mine);
      m = g(mine);
    }
  } else {
    for (int b = lane; b < a.n; b += 64) {
      const DocLanes x = load_docs<PAGED>(a, b);
      if (x.lq <= 0) continue;
      s += f(x);
      m = fmaxf(m, g(x));
    }
  }
  *sum = wave_sum64(s);
  *most = seg_max<64>(m);
}

// Keys that the query `tok` of a document sees: those before this one.
__device__ __forceinline__ int keys_seen(const HeadsArgs& a, const DocTile& w, int tok) {
  if (!a.causal) return w.lk;
  return clamp_i(max(tok + w.lk - w.lq + 1, w.prefix), 0, w.lk);
}

// Splits of the keys (paged).  All chunks of a call have the same length: the
// keys of all of its tiles of ROWS rows over the workgroups that fill the
// device, in whole tiles of 64 keys, at least min_chunk, and such that the
// longest request fits the launched splits.  0: not split.  Every wavefront of
// a call computes the same from the lengths; the first notes it for the join.
template <int ROWS>
__device__ __forceinline__ int split_chunk(const HeadsArgs& a, const DocLanes& mine) {
  if (a.splits <= 1) return 0;
  double sum;
  float longest;  // rounded up to the fp32 above
  over_docs<true>(
      a, mine,
      [&](const DocLanes& x) {
        return static_cast<double>(x.lk) * ((x.lq * a.group + ROWS - 1) / ROWS);
      },
      [](const DocLanes& x) { return __int2float_ru(x.lk); }, &sum, &longest);
  const int64_t all = static_cast<int64_t>(sum) * a.kv_heads;
  const int64_t most = static_cast<int64_t>(longest);
  int64_t chunk = max((all + a.target - 1) / a.target, (most + a.splits - 1) / a.splits);
  chunk = max((chunk + 63) / 64 * 64, static_cast<int64_t>(a.min_chunk));
  const int n = __builtin_amdgcn_readfirstlane(chunk >= most ? 0 : static_cast<int>(chunk));
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) a.part_head[0] = n;
  return n;
}

__device__ __forceinline__ int split_count(int end, int chunk) {
  return max(1, (end + chunk - 1) / chunk);
}

// Keys [from, to) of split `split` of a tile that sees the first `end`; false
// past its last split (a tile without keys has one).
__device__ __forceinline__ bool split_range(int end, int chunk, int split, int* from, int* to) {
  *from = 0;
  *to = end;
  if (chunk == 0) return split == 0;
  if (split > 0 && split * static_cast<int64_t>(chunk) >= end) return false;
  *from = split * chunk;
  *to = min(end, *from + chunk);
  return true;
}

// Key j of request b in a paged cache: its element offset, or -1 where the
// table holds no block of the cache.
__device__ __forceinline__ int64_t paged_row(const HeadsArgs& a, int b, int j, int64_t bs,
                                             int64_t ts) {
  const int id = a.table[static_cast<int64_t>(b) * a.width + (j >> a.log_block)];
  if (id < 0 || id >= a.blocks) return -1;
  return id * bs + (j & ((1 << a.log_block) - 1)) * ts;
}

// lse of a row without a maximum, from its sum: it sees no key (0), or all of its
// scores are NaN and the sum with them.
__device__ __forceinline__ float lse_of_none(float l) { return l == 0.0f ? -INFINITY : l; }

__device__ __forceinline__ float group4_max(float v) {  // over lanes l % 16
  v = fmaxf(v, row16_partner(v));
  return fmaxf(v, half32_partner(v));
}
__device__ __forceinline__ float group4_sum(float v) {
  v = v + row16_partner(v);
  return v + half32_partner(v);
}

}  // namespace smx
