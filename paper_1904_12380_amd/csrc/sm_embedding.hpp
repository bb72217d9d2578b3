// Rows of an embedding table by token, and the table's gradient
// (include/decoder_mi355x.h has the operations).  Both are bound by memory: a
// lookup reads and writes a row per token, the gradient reads a row per token and
// writes the table.
//
// The gradient sorts the tokens by id (a radix sort, digits of kDigit bits, which
// keeps tokens of one id in their order) and sums runs of equal ids:
//
//   k_embed_sort    up to kSortMost tokens: one workgroup sorts them in registers
//                   and LDS, while the others clear the table
//   k_embed_count, k_embed_base, k_embed_move
//                   more tokens: one pass per digit, by tiles of tokens
//   k_embed_sums    chunks of sorted tokens: a run that lies within a chunk is
//                   summed, scaled and written; the ends of runs that cross chunks
//                   go to the workspace
//   k_embed_join    sums the parts of those runs, in order
//
// No atomics: the order of every sum follows from the ids alone.
#pragma once

#include "sm_strips.hpp"

namespace smx {

constexpr int kDigit = 8;
constexpr int kBins = 1 << kDigit;
constexpr int kSortItems = 16;                          // of a thread
constexpr int kSortThreads = 1024;                      // of the workgroup that sorts alone
constexpr int kSortMost = kSortThreads * kSortItems;
constexpr int kMoveThreads = 256;
constexpr int kMoveTile = kMoveThreads * kSortItems;

struct EmbedArgs {
  const int64_t* ids;
  const void* in;       // the table, or dout
  int64_t pitch;        // of its rows, in elements
  void* out;            // rows of d, or the table's gradient
  int tokens, rows, d;
  float scale;
  // Workspace of the gradient.
  unsigned* key[2];     // ids of the sorted tokens (rows: padding), and the tokens
  int* token[2];
  int* bins;            // [kBins, tiles]
  float* part;          // [chunks, 2, d]: sums of a run that began before the chunk, and
                        // of one that goes on behind it
  int tiles, chunk, chunks;
  int passes;           // of the sort
  int64_t clear;        // strips of the table's gradient
};

__device__ __forceinline__ unsigned embed_key(const EmbedArgs& a, int t) {
  const int64_t id = a.ids[t];
  return id >= 0 && id < a.rows ? static_cast<unsigned>(id) : static_cast<unsigned>(a.rows);
}

// kPer strips per thread, all loads issued before the first store.
template <typename T>
__global__ __launch_bounds__(256) void k_embed_rows(EmbedArgs a) {
  constexpr int kN = Strip<T>::kN, kPer = 4;
  const unsigned strips = a.d / kN;
  const int64_t all = static_cast<int64_t>(a.tokens) * strips;
  const int64_t i0 = static_cast<int64_t>(blockIdx.x) * (256 * kPer) + threadIdx.x;
  typename Strip<T>::type v[kPer];
  bool live[kPer];
#pragma unroll
  for (int u = 0; u < kPer; ++u) {
    const int64_t i = i0 + u * 256;
    live[u] = false;
    v[u] = typename Strip<T>::type{};
    if (i < all) {
      const int t = static_cast<int>(row_of(i, strips, all));
      const unsigned key = embed_key(a, t);
      live[u] = key < static_cast<unsigned>(a.rows);
      if (live[u])
        v[u] = Strip<T>::load(static_cast<const T*>(a.in) + key * a.pitch +
                              (i - static_cast<int64_t>(t) * strips) * kN);
    }
  }
#pragma unroll
  for (int u = 0; u < kPer; ++u) {
    const int64_t i = i0 + u * 256;
    if (i >= all) continue;
    float w[kN];
#pragma unroll
    for (int e = 0; e < kN; ++e) w[e] = live[u] ? static_cast<float>(v[u][e]) * a.scale : 0.0f;
    Strip<T>::store(static_cast<T*>(a.out) + i * kN, w);
  }
}

__device__ __forceinline__ void clear_strips(const EmbedArgs& a, int64_t from, int64_t step) {
  f32x4* const out = static_cast<f32x4*>(a.out);
  for (int64_t i = from; i < a.clear; i += step) out[i] = f32x4{};
}

// The places of a wavefront's items by digit, in the order item by item and lane
// by lane; `counts` (its own, cleared) ends as the number of items per digit.  A
// lane's items with live = false have no place.
template <typename F>
__device__ __forceinline__ void rank_items(int (&rank)[kSortItems], int* counts, F digit) {
  const int lane = static_cast<int>(__lane_id());
#pragma unroll
  for (int i = 0; i < kSortItems; ++i) {
    const int x = digit(i);  // -1: none
    uint64_t same = __ballot(x >= 0);
    if (x < 0) same = ~same;
#pragma unroll
    for (int b = 0; b < kDigit; ++b) {
      const uint64_t ones = __ballot(x >> b & 1);
      same &= x >> b & 1 ? ones : ~ones;
    }
    const int before = __popcll(same & ((uint64_t(1) << lane) - 1));
    int base = 0;
    if (x >= 0) base = counts[x];
    // The wavefront's reads of LDS come before its writes: in order, and not
    // moved by the compiler (the addresses may be the same).
    if (x >= 0 && before == 0) counts[x] = base + __popcll(same);
    __builtin_amdgcn_wave_barrier();
    rank[i] = base + before;
  }
}

// One workgroup sorts all tokens; the others clear the table's gradient.
template <int UNUSED>
__global__ __launch_bounds__(kSortThreads) void k_embed_sort(EmbedArgs a) {
  constexpr int kWaves = kSortThreads / 64;
  __shared__ unsigned items[kSortMost];
  __shared__ int counts[kWaves][kBins];
  __shared__ int total[kBins];
  const int tid = threadIdx.x, wave = tid / 64, lane = tid % 64;
  if (blockIdx.x != 0) {
    clear_strips(a, static_cast<int64_t>(blockIdx.x - 1) * kSortThreads + tid,
                 static_cast<int64_t>(gridDim.x - 1) * kSortThreads);
    return;
  }
  unsigned key[kSortItems];
  int token[kSortItems], rank[kSortItems];
  const int at = wave * (64 * kSortItems) + lane;
#pragma unroll
  for (int i = 0; i < kSortItems; ++i) {
    token[i] = at + 64 * i;
    key[i] = token[i] < a.tokens ? embed_key(a, token[i]) : 0xffffffffu;
  }
  for (int p = 0; p < a.passes; ++p) {
    for (int i = tid; i < kWaves * kBins; i += kSortThreads) counts[i / kBins][i % kBins] = 0;
    __syncthreads();
    // Items past the tokens have the largest key, so that they stay last.
    auto digit = [&](int i) { return static_cast<int>(key[i] >> (kDigit * p) & (kBins - 1)); };
    rank_items(rank, counts[wave], digit);
    __syncthreads();
    if (tid < kBins) {
      int sum = 0;
      for (int w = 0; w < kWaves; ++w) {
        const int c = counts[w][tid];
        counts[w][tid] = sum;
        sum += c;
      }
      total[tid] = sum;
    }
    __syncthreads();
    if (wave == 0) {  // sums of the digits before each digit, four to a lane
      int c[kBins / 64], own = 0;
#pragma unroll
      for (int j = 0; j < kBins / 64; ++j) {
        c[j] = own;
        own += total[lane * (kBins / 64) + j];
      }
      int before = own;
#pragma unroll
      for (int s = 1; s < 64; s *= 2) {
        const int o = __shfl_up(before, s);
        if (lane >= s) before += o;
      }
#pragma unroll
      for (int j = 0; j < kBins / 64; ++j) total[lane * (kBins / 64) + j] = before - own + c[j];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kSortItems; ++i) rank[i] += total[digit(i)] + counts[wave][digit(i)];
#pragma unroll
    for (int i = 0; i < kSortItems; ++i) items[rank[i]] = key[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kSortItems; ++i) key[i] = items[at + 64 * i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kSortItems; ++i) items[rank[i]] = static_cast<unsigned>(token[i]);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kSortItems; ++i) token[i] = static_cast<int>(items[at + 64 * i]);
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < kSortItems; ++i)
    if (at + 64 * i < a.tokens) {
      a.key[0][at + 64 * i] = key[i];
      a.token[0][at + 64 * i] = token[i];
    }
}

// Items of a tile by digit.  In the first pass further workgroups clear the table's
// gradient.
template <int UNUSED>
__global__ __launch_bounds__(kMoveThreads) void k_embed_count(EmbedArgs a, int pass) {
  __shared__ int counts[kBins];
  const int tid = threadIdx.x, tile = blockIdx.x;
  if (tile >= a.tiles) {
    clear_strips(a, static_cast<int64_t>(tile - a.tiles) * kMoveThreads + tid,
                 static_cast<int64_t>(gridDim.x - a.tiles) * kMoveThreads);
    return;
  }
  counts[tid] = 0;
  __syncthreads();
  const int end = min(a.tokens - tile * kMoveTile, kMoveTile);
  for (int i = tid; i < end; i += kMoveThreads) {
    const int t = tile * kMoveTile + i;
    const unsigned key = pass == 0 ? embed_key(a, t) : a.key[pass & 1][t];
    atomicAdd(&counts[key >> (kDigit * pass) & (kBins - 1)], 1);
  }
  __syncthreads();
  a.bins[static_cast<int64_t>(tid) * a.tiles + tile] = counts[tid];
}

// Counts by digit and tile to the items before them, by one workgroup.
template <int UNUSED>
__global__ __launch_bounds__(1024) void k_embed_base(EmbedArgs a) {
  __shared__ int sums[16];
  const int tid = threadIdx.x, wave = tid / 64, lane = tid % 64;
  const int64_t all = static_cast<int64_t>(kBins) * a.tiles;
  int before = 0;
  for (int64_t i0 = 0; i0 < all; i0 += 1024) {
    const int64_t i = i0 + tid;
    const int own = i < all ? a.bins[i] : 0;
    int x = own;
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
      const int o = __shfl_up(x, s);
      if (lane >= s) x += o;
    }
    if (lane == 63) sums[wave] = x;
    __syncthreads();
    int all_before = before;
    for (int w = 0; w < 16; ++w) {
      if (w < wave) all_before += sums[w];
      before += sums[w];
    }
    if (i < all) a.bins[i] = all_before + x - own;
    __syncthreads();
  }
}

// Items of a tile to their places by digit.
template <int UNUSED>
__global__ __launch_bounds__(kMoveThreads) void k_embed_move(EmbedArgs a, int pass) {
  constexpr int kWaves = kMoveThreads / 64;
  __shared__ int counts[kWaves][kBins];
  const int tid = threadIdx.x, wave = tid / 64, lane = tid % 64, tile = blockIdx.x;
  const int at = tile * kMoveTile + wave * (64 * kSortItems) + lane;
  unsigned key[kSortItems];
  int token[kSortItems], rank[kSortItems];
#pragma unroll
  for (int i = 0; i < kSortItems; ++i) {
    const int t = at + 64 * i;
    token[i] = t;
    key[i] = 0;
    if (t < a.tokens) {
      key[i] = pass == 0 ? embed_key(a, t) : a.key[pass & 1][t];
      if (pass != 0) token[i] = a.token[pass & 1][t];
    }
  }
  for (int w = 0; w < kWaves; ++w) counts[w][tid] = 0;
  __syncthreads();
  auto digit = [&](int i) {
    return at + 64 * i < a.tokens ? static_cast<int>(key[i] >> (kDigit * pass) & (kBins - 1)) : -1;
  };
  rank_items(rank, counts[wave], digit);
  __syncthreads();
  int sum = a.bins[static_cast<int64_t>(tid) * a.tiles + tile];
  for (int w = 0; w < kWaves; ++w) {
    const int c = counts[w][tid];
    counts[w][tid] = sum;
    sum += c;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kSortItems; ++i) {
    if (digit(i) < 0) continue;
    const int to = rank[i] + counts[wave][digit(i)];
    a.key[~pass & 1][to] = key[i];
    a.token[~pass & 1][to] = token[i];
  }
}

// Sums of the runs in a chunk of sorted tokens.  G lanes take a chunk's G strips
// of columns, kAhead rows of them are loaded at a time.
template <typename T, int G>
__global__ __launch_bounds__(256) void k_embed_sums(EmbedArgs a) {
  constexpr int kN = Strip<T>::kN, kAhead = 8;
  const int strips = a.d / kN, slabs = (strips + G - 1) / G;
  const int64_t unit = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) / G;
  const int c = static_cast<int>(unit / slabs);
  const int strip = static_cast<int>(unit % slabs) * G + threadIdx.x % G;
  if (c >= a.chunks || strip >= strips) return;
  const unsigned* key = a.key[a.passes & 1];
  const int* token = a.token[a.passes & 1];
  const T* in = static_cast<const T*>(a.in) + strip * kN;
  const int64_t from = static_cast<int64_t>(c) * a.chunk;
  const int64_t to = min(from + a.chunk, static_cast<int64_t>(a.tokens));
  const unsigned before = from > 0 ? key[from - 1] : 0xffffffffu;
  const unsigned after = to < a.tokens ? key[to] : 0xffffffffu;
  const unsigned none = static_cast<unsigned>(a.rows);
  float sum[kN] = {};
  unsigned now = key[from];
  bool first = before == now;  // the run began in an earlier chunk
  auto flush = [&](bool goes_on) {
    if (now == none) return;
    if (first || goes_on) {
      float* p = a.part + (static_cast<int64_t>(c) * 2 + (first ? 0 : 1)) * a.d + strip * kN;
#pragma unroll
      for (int e = 0; e < kN; ++e) p[e] = sum[e];
    } else {
#pragma unroll
      for (int e = 0; e < kN; ++e) sum[e] *= a.scale;
      Strip<T>::store(static_cast<T*>(a.out) + static_cast<int64_t>(now) * a.d + strip * kN, sum);
    }
  };
  for (int64_t p = from; p < to; p += kAhead) {
    unsigned k[kAhead];
    typename Strip<T>::type v[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) k[u] = p + u < to ? key[p + u] : none;
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      v[u] = typename Strip<T>::type{};
      if (k[u] != none) v[u] = Strip<T>::load(in + token[p + u] * a.pitch);
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (p + u >= to) continue;
      if (k[u] != now) {
        flush(false);
        now = k[u];
        first = false;
#pragma unroll
        for (int e = 0; e < kN; ++e) sum[e] = 0.0f;
      }
#pragma unroll
      for (int e = 0; e < kN; ++e) sum[e] += static_cast<float>(v[u][e]);
    }
  }
  flush(now == after);
}

// Runs that cross chunks: the chunk in which one began sums its parts.
template <typename T, int G>
__global__ __launch_bounds__(256) void k_embed_join(EmbedArgs a) {
  constexpr int kN = Strip<T>::kN;
  const int strips = a.d / kN, slabs = (strips + G - 1) / G;
  const int64_t unit = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) / G;
  const int c = static_cast<int>(unit / slabs);
  const int strip = static_cast<int>(unit % slabs) * G + threadIdx.x % G;
  if (c + 1 >= a.chunks || strip >= strips) return;
  const unsigned* key = a.key[a.passes & 1];
  const int64_t from = static_cast<int64_t>(c) * a.chunk, to = from + a.chunk;
  const unsigned now = key[to - 1];
  if (now == static_cast<unsigned>(a.rows) || key[to] != now || (from > 0 && key[from - 1] == now))
    return;
  float sum[kN];
  const float* p = a.part + (static_cast<int64_t>(c) * 2 + 1) * a.d + strip * kN;
#pragma unroll
  for (int e = 0; e < kN; ++e) sum[e] = p[e];
  // The last chunk of the run, by bisection: its parts are then independent loads.
  int lo = c + 1, hi = a.chunks - 1;
  while (lo < hi) {
    const int mid = lo + (hi - lo + 1) / 2;
    if (key[static_cast<int64_t>(mid) * a.chunk] == now) lo = mid;
    else hi = mid - 1;
  }
  const float* q = a.part + static_cast<int64_t>(c + 1) * 2 * a.d + strip * kN;
#pragma unroll 4
  for (int i = c + 1; i <= lo; ++i, q += 2 * a.d) {
#pragma unroll
    for (int e = 0; e < kN; ++e) sum[e] += q[e];
  }
#pragma unroll
  for (int e = 0; e < kN; ++e) sum[e] *= a.scale;
  Strip<T>::store(static_cast<T*>(a.out) + static_cast<int64_t>(now) * a.d + strip * kN, sum);
}

}  // namespace smx
