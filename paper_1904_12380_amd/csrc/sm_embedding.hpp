// Rows of an embedding table by token, and the table's gradient
// (include/decoder_mi355x.h has the operations).  Both are bound by memory: a
// lookup reads and writes a row per token, the gradient reads a row per token and
// writes the table.
//
// The gradient sorts the tokens by id, tokens of one id in their order, and sums runs
// of equal ids:
//
//   k_embed_sort    tiles of kTile tokens, each sorted by a workgroup in registers and
//                   LDS (a radix sort, digits of kDigit bits); further workgroups
//                   clear the table
//   k_embed_merge   up to kMergeMost tokens: a token's place among all is its place in
//                   its own tile and, by bisection, in every other one
//   k_embed_count, k_embed_base, k_embed_move
//                   more tokens: the radix sort over all of them, a pass per digit
//   k_embed_sums    chunks of sorted tokens: a run that lies within a chunk is
//                   summed, scaled and written; the ends of runs that cross chunks
//                   go to the workspace
//   k_embed_join    sums the parts of those runs, in order
//
// 16384 tokens x 50001 x 2048 of bf16: lookup 26 us (4.9 TB/s); sort beside the clearing
// 34 (6.1 TB/s), merge 9, sums 30, join 10.
//
// No atomics but in counts: the order of every sum follows from the ids alone.
#pragma once

#include "sm_strips.hpp"

namespace smx {

constexpr int kDigit = 9;
constexpr int kBins = 1 << kDigit;
constexpr int kSortThreads = 256;
constexpr int kSortItems = 4;  // of a thread
constexpr int kTile = kSortThreads * kSortItems;
constexpr int kMergeMost = 32 * kTile;
constexpr int kMoveItems = 16;
constexpr int kMoveTile = kSortThreads * kMoveItems;

struct EmbedArgs {
  const int64_t* ids;
  const void* in;       // the table, or dout
  int64_t pitch;        // of its rows, in elements
  void* out;            // rows of d, or the table's gradient
  int tokens, rows, d;
  float scale;
  // Workspace of the gradient.
  unsigned* key[2];     // ids of tokens in order (rows: padding), and the tokens
  int* token[2];
  int sorted;           // which of the two is
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
// by lane; `counts` (its own, cleared) ends as the number of items per digit.  An item
// of digit -1 has no place.
template <int ITEMS, typename F>
__device__ __forceinline__ void rank_items(int (&rank)[ITEMS], int* counts, F digit) {
  const int lane = static_cast<int>(__lane_id());
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const int x = digit(i);
    uint64_t same = __ballot(x >= 0);
#pragma unroll
    for (int b = 0; b < kDigit; ++b) {
      const uint64_t ones = __ballot(x >> b & 1);
      same &= x >> b & 1 ? ones : ~ones;
    }
    const int before = __popcll(same & ((uint64_t(1) << lane) - 1));
    int base = 0;
    if (x >= 0) base = counts[x];
    // The first of the lanes with a digit counts them.  A wavefront's reads and
    // writes of LDS take place in order.
    if (x >= 0 && before == 0) counts[x] = base + __popcll(same);
    __builtin_amdgcn_wave_barrier();
    rank[i] = base + before;
  }
}

constexpr int kSortWaves = kSortThreads / 64;

// Tiles of tokens, each sorted by id.  The workgroups behind them clear the table's
// gradient.
template <int UNUSED>
__global__ __launch_bounds__(kSortThreads) void k_embed_sort(EmbedArgs a, int tiles, int to) {
  __shared__ unsigned keys[kTile];
  __shared__ int tokens[kTile];
  __shared__ int counts[kSortWaves][kBins];
  __shared__ int total[kSortWaves];
  const int tid = threadIdx.x, wave = tid / 64, lane = tid % 64;
  if (static_cast<int>(blockIdx.x) >= tiles) {
    clear_strips(a, static_cast<int64_t>(blockIdx.x - tiles) * kSortThreads + tid,
                 static_cast<int64_t>(gridDim.x - tiles) * kSortThreads);
    return;
  }
  unsigned key[kSortItems];
  int token[kSortItems], rank[kSortItems];
  const int first = blockIdx.x * kTile, at = wave * (64 * kSortItems) + lane;
#pragma unroll
  for (int i = 0; i < kSortItems; ++i) {
    token[i] = first + at + 64 * i;
    // Items past the tokens have the largest key, and are behind others of it.
    key[i] = token[i] < a.tokens ? embed_key(a, token[i]) : 0xffffffffu;
  }
  for (int p = 0; p < a.passes; ++p) {
    for (int i = tid; i < kSortWaves * kBins; i += kSortThreads) counts[i / kBins][i % kBins] = 0;
    __syncthreads();
    auto digit = [&](int i) { return static_cast<int>(key[i] >> (kDigit * p) & (kBins - 1)); };
    rank_items(rank, counts[wave], digit);
    __syncthreads();
    // A thread's two digits: the items before them, over digits and wavefronts.
    static_assert(kBins == 2 * kSortThreads, "two digits a thread");
    int own[2] = {0, 0};
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int w = 0; w < kSortWaves; ++w) {
        const int c = counts[w][2 * tid + j];
        counts[w][2 * tid + j] = own[j];
        own[j] += c;
      }
    int before = own[0] + own[1];
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
      const int o = __shfl_up(before, s);
      if (lane >= s) before += o;
    }
    if (lane == 63) total[wave] = before;
    __syncthreads();
    before -= own[0] + own[1];
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) before += w < wave ? total[w] : 0;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
      counts[w][2 * tid] += before;
      counts[w][2 * tid + 1] += before + own[0];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kSortItems; ++i) {
      rank[i] += counts[wave][digit(i)];
      keys[rank[i]] = key[i];
      tokens[rank[i]] = token[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kSortItems; ++i) {
      key[i] = keys[at + 64 * i];
      token[i] = tokens[at + 64 * i];
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < kSortItems; ++i)
    if (first + at + 64 * i < a.tokens) {
      a.key[to][first + at + 64 * i] = key[i];
      a.token[to][first + at + 64 * i] = token[i];
    }
}

// Sorted tiles (key[1], token[1]) to one order (key[0], token[0]): before a token come
// those of smaller ids, and those of its own id in earlier tiles.  Eight lanes take a
// token, each every eighth tile: a bisection is a chain of loads, and a lane's up to
// four are independent (16384 tokens: 36 us with one lane for all tiles, 8.8 so).
constexpr int kMergeLanes = 8;
template <int UNUSED>
__global__ __launch_bounds__(kSortThreads) void k_embed_merge(EmbedArgs a, int tiles) {
  constexpr int kEach = kMergeMost / kTile / kMergeLanes;
  const int at = blockIdx.x * (kSortThreads / kMergeLanes) + threadIdx.x / kMergeLanes;
  const int e = min(at, a.tokens - 1);
  const int own = e / kTile, part = threadIdx.x % kMergeLanes;
  const unsigned key = a.key[1][e];
  int lo[kEach], hi[kEach];
#pragma unroll
  for (int u = 0; u < kEach; ++u) {
    const int j = part + u * kMergeLanes;
    lo[u] = 0;
    hi[u] = j < tiles && j != own ? min(a.tokens - j * kTile, kTile) : 0;
  }
  static_assert(kTile == 1 << 10, "steps of a bisection");
  for (int step = 0; step <= 10; ++step) {
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
      const int j = part + u * kMergeLanes, mid = (lo[u] + hi[u]) / 2;
      if (lo[u] >= hi[u]) continue;
      const unsigned other = a.key[1][j * kTile + mid];
      if (other < key || (other == key && j < own)) lo[u] = mid + 1;
      else hi[u] = mid;
    }
  }
  int before = 0;
#pragma unroll
  for (int u = 0; u < kEach; ++u) before += lo[u];
#pragma unroll
  for (int s = 1; s < kMergeLanes; s *= 2) before += __shfl_xor(before, s);
  if (part == 0 && at < a.tokens) {
    const int to = e - own * kTile + before;
    a.key[0][to] = key;
    a.token[0][to] = a.token[1][e];
  }
}

// Items of a tile by digit.
template <int UNUSED>
__global__ __launch_bounds__(kSortThreads) void k_embed_count(EmbedArgs a, int pass) {
  __shared__ int counts[kBins];
  const int tid = threadIdx.x, tile = blockIdx.x;
  if (tile >= a.tiles) {
    clear_strips(a, static_cast<int64_t>(tile - a.tiles) * kSortThreads + tid,
                 static_cast<int64_t>(gridDim.x - a.tiles) * kSortThreads);
    return;
  }
  for (int b = tid; b < kBins; b += kSortThreads) counts[b] = 0;
  __syncthreads();
  const int end = min(a.tokens - tile * kMoveTile, kMoveTile);
  for (int i = tid; i < end; i += kSortThreads) {
    const int t = tile * kMoveTile + i;
    const unsigned key = pass == 0 ? embed_key(a, t) : a.key[pass & 1][t];
    atomicAdd(&counts[key >> (kDigit * pass) & (kBins - 1)], 1);
  }
  __syncthreads();
  for (int b = tid; b < kBins; b += kSortThreads)
    a.bins[static_cast<int64_t>(b) * a.tiles + tile] = counts[b];
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
__global__ __launch_bounds__(kSortThreads) void k_embed_move(EmbedArgs a, int pass) {
  __shared__ int counts[kSortWaves][kBins];
  const int tid = threadIdx.x, wave = tid / 64, lane = tid % 64, tile = blockIdx.x;
  const int at = tile * kMoveTile + wave * (64 * kMoveItems) + lane;
  unsigned key[kMoveItems];
  int token[kMoveItems], rank[kMoveItems];
#pragma unroll
  for (int i = 0; i < kMoveItems; ++i) {
    const int t = at + 64 * i;
    token[i] = t;
    key[i] = 0;
    if (t < a.tokens) {
      key[i] = pass == 0 ? embed_key(a, t) : a.key[pass & 1][t];
      if (pass != 0) token[i] = a.token[pass & 1][t];
    }
  }
  for (int i = tid; i < kSortWaves * kBins; i += kSortThreads) counts[i / kBins][i % kBins] = 0;
  __syncthreads();
  auto digit = [&](int i) {
    return at + 64 * i < a.tokens ? static_cast<int>(key[i] >> (kDigit * pass) & (kBins - 1)) : -1;
  };
  rank_items(rank, counts[wave], digit);
  __syncthreads();
  for (int b = tid; b < kBins; b += kSortThreads) {
    int sum = a.bins[static_cast<int64_t>(b) * a.tiles + tile];
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
      const int c = counts[w][b];
      counts[w][b] = sum;
      sum += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kMoveItems; ++i) {
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
  const unsigned* key = a.key[a.sorted];
  const int* token = a.token[a.sorted];
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
  // Ids and tokens are loaded a turn ahead of the rows.
  unsigned k[kAhead], k_next[kAhead];
  int t_next[kAhead];
  auto ahead = [&](int64_t p) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int64_t at = min(p + u, to - 1);
      k_next[u] = p + u < to ? key[at] : none;
      t_next[u] = token[at];
    }
  };
  ahead(from);
  for (int64_t p = from; p < to; p += kAhead) {
    typename Strip<T>::type v[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      k[u] = k_next[u];
      v[u] = typename Strip<T>::type{};
      if (k[u] != none) v[u] = Strip<T>::load(in + t_next[u] * a.pitch);
    }
    ahead(p + kAhead);
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
  const unsigned* key = a.key[a.sorted];
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
