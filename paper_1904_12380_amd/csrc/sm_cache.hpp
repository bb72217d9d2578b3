// The paged cache of keys and values: slots for a step's new tokens, and their
// append (include/attention_mi355x.h).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace smx {

constexpr int kSlotThreads = 256;

struct SlotArgs {
  const int* context;
  const int* fresh;   // new tokens of each request
  int* table;
  const int* free_blocks;
  const int* free_count;
  int* cu_q;
  int* key_lens;
  int64_t* slots;
  int* free_left;
  int* missing;
  int64_t total, capacity;
  int n, width, log_block;
};

// A request's lengths and the blocks that it takes: columns [first, last).
struct SlotRequest {
  int64_t context, fresh, first, last, wanted;
};

__device__ __forceinline__ SlotRequest slot_request(const SlotArgs& a, int b) {
  SlotRequest r;
  r.context = max(a.context[b], 0);
  r.fresh = max(a.fresh[b], 0);
  const int64_t up = (int64_t(1) << a.log_block) - 1;
  const int64_t from = (r.context + up) >> a.log_block;
  const int64_t to = (r.context + r.fresh + up) >> a.log_block;
  const int64_t width = a.width;
  r.wanted = to - from;
  r.first = min(from, width);
  r.last = min(to, width);
  return r;
}

// One launch.  Every workgroup forms the running sums of new tokens and of
// blocks over all requests by itself (a thread sums n / 256 consecutive
// requests, then a scan over the threads), so none waits for another; the
// tokens are then shared out, 256 a turn.  A token finds its request by binary
// search over the threads' sums in LDS and a walk over that thread's
// requests.  The token at a block's first row writes the block's table entry:
// every new block starts with a new token, so each entry has one writer, and
// entries that are read (blocks held before) are never written.  Where there are
// more tokens than slots to write, the entries are shared out by themselves: the
// turns are then bounded by the outputs' sizes, not by lengths that the device's
// data holds.
// Bound by latency: 8 requests of one token 3.9 us, 2048 of up to 320 (65536
// tokens) 9.0 us, of a call of 11.7 and 12.5.
__global__ __launch_bounds__(kSlotThreads) void k_cache_slots(SlotArgs a) {
  __shared__ int64_t tokens_before[kSlotThreads + 1], blocks_before[kSlotThreads];
  __shared__ int64_t wave_sums[3][kSlotThreads / 64];
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  const int per = (a.n + kSlotThreads - 1) / kSlotThreads;
  const int begin = min(a.n, tid * per), end = min(a.n, begin + per);
  int64_t sum[3] = {0, 0, 0};  // tokens, blocks, blocks wanted
  for (int b = begin; b < end; ++b) {
    const SlotRequest r = slot_request(a, b);
    sum[0] += r.fresh;
    sum[1] += r.last - r.first;
    sum[2] += r.wanted;
  }
  int64_t scan[3];
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    int64_t x = sum[i];
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
      const int64_t y = __shfl_up(x, o);
      if (lane >= o) x += y;
    }
    if (lane == 63) wave_sums[i][wave] = x;
    scan[i] = x - sum[i];
  }
  __syncthreads();
  int64_t all[3] = {0, 0, 0};
#pragma unroll
  for (int w = 0; w < kSlotThreads / 64; ++w) {
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      if (w < wave) scan[i] += wave_sums[i][w];
      all[i] += wave_sums[i][w];
    }
  }
  tokens_before[tid] = scan[0];
  blocks_before[tid] = scan[1];
  const int64_t count = min(static_cast<int64_t>(max(*a.free_count, 0)), a.capacity);
  if (blockIdx.x == 0) {
    int64_t at = scan[0];
    for (int b = begin; b < end; ++b) {
      const SlotRequest r = slot_request(a, b);
      a.cu_q[b] = static_cast<int>(at);
      a.key_lens[b] = static_cast<int>(r.context + r.fresh);
      at += r.fresh;
    }
    if (tid == 0) {
      const int64_t taken = min(all[1], count);
      a.cu_q[a.n] = static_cast<int>(all[0]);
      *a.free_left = static_cast<int>(count - taken);
      *a.missing = static_cast<int>(all[2] - taken);
    }
  }
  __syncthreads();
  // The last thread whose sum is at most x.  Threads without tokens (or blocks)
  // share their sum with the next that has some: the last of them holds x.
  auto holder = [](const int64_t* before, int64_t x) {
    int lo = 0, hi = kSlotThreads - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if (before[mid] <= x)
        lo = mid;
      else
        hi = mid - 1;
    }
    return lo;
  };
  const int64_t turn0 = static_cast<int64_t>(blockIdx.x) * kSlotThreads + tid;
  const int64_t step = static_cast<int64_t>(gridDim.x) * kSlotThreads;
  const bool by_blocks = all[0] > a.total;
  for (int64_t t = turn0; t < a.total; t += step) {
    int64_t slot = -1;
    if (t < all[0]) {
      const int lo = holder(tokens_before, t);
      int64_t token = tokens_before[lo], block = blocks_before[lo];
      int b = lo * per;
      SlotRequest r = slot_request(a, b);
      while (token + r.fresh <= t) {
        token += r.fresh;
        block += r.last - r.first;
        r = slot_request(a, ++b);
      }
      const int64_t pos = r.context + t - token;
      const int64_t col = pos >> a.log_block, row = pos & ((1 << a.log_block) - 1);
      if (col < a.width) {
        int* entry = a.table + static_cast<int64_t>(b) * a.width + col;
        int id;
        if (col >= r.first) {
          const int64_t k = block + col - r.first;
          id = k < count ? a.free_blocks[count - 1 - k] : -1;
          if (row == 0 && !by_blocks) *entry = id;
        } else {
          id = *entry;
        }
        if (id >= 0) slot = (static_cast<int64_t>(id) << a.log_block) + row;
      }
    }
    a.slots[t] = slot;
  }
  if (!by_blocks) return;
  for (int64_t k = turn0; k < all[1]; k += step) {
    const int lo = holder(blocks_before, k);
    int64_t block = blocks_before[lo];
    int b = lo * per;
    SlotRequest r = slot_request(a, b);
    while (block + r.last - r.first <= k) {
      block += r.last - r.first;
      r = slot_request(a, ++b);
    }
    a.table[b * static_cast<int64_t>(a.width) + r.first + k - block] =
        k < count ? a.free_blocks[count - 1 - k] : -1;
  }
}

struct AppendArgs {
  const uint4 *k, *v;      // tensors [tokens, heads, d], in 16-byte strips
  uint4 *k_cache, *v_cache;
  const int64_t* slots;
  int64_t k_ts, k_hs, v_ts, v_hs;                     // strips
  int64_t kc_bs, kc_ts, kc_hs, vc_bs, vc_ts, vc_hs;   // strips
  int64_t blocks;
  int64_t strips;          // of all tokens
  int per_head, heads, log_block;
};

// One strip of a key and of its value per thread and turn: neighbouring lanes
// take neighbouring strips of a row, so that both sides move whole lines.  Bound
// by memory: 16384 tokens of 8 heads of 128 (134 MB in all) 21.9 us, 6.1 TB/s;
// 64 tokens 3-5 us, the launch.
__global__ __launch_bounds__(256) void k_cache_append(AppendArgs a) {
  const unsigned per_head = a.per_head, heads = a.heads;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < a.strips;
       i += static_cast<int64_t>(gridDim.x) * 256) {
    const int64_t rest = i / per_head;
    const unsigned s = static_cast<unsigned>(i - rest * per_head);
    const int64_t t = rest / heads;
    const unsigned h = static_cast<unsigned>(rest - t * heads);
    const int64_t slot = a.slots[t];
    const int64_t block = slot >> a.log_block;
    if (slot < 0 || block >= a.blocks) continue;
    const int64_t row = slot & ((int64_t(1) << a.log_block) - 1);
    const uint4 x = a.k[t * a.k_ts + h * a.k_hs + s];
    const uint4 y = a.v[t * a.v_ts + h * a.v_hs + s];
    a.k_cache[block * a.kc_bs + row * a.kc_ts + h * a.kc_hs + s] = x;
    a.v_cache[block * a.vc_bs + row * a.vc_ts + h * a.vc_hs + s] = y;
  }
}

}  // namespace smx
