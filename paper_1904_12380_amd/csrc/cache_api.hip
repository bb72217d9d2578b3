// C ABI of the paged cache: argument checks and launches.
// Declarations and contract: include/attention_mi355x.h.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "../../include/attention_mi355x.h"
#include "sm_cache.hpp"
#include "sm_heads_host.hpp"

namespace {

using namespace smx;
using namespace smx_host;

}  // namespace

extern "C" {

SOFTMAX_API int softmax_cache_slots(const int32_t* context_lens, const int32_t* new_lens,
                                    int64_t requests, int32_t* block_table, int64_t table_width,
                                    const int32_t* free_blocks, int64_t capacity,
                                    const int32_t* free_count, int64_t block_size, int32_t* cu_q,
                                    int32_t* key_lens, int64_t* slots, int64_t total,
                                    int32_t* free_left, int32_t* missing, hipStream_t stream) {
  if (requests < 0 || requests > SOFTMAX_CACHE_MAX_REQUESTS || table_width < 0 ||
      table_width > INT32_MAX || capacity < 0 || capacity > INT32_MAX || total < 0 ||
      total > INT32_MAX || log2_of(block_size) < 0)
    return SOFTMAX_ERR_INVALID_ARG;
  const int64_t table_bytes = requests * table_width * 4;
  const Range inputs[] = {{context_lens, requests * 4},
                          {new_lens, requests * 4},
                          {free_blocks, capacity * 4},
                          {free_count, 4}};
  const Range outputs[] = {{block_table, table_bytes}, {cu_q, (requests + 1) * 4},
                           {key_lens, requests * 4},   {slots, total * 8},
                           {free_left, 4},             {missing, 4}};
  int rc = check_ranges(inputs, outputs);
  if (rc != SOFTMAX_OK) return rc;
  SlotArgs a = {};
  a.context = context_lens;
  a.fresh = new_lens;
  a.table = block_table;
  a.free_blocks = free_blocks;
  a.free_count = free_count;
  a.cu_q = cu_q;
  a.key_lens = key_lens;
  a.slots = slots;
  a.free_left = free_left;
  a.missing = missing;
  a.total = total;
  a.capacity = capacity;
  a.n = static_cast<int>(requests);
  a.width = static_cast<int>(table_width);
  a.log_block = log2_of(block_size);
  // One turn of 256 tokens per workgroup, up to a device full of them.
  const int64_t grid = std::clamp<int64_t>(ceil_div(total, kSlotThreads), 1, 1024);
  void* args[] = {&a};
  const hipError_t e = launch(reinterpret_cast<const void*>(&k_cache_slots), grid, kSlotThreads,
                              args, stream);
  return e == hipSuccess ? SOFTMAX_OK : fail_hip(e);
}

SOFTMAX_API int softmax_cache_append(const softmax_heads_t* k, const softmax_heads_t* v,
                                     const softmax_cache_t* k_cache,
                                     const softmax_cache_t* v_cache, const int64_t* slots,
                                     int dtype, hipStream_t stream) {
  const int size = dtype_size(dtype);
  int64_t kb = 0, vb = 0, kcb = 0, vcb = 0;
  if (size == 0 || !heads_ok(k, size, &kb) || !heads_ok(v, size, &vb) ||
      !cache_ok(k_cache, size, &kcb) || !cache_ok(v_cache, size, &vcb))
    return SOFTMAX_ERR_INVALID_ARG;
  if (k->tokens != v->tokens || k->heads != v->heads || k->d != v->d ||
      k->heads != k_cache->heads || k->d != k_cache->d || !same_cache(k_cache, v_cache))
    return SOFTMAX_ERR_INVALID_ARG;
  if (kb == 0 || kcb == 0) return SOFTMAX_OK;
  const Range inputs[] = {{k->data, kb}, {v->data, vb}, {slots, k->tokens * 8}};
  const Range outputs[] = {{k_cache->data, kcb}, {v_cache->data, vcb}};
  // Keys and values of one allocation may interleave: a cache of both.
  if (caches_meet(k_cache, kcb, v_cache, vcb, size)) return SOFTMAX_ERR_INVALID_ARG;
  const int rc = check_ranges(inputs, outputs, true);
  if (rc != SOFTMAX_OK) return rc;
  const int per = 16 / size;
  AppendArgs a = {};
  a.k = static_cast<const uint4*>(k->data);
  a.v = static_cast<const uint4*>(v->data);
  a.k_cache = static_cast<uint4*>(k_cache->data);
  a.v_cache = static_cast<uint4*>(v_cache->data);
  a.slots = slots;
  a.k_ts = k->token_stride / per;
  a.k_hs = k->head_stride / per;
  a.v_ts = v->token_stride / per;
  a.v_hs = v->head_stride / per;
  a.kc_bs = k_cache->block_stride / per;
  a.kc_ts = k_cache->token_stride / per;
  a.kc_hs = k_cache->head_stride / per;
  a.vc_bs = v_cache->block_stride / per;
  a.vc_ts = v_cache->token_stride / per;
  a.vc_hs = v_cache->head_stride / per;
  a.blocks = k_cache->blocks;
  a.per_head = static_cast<int>(k->d / per);
  a.heads = static_cast<int>(k->heads);
  a.log_block = log2_of(k_cache->block_size);
  a.strips = k->tokens * k->heads * a.per_head;
  const int64_t grid = std::min(ceil_div(a.strips, 256), kMaxGrid);
  void* args[] = {&a};
  const hipError_t e =
      launch(reinterpret_cast<const void*>(&k_cache_append), grid, 256, args, stream);
  return e == hipSuccess ? SOFTMAX_OK : fail_hip(e);
}

}  // extern "C"
