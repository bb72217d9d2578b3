// C ABI of multi-head attention: argument checks and launches.
// Declarations and contract: include/attention_mi355x.h.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "../../include/attention_mi355x.h"
#include "sm_heads.hpp"
#include "sm_heads_bwd.hpp"
#include "sm_heads_f32.hpp"
#include "sm_heads_host.hpp"
#include "sm_heads_launch.hpp"
#include "sm_heads_mfma.hpp"

namespace {

using namespace smx;
using namespace smx_host;

HeadsView view(const softmax_heads_t* t) { return {t->data, t->token_stride, t->head_stride}; }

// Workgroup slots of tiles of T rows (sm_heads.hpp).
int64_t tile_slots(int64_t rows, int64_t docs, int tile) { return rows / tile + docs + 1; }

void set_shape(HeadsArgs* a, int64_t tokens_q, int64_t tokens_k, int64_t heads, int64_t kv_heads,
               int64_t d, int64_t docs, const softmax_score_t* s) {
  a->tokens_q = static_cast<int>(tokens_q);
  a->tokens_k = static_cast<int>(tokens_k);
  a->heads = static_cast<int>(heads);
  a->kv_heads = static_cast<int>(kv_heads);
  a->group = static_cast<int>(heads / kv_heads);
  a->d = static_cast<int>(d);
  a->n = static_cast<int>(docs);
  a->slopes = s->slopes;
  a->prefix = s->prefix;
  a->causal = s->causal;
  a->scale = s->scale;
  a->cap = s->cap;
  a->exp_cap = s->cap > 0.0f ? 2.0f * kLog2eF / s->cap : 0.0f;
}

// Rows (keys) of a workgroup's tile: the kernels' kF32Rows and kTileRows, with
// kF32Threads = kTileThreads threads.
int tile_rows(int dtype) { return dtype == SOFTMAX_F32 ? kF32Rows : kTileRows; }
static_assert(kF32Threads == kTileThreads, "one launch shape");

// Workgroups of kTileThreads threads along a launch's first axis, whose threads
// have to stay below 2^32.
constexpr int64_t kMaxTiles = (int64_t(1) << 32) / kTileThreads - 1;

// Sizes that a call's index arithmetic and its launches, for tiles of `tile` rows,
// hold.
bool sizes_ok(int64_t tokens, int64_t heads, int64_t kv_heads, int64_t docs, int tile) {
  return kv_heads > 0 && heads % kv_heads == 0 && docs >= 0 && docs <= kMaxTiles &&
         tokens <= INT32_MAX / std::max<int64_t>(heads, 1) &&
         tile_slots(tokens * heads / kv_heads, docs, tile) <= kMaxTiles / kv_heads;
}

hipError_t launch2(const void* fn, int64_t x, int64_t y, int block, HeadsArgs* a, hipStream_t s) {
  void* args[] = {a};
  return hipLaunchKernel(fn, dim3(static_cast<uint32_t>(x), static_cast<uint32_t>(y)),
                         dim3(block), args, 0, s);
}

// The fp32 instance of a head width: its columns padded to a multiple of 32
// up to 128 (a matrix op takes 4), then to 192 or 256.
#define SMX_BY_WIDTH_F32(d, ...)                                                   \
  ((d) <= 32    ? SMX_FN(__VA_ARGS__(32))                                          \
   : (d) <= 64  ? SMX_FN(__VA_ARGS__(64))                                          \
   : (d) <= 96  ? SMX_FN(__VA_ARGS__(96))                                          \
   : (d) <= 128 ? SMX_FN(__VA_ARGS__(128))                                         \
   : (d) <= 192 ? SMX_FN(__VA_ARGS__(192)) : SMX_FN(__VA_ARGS__(256)))
#define SMX_FWD_PACKED(DP) k_heads_fwd_f32<DP, false>
#define SMX_FWD_PAGED(DP) k_heads_fwd_f32<DP, true>
#define SMX_DQ(DP) k_heads_dq_f32<DP>
#define SMX_DKV(DP) k_heads_dkv_f32<DP>

const void* packed_fn(int dtype, const HeadsArgs& a) {
  return dtype == SOFTMAX_F32   ? SMX_BY_WIDTH_F32(a.d, SMX_FWD_PACKED)
         : dtype == SOFTMAX_F16 ? heads_fwd_f16(a, kPacked)
                                : heads_fwd_bf16(a, kPacked);
}

const void* paged_fn(int dtype, const HeadsArgs& a) {
  const int where = 1 << a.log_block >= kGroup ? kBlocks : kSmallBlocks;
  return dtype == SOFTMAX_F32   ? SMX_BY_WIDTH_F32(a.d, SMX_FWD_PAGED)
         : dtype == SOFTMAX_F16 ? heads_fwd_f16(a, where)
                                : heads_fwd_bf16(a, where);
}

const void* dq_fn(int dtype, const HeadsArgs& a) {
  return dtype == SOFTMAX_F32   ? SMX_BY_WIDTH_F32(a.d, SMX_DQ)
         : dtype == SOFTMAX_F16 ? heads_dq_f16(a)
                                : heads_dq_bf16(a);
}

const void* dkv_fn(int dtype, const HeadsArgs& a) {
  return dtype == SOFTMAX_F32   ? SMX_BY_WIDTH_F32(a.d, SMX_DKV)
         : dtype == SOFTMAX_F16 ? heads_dkv_f16(a)
                                : heads_dkv_bf16(a);
}

const void* join_fn(int dtype) {
  return dtype == SOFTMAX_F32   ? SMX_FN(k_heads_join<float>)
         : dtype == SOFTMAX_F16 ? SMX_FN(k_heads_join<f16>)
                                : SMX_FN(k_heads_join<bf16>);
}

const void* sum_fn(int dtype) {
  return dtype == SOFTMAX_F16 ? SMX_FN(k_heads_sum<f16>) : SMX_FN(k_heads_sum<bf16>);
}

// Splits of the keys to launch: enough that the call's tiles fill `target`
// workgroups, no more than the longest request has chunks of, at most 64.
constexpr int64_t kMaxSplits = 64;

// Fewest keys of a split: a split costs a workgroup's start and its part of
// the join.  One token over 4001 keys of 8 heads of 128: 19.9 us with 128 keys,
// 16.5 with 256, 17.2 with 512.  Wider heads have one workgroup per CU: 16 tokens
// over 8192 keys of one head of 256 96, 65 and 56 us.
int64_t min_chunk(int64_t d) { return d <= 128 ? 256 : 512; }

struct PagedSplits {
  int64_t splits;  // launched
  int64_t target;  // workgroups that a call aims at
};

PagedSplits paged_splits(int64_t tokens, int64_t heads, int64_t kv_heads, int64_t d,
                         int64_t requests, int64_t max_keys, int64_t cus) {
  // Tiles that the requests have at least.
  const int64_t rows = tokens * (heads / kv_heads);
  const int64_t tiles = std::max<int64_t>(1, std::max(rows / kTileRows, std::min(requests, tokens)));
  // Requests' lengths differ, so a call is split into four times the resident
  // workgroups, which evens them out (64 single tokens over up to 8192 keys 255
  // -> 236 us; 12 beside four chunks of 509 212 -> 207), but for chunks whose
  // tiles fill the device by themselves: their split sums cost more than they
  // even out.
  const int64_t target = 8 * cus;
  const bool fills = rows > 32 * requests && tiles * kv_heads >= 2 * cus;
  const int64_t wanted = fills ? 1 : ceil_div(target, tiles * kv_heads);
  return {std::clamp<int64_t>(std::min(wanted, ceil_div(max_keys, min_chunk(d))), 1, kMaxSplits),
          target};
}

int64_t split_bytes(int64_t splits, int64_t tokens, int64_t heads, int64_t d) {
  return splits <= 1 ? 0 : 16 + splits * tokens * heads * (d * 4 + 16);
}

// Splits of a key tile's rows to launch in the backward pass of 16-bit types:
// enough that the tiles of one long document make kKeyTarget workgroups, and
// no more than its turns allow.
constexpr int kKeyTarget = 2048;

int64_t key_splits(int64_t tokens_q, int64_t tokens_k, int64_t heads, int64_t kv_heads,
                   int dtype) {
  if (dtype == SOFTMAX_F32) return 1;
  const int64_t tiles = std::max<int64_t>(1, ceil_div(tokens_k, kTileRows) * kv_heads);
  const int64_t turns = ceil_div(tokens_q, kTurnRows) * (heads / kv_heads);
  return std::clamp<int64_t>(std::min(ceil_div(kKeyTarget, tiles), turns / kMinTurns), 1, 16);
}

// Workgroups that share a key tile's sum: the sum of one is a few loads behind
// one another, and most tiles of short documents have nothing to sum.
constexpr int kSumParts = 4;

// The backward pass' statistics of every row, in whole 16-byte strips, and
// its split sums.
int64_t stat_bytes(int64_t tokens_q, int64_t heads) { return (tokens_q * heads * 8 + 15) / 16 * 16; }
int64_t part_bytes(int64_t splits, int64_t tokens_k, int64_t kv_heads, int64_t d) {
  return splits <= 1 ? 0 : splits * tokens_k * kv_heads * d * 8;
}

// Workgroups of a join, each of four rows at a time: one that finds nothing
// to join ends at once, but 8192 of them take 12 us to do so.
constexpr int64_t kJoinGrid = 2048;

int current_cus(int64_t* cus) {
  int dev = 0, n = 0;
  const hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return fail_hip(e);
  const int rc = device_cus(dev, &n);
  *cus = n;
  return rc;
}

}  // namespace

extern "C" {

SOFTMAX_API int softmax_packed_attention_fwd(const softmax_heads_t* q, const softmax_heads_t* k,
                                             const softmax_heads_t* v, void* o, float* lse,
                                             const int32_t* cu_q, const int32_t* cu_k,
                                             int64_t docs, const softmax_score_t* score,
                                             int dtype, hipStream_t stream) {
  const int size = dtype_size(dtype);
  int64_t qb = 0, kb = 0, vb = 0;
  if (size == 0 || !score_ok(score) || !heads_ok(q, size, &qb) || !heads_ok(k, size, &kb) ||
      !heads_ok(v, size, &vb))
    return SOFTMAX_ERR_INVALID_ARG;
  if (k->tokens != v->tokens || k->heads != v->heads || k->d != v->d || q->d != k->d ||
      !sizes_ok(q->tokens, q->heads, k->heads, docs, tile_rows(dtype)) ||
      !sizes_ok(k->tokens, q->heads, k->heads, docs, tile_rows(dtype)) || !aligned16(o))
    return SOFTMAX_ERR_INVALID_ARG;
  if (qb == 0) return SOFTMAX_OK;
  const int64_t rows = q->tokens * q->heads;
  const Range inputs[] = {{q->data, qb},
                          {k->data, kb},
                          {v->data, vb},
                          {cu_q, (docs + 1) * 4},
                          {cu_k, (docs + 1) * 4},
                          {score->slopes, score->slopes ? q->heads * 4 : 0},
                          {score->prefix, score->prefix ? docs * 4 : 0}};
  const Range outputs[] = {{o, rows * q->d * size}, {lse, rows * 4}};
  const int rc = check_ranges(inputs, outputs);
  if (rc != SOFTMAX_OK) return rc;
  HeadsArgs a = {};
  set_shape(&a, q->tokens, k->tokens, q->heads, k->heads, q->d, docs, score);
  a.q = view(q);
  a.k = view(k);
  a.v = view(v);
  a.out = o;
  a.lse = lse;
  a.cu_q = cu_q;
  a.cu_k = cu_k;
  const int64_t slots = tile_slots(q->tokens * a.group, docs, tile_rows(dtype));
  const hipError_t e =
      launch2(packed_fn(dtype, a), slots * a.kv_heads, 1, kTileThreads, &a, stream);
  return e == hipSuccess ? SOFTMAX_OK : fail_hip(e);
}

SOFTMAX_API int64_t softmax_packed_attention_bwd_workspace(int64_t tokens_q, int64_t tokens_k,
                                                           int64_t heads, int64_t kv_heads,
                                                           int64_t d, int dtype) {
  if (tokens_q < 0 || tokens_k < 0 || heads < 0 || d < 8 || d > SOFTMAX_HEADS_MAX_DIM ||
      dtype_size(dtype) == 0 || !sizes_ok(tokens_q, heads, kv_heads, 0, tile_rows(dtype)) ||
      !sizes_ok(tokens_k, heads, kv_heads, 0, tile_rows(dtype)))
    return -1;
  return stat_bytes(tokens_q, heads) +
         part_bytes(key_splits(tokens_q, tokens_k, heads, kv_heads, dtype), tokens_k, kv_heads, d);
}

SOFTMAX_API int softmax_packed_attention_bwd(const softmax_heads_t* dout,
                                             const softmax_heads_t* q, const softmax_heads_t* k,
                                             const softmax_heads_t* v, const softmax_heads_t* o,
                                             const float* lse, void* dq, void* dk, void* dv,
                                             const int32_t* cu_q, const int32_t* cu_k,
                                             int64_t docs, const softmax_score_t* score,
                                             int dtype, void* workspace, int64_t workspace_bytes,
                                             hipStream_t stream) {
  const int size = dtype_size(dtype);
  int64_t qb = 0, kb = 0, vb = 0, ob = 0, db = 0;
  if (size == 0 || !score_ok(score) || !heads_ok(q, size, &qb) || !heads_ok(k, size, &kb) ||
      !heads_ok(v, size, &vb) || !heads_ok(o, size, &ob) || !heads_ok(dout, size, &db))
    return SOFTMAX_ERR_INVALID_ARG;
  if (k->tokens != v->tokens || k->heads != v->heads || k->d != v->d || q->d != k->d ||
      o->tokens != q->tokens || o->heads != q->heads || o->d != q->d ||
      dout->tokens != q->tokens || dout->heads != q->heads || dout->d != q->d ||
      !sizes_ok(q->tokens, q->heads, k->heads, docs, tile_rows(dtype)) ||
      !sizes_ok(k->tokens, q->heads, k->heads, docs, tile_rows(dtype)) || !aligned16(dq) ||
      !aligned16(dk) || !aligned16(dv) || !aligned16(workspace))
    return SOFTMAX_ERR_INVALID_ARG;
  const int64_t rows = q->tokens * q->heads, krows = k->tokens * k->heads;
  const int64_t splits = key_splits(q->tokens, k->tokens, q->heads, k->heads, dtype);
  const int64_t need =
      stat_bytes(q->tokens, q->heads) + part_bytes(splits, k->tokens, k->heads, k->d);
  if (workspace_bytes < need) return SOFTMAX_ERR_INVALID_ARG;
  if (rows == 0 && krows == 0) return SOFTMAX_OK;
  const Range inputs[] = {{dout->data, db},
                          {q->data, qb},
                          {k->data, kb},
                          {v->data, vb},
                          {o->data, ob},
                          {lse, rows * 4},
                          {cu_q, (docs + 1) * 4},
                          {cu_k, (docs + 1) * 4},
                          {score->slopes, score->slopes ? q->heads * 4 : 0},
                          {score->prefix, score->prefix ? docs * 4 : 0}};
  const Range outputs[] = {{dq, rows * q->d * size},
                           {dk, krows * k->d * size},
                           {dv, krows * k->d * size},
                           {workspace, need}};
  const int rc = check_ranges(inputs, outputs);
  if (rc != SOFTMAX_OK) return rc;
  HeadsArgs a = {};
  set_shape(&a, q->tokens, k->tokens, q->heads, k->heads, q->d, docs, score);
  a.q = view(q);
  a.k = view(k);
  a.v = view(v);
  a.o = view(o);
  a.dout = view(dout);
  a.out = dq;
  a.dk = dk;
  a.dv = dv;
  a.lse = const_cast<float*>(lse);
  a.delta = static_cast<float*>(workspace);
  a.part_o = a.delta + stat_bytes(q->tokens, q->heads) / 4;
  a.splits = static_cast<int>(splits);
  a.target = kKeyTarget;
  a.cu_q = cu_q;
  a.cu_k = cu_k;
  if (rows > 0) {
    const int64_t slots = tile_slots(q->tokens * a.group, docs, tile_rows(dtype));
    const hipError_t e =
        launch2(dq_fn(dtype, a), slots * a.kv_heads, 1, kTileThreads, &a, stream);
    if (e != hipSuccess) return fail_hip(e);
  }
  if (krows > 0) {
    const int64_t slots = tile_slots(k->tokens, docs, tile_rows(dtype));
    const hipError_t e =
        launch2(dkv_fn(dtype, a), slots * a.kv_heads, splits, kTileThreads, &a, stream);
    if (e != hipSuccess) return fail_hip(e);
    if (splits > 1) {
      const hipError_t f = launch2(sum_fn(dtype), slots * a.kv_heads, kSumParts, 256, &a, stream);
      if (f != hipSuccess) return fail_hip(f);
    }
  }
  return SOFTMAX_OK;
}

SOFTMAX_API int64_t softmax_paged_attention_workspace(int64_t tokens, int64_t heads,
                                                      int64_t kv_heads, int64_t d,
                                                      int64_t requests, int64_t max_keys) {
  if (tokens < 0 || heads < 0 || d < 8 || d > SOFTMAX_HEADS_MAX_DIM || max_keys < 0 ||
      !sizes_ok(tokens, heads, kv_heads, requests, kTileRows))
    return -1;
  int64_t cus = 0;
  if (current_cus(&cus) != SOFTMAX_OK) return -1;
  return split_bytes(paged_splits(tokens, heads, kv_heads, d, requests, max_keys, cus).splits,
                     tokens, heads, d);
}

SOFTMAX_API int softmax_paged_attention_fwd(const softmax_heads_t* q, const softmax_cache_t* k,
                                            const softmax_cache_t* v, const int32_t* block_table,
                                            int64_t table_width, const int32_t* cu_q,
                                            const int32_t* key_lens, int64_t requests,
                                            const softmax_score_t* score, int dtype, void* o,
                                            float* lse, void* workspace, int64_t workspace_bytes,
                                            hipStream_t stream) {
  const int size = dtype_size(dtype);
  int64_t qb = 0, kb = 0, vb = 0;
  if (size == 0 || !score_ok(score) || !heads_ok(q, size, &qb) || !cache_ok(k, size, &kb) ||
      !cache_ok(v, size, &vb) || !same_cache(k, v) || q->d != k->d || table_width < 0 ||
      table_width > kMaxTokens / k->block_size ||
      !sizes_ok(q->tokens, q->heads, k->heads, requests, tile_rows(dtype)) || !aligned16(o) ||
      !aligned16(workspace))
    return SOFTMAX_ERR_INVALID_ARG;
  if (qb == 0) return SOFTMAX_OK;
  int64_t cus = 0;
  int rc = current_cus(&cus);
  if (rc != SOFTMAX_OK) return rc;
  const int64_t max_keys = table_width * k->block_size;
  const auto [splits, target] =
      paged_splits(q->tokens, q->heads, k->heads, q->d, requests, max_keys, cus);
  const int64_t need = split_bytes(splits, q->tokens, q->heads, q->d);
  if (workspace_bytes < need) return SOFTMAX_ERR_INVALID_ARG;
  const int64_t rows = q->tokens * q->heads;
  const Range inputs[] = {{q->data, qb},
                          {k->data, kb},
                          {v->data, vb},
                          {block_table, requests * table_width * 4},
                          {cu_q, (requests + 1) * 4},
                          {key_lens, requests * 4},
                          {score->slopes, score->slopes ? q->heads * 4 : 0},
                          {score->prefix, score->prefix ? requests * 4 : 0}};
  const Range outputs[] = {
      {o, rows * q->d * size}, {lse, lse ? rows * 4 : 0}, {workspace, need}};
  rc = check_ranges(inputs, outputs);
  if (rc != SOFTMAX_OK) return rc;
  HeadsArgs a = {};
  set_shape(&a, q->tokens, 0, q->heads, k->heads, q->d, requests, score);
  a.q = view(q);
  a.k = {k->data, k->token_stride, k->head_stride};
  a.v = {v->data, v->token_stride, v->head_stride};
  a.k_bs = k->block_stride;
  a.v_bs = v->block_stride;
  a.blocks = k->blocks;
  a.max_keys = max_keys;
  a.width = static_cast<int>(table_width);
  a.log_block = log2_of(k->block_size);
  a.table = block_table;
  a.out = o;
  a.lse = lse;
  a.cu_q = cu_q;
  a.cu_k = key_lens;
  a.splits = static_cast<int>(splits);
  a.target = static_cast<int>(target);
  a.min_chunk = static_cast<int>(min_chunk(q->d));
  a.part_head = static_cast<int*>(workspace);
  a.part_stat = reinterpret_cast<SplitStat*>(a.part_head + 4);
  a.part_o = reinterpret_cast<float*>(a.part_stat + splits * rows);
  const int64_t slots = tile_slots(q->tokens * a.group, requests, tile_rows(dtype));
  hipError_t e =
      launch2(paged_fn(dtype, a), slots * a.kv_heads, splits, kTileThreads, &a, stream);
  if (e == hipSuccess && splits > 1)
    e = launch2(join_fn(dtype), std::min<int64_t>(ceil_div(rows, 4), kJoinGrid), 1, 256, &a,
                stream);
  return e == hipSuccess ? SOFTMAX_OK : fail_hip(e);
}

}  // extern "C"
