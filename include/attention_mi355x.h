/*
 * attention_mi355x.h -- C ABI of the attention of language models on MI355X
 * (gfx950): packed documents with gradients for training, chunks of new
 * tokens over a paged cache for serving, and the cache's block tables, slot
 * maps and appends.  Part of the library of softmax_mi355x.h, whose return
 * codes, ownership and asynchrony rules hold here too: all memory is the
 * caller's and usable by the current device, work is enqueued on `stream`
 * and the call returns without waiting, nothing is launched on an error
 * (except SOFTMAX_ERR_HIP from a failed launch), no call allocates.
 *
 * The operation, for a query i of a document (or request) with lq queries
 * and lk keys, at position p_i = i + lk - lq among the keys, for the query
 * head h and its key/value head h / (heads / kv_heads):
 *
 *     x_ij = scale * sum_c q_ic k_jc
 *     x_ij = cap * tanh(x_ij / cap)                 if cap > 0
 *     x_ij = x_ij - slopes[h] * |p_i - j|           if slopes
 *     key j is seen if j <= p_i or j < prefix of the document (causal),
 *                   always (not causal)
 *     lse_i = ln sum_{j seen} exp(x_ij)
 *     o_i   = sum_{j seen} exp(x_ij - lse_i) v_j
 *
 * A query that sees no key gets o = 0 and lse = -infinity, and zero
 * gradients.  No clip is applied.  This is the softmax of Sec. 1.1 Eq. (1)
 * of the paper (Sec. 2.3 Fig. 4, no ValueClip) between two products.
 *
 * Types: SOFTMAX_F32, SOFTMAX_F16 or SOFTMAX_BF16 for all tensors of a call;
 * lse and slopes are fp32.  Sums, statistics and gradients accumulate in
 * fp32; with 16-bit types the weights are rounded to the type for the
 * products on the matrix cores (in two parts, which keep 16 bits or more, where
 * one weight's rounding is not averaged over many: in the forward pass the first
 * 64 keys of rows that see at most 128, in the gradients any block with a weight
 * above 1/8).  In the gradients of fp16 weights and score gradients are scaled
 * into the type's range before they are rounded, and back in the sums.  Results are
 * bitwise deterministic.
 *
 * Layout: a tensor [tokens, heads, d] has its d entries contiguous; strides
 * between tokens and heads are in elements and not negative.  d is a
 * multiple of 8 up to SOFTMAX_HEADS_MAX_DIM; the data and all strides are
 * multiples of 16 bytes.
 *
 * Sizes: tokens * heads is below 2^31, and a launch has fewer than 2^24
 * workgroups: with T = 128 (fp32: 64), (tokens * heads / kv_heads / T + documents
 * + 1) * kv_heads < 2^24.
 *
 * Device data is not trusted for addressing: sums outside [0, tokens] are
 * clamped to it, and block ids outside the cache hold no keys.
 */
#ifndef ATTENTION_MI355X_H
#define ATTENTION_MI355X_H

#include "softmax_mi355x.h"

#ifdef __cplusplus
extern "C" {
#endif

#define SOFTMAX_F32 0
#define SOFTMAX_F16 1
#define SOFTMAX_BF16 2

#define SOFTMAX_HEADS_MAX_DIM 256
#define SOFTMAX_HEADS_MAX_STRIDE 8388608 /* elements between tokens */
#define SOFTMAX_MIN_CAP 1e-30f           /* smallest cap but 0 */

/* A tensor [tokens, heads, d] of a call's type. */
typedef struct softmax_heads_t {
  const void* data;
  int64_t tokens;
  int64_t heads;
  int64_t d;
  int64_t token_stride; /* elements */
  int64_t head_stride;  /* elements */
} softmax_heads_t;

/* A paged cache [blocks, block_size, heads, d]: the key or value of slot s is
 * at block s / block_size, row s % block_size.  block_size is a power of two;
 * any strides, so heads may lie before the rows of a block. */
typedef struct softmax_cache_t {
  void* data;
  int64_t blocks;
  int64_t block_size;
  int64_t heads;
  int64_t d;
  int64_t block_stride; /* elements */
  int64_t token_stride; /* elements */
  int64_t head_stride;  /* elements */
} softmax_cache_t;

/* How scores are formed from the dot products. */
typedef struct softmax_score_t {
  float scale;           /* finite */
  float cap;             /* 0: no cap, or SOFTMAX_MIN_CAP and up, finite */
  int32_t causal;        /* 0 or 1 */
  const float* slopes;   /* device, [heads]; NULL: no bias.  Constants: they
                            get no gradient */
  const int32_t* prefix; /* device, [documents]; NULL: none; causal only */
} softmax_score_t;

/*
 * softmax_packed_attention_fwd -- attention of packed documents: document b
 * has the queries cu_q[b] .. cu_q[b + 1] - 1 of q and the keys cu_k[b] ..
 * cu_k[b + 1] - 1 of k and v (self attention: cu_k = cu_q).
 *
 *   q          [tokens_q, heads, d]
 *   k, v       [tokens_k, kv_heads, d]; heads is a multiple of kv_heads
 *   o          [tokens_q, heads, d], contiguous; written
 *   lse        [tokens_q, heads] fp32, contiguous; written
 *   cu_q, cu_k device, [docs + 1] int32, ascending from 0
 *
 * Tokens past the last document get o = 0 and lse = -infinity.  o and lse
 * may not overlap the inputs.  tokens_k is at most 2^30, and its product with heads
 * is bounded like that of tokens_q.
 *
 * NaN and infinity stay in their document: in q they reach their own row's o and
 * lse, in k and v any row of the document (also of one that does not see the key,
 * when both lie in one tile).
 */
SOFTMAX_API int softmax_packed_attention_fwd(const softmax_heads_t* q, const softmax_heads_t* k,
                                             const softmax_heads_t* v, void* o, float* lse,
                                             const int32_t* cu_q, const int32_t* cu_k,
                                             int64_t docs, const softmax_score_t* score,
                                             int dtype, hipStream_t stream);

/* Bytes of workspace that softmax_packed_attention_bwd needs, or -1 for bad
 * sizes: 8 per query row, and fp32 sums of dk and dv for up to 16 splits where
 * there are few key tiles to fill the device. */
SOFTMAX_API int64_t softmax_packed_attention_bwd_workspace(int64_t tokens_q, int64_t tokens_k,
                                                           int64_t heads, int64_t kv_heads,
                                                           int64_t d, int dtype);

/*
 * softmax_packed_attention_bwd -- the gradients of softmax_packed_attention_fwd:
 * with P_ij the weights, D_i = sum_c do_ic o_ic and x' the derivative of the
 * cap (1 - tanh^2, or 1),
 *
 *     dv_j = sum_i P_ij do_i
 *     ds_ij = P_ij (do_i . v_j - D_i) x'_ij scale
 *     dq_i = sum_j ds_ij k_j        dk_j = sum_i ds_ij q_i
 *
 * the sums for dk and dv over all query heads of a key/value head too.
 *
 *   dout       gradient of o, [tokens_q, heads, d]
 *   o, lse     of the forward call.  Weights come from lse, whose fp32 leaves
 *              them off by 2^-23 of the largest score's size: gradients are
 *              meant for scores of up to 10^5, and need not be finite past 10^7
 *   dq, dk, dv contiguous, of the shapes of q, k and v; written in full
 *              (zeros for tokens that no document holds)
 *   workspace  at least softmax_packed_attention_bwd_workspace() bytes of
 *              device memory, 16-byte aligned, for this call alone until the
 *              stream has passed it
 */
SOFTMAX_API int softmax_packed_attention_bwd(const softmax_heads_t* dout,
                                             const softmax_heads_t* q, const softmax_heads_t* k,
                                             const softmax_heads_t* v, const softmax_heads_t* o,
                                             const float* lse, void* dq, void* dk, void* dv,
                                             const int32_t* cu_q, const int32_t* cu_k,
                                             int64_t docs, const softmax_score_t* score,
                                             int dtype, void* workspace, int64_t workspace_bytes,
                                             hipStream_t stream);

/* Bytes of workspace that softmax_paged_attention_fwd needs on the current
 * device for these sizes, or -1 for bad ones.  max_keys is table_width *
 * block_size. */
SOFTMAX_API int64_t softmax_paged_attention_workspace(int64_t tokens, int64_t heads,
                                                      int64_t kv_heads, int64_t d,
                                                      int64_t requests, int64_t max_keys);

/*
 * softmax_paged_attention_fwd -- attention of chunks of new tokens (or of a
 * single one) over a paged cache that already holds their own keys and
 * values: request b has the queries cu_q[b] .. cu_q[b + 1] - 1 of q, the last
 * of its key_lens[b] keys.
 *
 *   q            [tokens, heads, d]
 *   k, v         caches of the same blocks, block_size, heads and d
 *   block_table  device, [requests, table_width] int32: the block that holds
 *                the keys c * block_size .. of a request at column c
 *   cu_q         device, [requests + 1] int32, ascending from 0
 *   key_lens     device, [requests] int32; clamped to table_width * block_size,
 *                which is at most 2^30
 *   o            [tokens, heads, d], contiguous; written
 *   lse          [tokens, heads] fp32, or NULL
 *   workspace    as for softmax_packed_attention_bwd
 *
 * Keys past key_lens are never read, whatever the cache holds there.  Long
 * contexts of few tokens are split over workgroups and joined in a second
 * launch.
 */
SOFTMAX_API int softmax_paged_attention_fwd(const softmax_heads_t* q, const softmax_cache_t* k,
                                            const softmax_cache_t* v, const int32_t* block_table,
                                            int64_t table_width, const int32_t* cu_q,
                                            const int32_t* key_lens, int64_t requests,
                                            const softmax_score_t* score, int dtype, void* o,
                                            float* lse, void* workspace, int64_t workspace_bytes,
                                            hipStream_t stream);

/*
 * softmax_cache_slots -- the bookkeeping of one serving step, on the device:
 * request b holds context_lens[b] tokens and gets new_lens[b] more.
 *
 *   block_table  [requests, table_width] int32; the blocks that the new
 *                tokens need are taken from the free list and written into
 *                it, in the order of the requests and then of the columns
 *   free_blocks  [capacity] int32, a stack of free block ids: the ids are
 *                taken from free_blocks[*free_count - 1] down
 *   free_count   [1] int32, clamped to [0, capacity]
 *   cu_q         [requests + 1] int32; written: sums of new_lens
 *   key_lens     [requests] int32; written: context_lens + new_lens
 *   slots        [total] int64; written: the slot block * block_size + row of
 *                each new token, request by request; -1 past the last one
 *                and for tokens without a block
 *   free_left    [1] int32; written: what is left of free_count
 *   missing      [1] int32; written: blocks that were needed but not had.
 *                Their entries are -1 where the table has them
 *
 * Negative lengths count as 0; sums are meant to stay below 2^31 (past it cu_q,
 * key_lens and missing are not specified).  The work of a call goes by the sizes
 * of its arrays, whatever the lengths.  Written arrays may not overlap each
 * other or the inputs, except that the table is both.  At most
 * SOFTMAX_CACHE_MAX_REQUESTS requests.
 */
#define SOFTMAX_CACHE_MAX_REQUESTS 65536
SOFTMAX_API int softmax_cache_slots(const int32_t* context_lens, const int32_t* new_lens,
                                    int64_t requests, int32_t* block_table, int64_t table_width,
                                    const int32_t* free_blocks, int64_t capacity,
                                    const int32_t* free_count, int64_t block_size, int32_t* cu_q,
                                    int32_t* key_lens, int64_t* slots, int64_t total,
                                    int32_t* free_left, int32_t* missing, hipStream_t stream);

/*
 * softmax_cache_append -- k[t] and v[t] into slot slots[t] of the caches, for
 * every token t; slots outside the cache (-1) are skipped.  Slots of a call
 * are meant to be distinct.  The caches may lie between each other's rows (a
 * tensor of both), but have no element in common.
 *
 *   k, v   [tokens, heads, d];  k_cache, v_cache of the same heads and d
 *   slots  device, [tokens] int64
 */
SOFTMAX_API int softmax_cache_append(const softmax_heads_t* k, const softmax_heads_t* v,
                                     const softmax_cache_t* k_cache,
                                     const softmax_cache_t* v_cache, const int64_t* slots,
                                     int dtype, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* ATTENTION_MI355X_H */
