/*
 * decoder_mi355x.h -- C ABI of what a decoder has around its attention on MI355X
 * (gfx950), with gradients for training: the loss of hidden states against a
 * vocabulary, rows of an embedding table, and the norm of rows.  Part of the
 * library of softmax_mi355x.h, whose return codes, ownership and asynchrony
 * rules hold here too: all memory is the caller's and usable by the current
 * device, work is enqueued on `stream` and the call returns without waiting,
 * nothing is launched on an error (except SOFTMAX_ERR_HIP from a failed
 * launch), no call allocates.
 *
 * Types: SOFTMAX_F32, SOFTMAX_F16 or SOFTMAX_BF16 (attention_mi355x.h) for all
 * tensors of a call but those declared fp32 here.  Sums and statistics are held
 * in fp32 or more, and results rounded once.  Results are bitwise deterministic.
 *
 * Layout: rows of d entries side by side; d is a multiple of 8 up to
 * SOFTMAX_MAX_WIDTH.  Rows and tokens are at most 2^29.  Strides between rows are in
 * elements, not negative, and with the data multiples of 16 bytes.  What a call writes is contiguous, and overlaps
 * neither its inputs nor anything else that it writes.  Where there are no rows,
 * pointers may be null.
 *
 * Workspaces are device memory, 16-byte aligned, of at least the bytes that the
 * call's _workspace function gives, for that call alone until the stream has passed
 * it.
 */
#ifndef DECODER_MI355X_H
#define DECODER_MI355X_H

#include "attention_mi355x.h"

#ifdef __cplusplus
extern "C" {
#endif

#define SOFTMAX_MAX_WIDTH 16384
#define SOFTMAX_MAX_ROW_STRIDE 1048576 /* elements between rows of a weight or table */

/* Bytes of workspace of softmax_linear_nll_fwd, or -1 for bad sizes. */
SOFTMAX_API int64_t softmax_linear_nll_fwd_workspace(int64_t rows, int64_t vocab, int64_t d,
                                                     int dtype);

/*
 * softmax_linear_nll_fwd -- the negative log-likelihood of each row's label under
 * the softmax of its logits, which are its products with the rows of a weight and
 * are not kept:
 *
 *     l_tv   = sum_c x_tc w_vc
 *     lse_t  = ln sum_v exp(l_tv)
 *     loss_t = lse_t - l_t,labels[t]
 *
 *   x       [rows, d], rows x_stride apart
 *   weight  [vocab, d], rows w_stride apart (at most SOFTMAX_MAX_ROW_STRIDE)
 *   labels  device, [rows] int64
 *   ignore  the label of rows without a loss: they get loss = lse = 0, whatever
 *           their x holds
 *   loss    [rows] fp32; written.  NaN for a label that is neither `ignore` nor in
 *           [0, vocab), as from softmax_nll_fwd
 *   lse     [rows] fp32; written
 *
 * This is softmax_nll_fwd of x weight^T without a clip: the row softmax of the
 * paper's Sec. 1.1 Eq. (1) behind the product that makes its logits.  A row whose
 * logits hold NaN or +infinity has no finite loss.  vocab is at most 2^29, and of
 * rows x vocab, rows x d and vocab x d each has fewer than 2^23 - 64 tiles of 256 x 256
 * (fp32: 2^24 - 64 of 128 x 128).
 */
SOFTMAX_API int softmax_linear_nll_fwd(const void* x, int64_t x_stride, const void* weight,
                                       int64_t w_stride, const int64_t* labels, int64_t rows,
                                       int64_t vocab, int64_t d, int64_t ignore, int dtype,
                                       float* loss, float* lse, void* workspace,
                                       int64_t workspace_bytes, hipStream_t stream);

/* Bytes of workspace of softmax_linear_nll_bwd, or -1 for bad sizes.  A piece of
 * the vocabulary's gradients of logits is in it, not all of them. */
SOFTMAX_API int64_t softmax_linear_nll_bwd_workspace(int64_t rows, int64_t vocab, int64_t d,
                                                     int dtype);

/*
 * softmax_linear_nll_bwd -- the gradients of softmax_linear_nll_fwd, its logits
 * formed again:
 *
 *     g_tv  = dloss_t (exp(l_tv - lse_t) - [v = labels[t]])
 *     dx_t  = sum_v g_tv w_v        dweight_v = sum_t g_tv x_t
 *
 *   dloss      [rows] fp32, the gradient of loss (lse gets none)
 *   loss, lse  of the forward call with the same x, weight, labels and ignore.
 *              lse's fp32 leaves g off by 2^-24 of its size: gradients are meant
 *              for logits of up to 10^5
 *   dx         [rows, d], or NULL; zeros for ignored rows
 *   dweight    [vocab, d], or NULL
 *
 * With 16-bit types g is rounded to the type for the products on the matrix cores.
 * It is formed relative to the largest finite |dloss|, and with fp16 2^14 times as
 * large: entries below 2^-28 of that are held in fewer than 11 bits there.
 *
 * A label outside the vocabulary that is not `ignore` makes the gradients of its
 * row, and dweight, NaN.
 */
SOFTMAX_API int softmax_linear_nll_bwd(const float* dloss, const void* x, int64_t x_stride,
                                       const void* weight, int64_t w_stride,
                                       const int64_t* labels, int64_t rows, int64_t vocab,
                                       int64_t d, int64_t ignore, int dtype, const float* loss,
                                       const float* lse, void* dx, void* dweight,
                                       void* workspace, int64_t workspace_bytes,
                                       hipStream_t stream);

/*
 * softmax_embedding_fwd -- rows of a table: out_t = scale * table[ids[t]].
 *
 *   ids    device, [tokens] int64; an id outside [0, rows), such as -1, is padding
 *          and gets zeros
 *   table  [rows, d], rows table_stride apart (at most SOFTMAX_MAX_ROW_STRIDE)
 *   out    [tokens, d], at most 2^38 - 2^14 bytes; written
 *   scale  finite
 */
SOFTMAX_API int softmax_embedding_fwd(const int64_t* ids, int64_t tokens, const void* table,
                                      int64_t table_stride, int64_t rows, int64_t d, float scale,
                                      int dtype, void* out, hipStream_t stream);

/* Bytes of workspace of softmax_embedding_bwd, or -1 for bad sizes. */
SOFTMAX_API int64_t softmax_embedding_bwd_workspace(int64_t tokens, int64_t rows, int64_t d,
                                                    int dtype);

/*
 * softmax_embedding_bwd -- the gradient of softmax_embedding_fwd:
 * dtable_v = scale * sum over the tokens t with ids[t] = v of dout_t, summed in
 * fp32 in an order that only the ids set.
 *
 *   dout    [tokens, d], rows dout_stride apart
 *   dtable  [rows, d]; written in full (zeros for rows that no token has)
 */
SOFTMAX_API int softmax_embedding_bwd(const void* dout, int64_t dout_stride, const int64_t* ids,
                                      int64_t tokens, int64_t rows, int64_t d, float scale,
                                      int dtype, void* dtable, void* workspace,
                                      int64_t workspace_bytes, hipStream_t stream);

/*
 * softmax_layer_norm_fwd -- rows brought to mean 0 and variance 1 (center = 1) or
 * to mean square 1 (center = 0), then scaled and moved by column:
 *
 *     mean_t = sum_c x_tc / d                          (0 without center)
 *     rstd_t = (sum_c (x_tc - mean_t)^2 / d + eps)^(-1/2)
 *     y_tc   = (x_tc - mean_t) rstd_t weight_c + bias_c
 *
 *   x       [rows, d], rows x_stride apart
 *   weight  [d], or NULL for ones;  bias  [d], or NULL for zeros
 *   eps     finite, not negative
 *   y       [rows, d]; written
 *   mean    [rows] fp32, written; NULL exactly where center = 0
 *   rstd    [rows] fp32; written
 *
 * The sums over a row are held in fp32: where one of them is past its range (entries
 * from 10^17 on) rstd is 0 or NaN, and where all squares are below it (entries under
 * 10^-19, which only matters with eps = 0) rstd is infinite.
 */
SOFTMAX_API int softmax_layer_norm_fwd(const void* x, int64_t x_stride, const void* weight,
                                       const void* bias, int64_t rows, int64_t d, float eps,
                                       int center, int dtype, void* y, float* mean, float* rstd,
                                       hipStream_t stream);

/* Bytes of workspace of softmax_layer_norm_bwd, or -1 for bad sizes. */
SOFTMAX_API int64_t softmax_layer_norm_bwd_workspace(int64_t rows, int64_t d, int dtype);

/*
 * softmax_layer_norm_bwd -- the gradients of softmax_layer_norm_fwd: with h_tc =
 * (x_tc - mean_t) rstd_t and g_tc = dy_tc weight_c,
 *
 *     dx_tc     = rstd_t (g_tc - sum_c g_tc / d - h_tc sum_c g_tc h_tc / d)
 *                 (without center: no sum of g alone)
 *     dweight_c = sum_t dy_tc h_tc        dbias_c = sum_t dy_tc
 *
 *   dy          [rows, d], rows dy_stride apart
 *   mean, rstd  of the forward call; mean NULL: without center
 *   dx          [rows, d], or NULL
 *   dweight, dbias  [d], or NULL
 */
SOFTMAX_API int softmax_layer_norm_bwd(const void* dy, int64_t dy_stride, const void* x,
                                       int64_t x_stride, const void* weight, const float* mean,
                                       const float* rstd, int64_t rows, int64_t d, int dtype,
                                       void* dx, void* dweight, void* dbias, void* workspace,
                                       int64_t workspace_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* DECODER_MI355X_H */
