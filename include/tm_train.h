/*
 * tm_train.h -- the operators of a training step on distances, on AMD MI355X
 * (gfx950): log-probabilities of given labels with the expected distance
 * field under the softmax, and learned biases by buckets of distance, each
 * with its gradient.  Part of libtm_edt.so; status codes, metrics and element
 * types are those of tm_edt.h.
 *
 * Conventions shared by every entry point:
 *   - Memory: pointers are DEVICE pointers owned by the caller, except shape,
 *     stride, offset and sampling arrays, which are HOST pointers read during
 *     the call.  Nothing is allocated.  Outputs are written completely and may
 *     overlap nothing else (TM_ERR_ALIAS).  Elements are aligned to their own
 *     size; no wider alignment is asked for (16-byte rows are faster).
 *   - Streams: all work is enqueued on `stream` of the current device; calls
 *     are reentrant, and calls that can run at the same time must not share a
 *     workspace or outputs.
 *   - Results depend on the inputs alone: the order of every sum is fixed by
 *     the sizes, so two calls give the same bits.
 *   - Errors: every function returns a tm_status; arguments are checked on
 *     the host before any HIP call and a rejected call enqueues nothing.
 *     A request with no elements is TM_OK and enqueues nothing, but for a
 *     table's gradient over no elements, which is written as zeros.
 */
#ifndef TM_TRAIN_H
#define TM_TRAIN_H

#include "tm_edt.h"

#ifdef __cplusplus
extern "C" {
#endif

enum {
    TM_METRIC_OFFSET = 3,         /* relative biases of rank 1: the signed offset key - query */
    TM_LABEL_MAX_TOP = 32,        /* most alternatives tm_label_logp reports */
    TM_LABEL_MAX_RECOMPUTE = 32,  /* most classes whose gradient needs no out_stats */
    TM_BIAS_MAX_BUCKETS = 256
};

/*
 * tm_label_logp -- log-probabilities of given labels.
 *
 * At each of outer * inner positions, over its classes c with logits x_c, with
 * l_c = x_c - log sum exp x and p_c = exp l_c:
 *
 *   out_logp     l_y of the position's label y; 0 where y lies outside
 *                [0, classes) (an element without a label)
 *   out_entropy  - sum_c p_c l_c
 *   out_mean     sum_c p_c field_c, the expected field (the boundary loss,
 *                for the signed distance field of each class)
 *   out_top, out_index  l and number of the top_k classes with the largest
 *                logits, in falling order; equal logits by rising number
 *   out_stats    a reference near the largest logit and the log of the sum of
 *                exp(x - it), for tm_label_logp_grad
 *
 * A class with p_c = 0 adds nothing to the entropy and to the mean, whatever
 * its logit and field hold there.  Where every logit is -inf, log-probabilities
 * are -inf and the entropy, the mean and the gradient 0.  Where one is NaN or
 * +inf, the position's float results are NaN (out_logp stays 0 without a label)
 * and its out_index is any class.
 * All arithmetic is float32.
 *
 *   logits   dtype TM_DTYPE_F32, _F16 or _BF16; element (o, c, i) lies at
 *            o strides[0] + c strides[1] + i strides[2] (elements, >= 0).
 *   labels   [outer][inner] contiguous, label_dtype TM_DTYPE_U8 (read
 *            unsigned), _I32 or _I64; NULL only if out_logp is.
 *   field    float32 with its own strides (0 repeats a value), or NULL.
 *   out_logp, out_entropy, out_mean  [outer][inner] float32, each may be NULL.
 *   out_top float32, out_index int32: [outer][top_k][inner]; both or neither.
 *   out_stats  [outer][inner][2] float32, or NULL.
 *   workspace  at least tm_label_logp_workspace_size() bytes (0 for most
 *            requests), 8-byte aligned; needs no initialisation.
 *
 * Errors: TM_ERR_SHAPE (classes < 1, negative extent or stride), TM_ERR_NULL,
 * TM_ERR_NO_OUTPUT, TM_ERR_DTYPE, TM_ERR_UNSUPPORTED (top_k outside [0,
 * min(classes, TM_LABEL_MAX_TOP)]), TM_ERR_TOO_LARGE (2^31 positions or
 * classes), TM_ERR_WORKSPACE, TM_ERR_ALIAS, TM_ERR_HIP.
 */
int tm_label_logp(const void *logits, int dtype, int64_t outer, int64_t classes, int64_t inner,
                  const int64_t *strides, const void *labels, int label_dtype, const float *field,
                  const int64_t *field_strides, int top_k, float *out_logp, float *out_entropy, float *out_mean,
                  float *out_top, int32_t *out_index, float *out_stats, void *workspace, size_t workspace_bytes,
                  hipStream_t stream);
size_t tm_label_logp_workspace_size(int dtype, int64_t outer, int64_t classes, int64_t inner,
                                    const int64_t *strides, int top_k);

/*
 * tm_label_logp_grad -- the logits' gradient, given the upstream gradients of
 * out_logp, out_entropy and out_mean (a, h, f; each may be NULL, not all):
 *
 *   a (1[c = y] - p_c) - h p_c (l_c + entropy) + f p_c (field_c - mean)
 *
 * with a = 0 where there is no label.  out_grad has the logits' type and its
 * own strides, in which no two elements may coincide.  stats, entropy and mean
 * are what tm_label_logp gave (entropy with up_entropy, mean with up_mean);
 * with at most TM_LABEL_MAX_RECOMPUTE classes they are computed anew from the
 * logits and may be NULL.
 * Errors: as tm_label_logp.
 */
int tm_label_logp_grad(const void *logits, int dtype, int64_t outer, int64_t classes, int64_t inner,
                       const int64_t *strides, const void *labels, int label_dtype, const float *field,
                       const int64_t *field_strides, const float *stats, const float *entropy, const float *mean,
                       const float *up_logp, const float *up_entropy, const float *up_mean, void *out_grad,
                       const int64_t *grad_strides, hipStream_t stream);

/*
 * tm_distance_bias -- a learned bias by buckets of a distance field:
 *
 *   out[b][h][p] = add[b][h][p] + table[bucket(distances[b][p])][h]
 *
 * bucket(d) is the number of edges <= d, a NaN distance falling into bucket 0;
 * edges are buckets - 1 ascending float32 values, table is [buckets][heads]
 * contiguous.  distances: float32, or int32 read as float32, [batch][positions]
 * contiguous.  add (NULL: nothing is added) and out are [batch][heads]
 * [positions] of out_dtype; the sum is made in float32 and rounded once.
 * table_dtype and out_dtype: TM_DTYPE_F32, _F16 or _BF16.
 * Errors: TM_ERR_SHAPE (buckets outside [1, TM_BIAS_MAX_BUCKETS], heads < 1,
 * negative extents), TM_ERR_NULL, TM_ERR_NO_OUTPUT, TM_ERR_DTYPE,
 * TM_ERR_TOO_LARGE (2^31 positions or samples, more than 2^16 heads),
 * TM_ERR_ALIAS, TM_ERR_HIP.
 */
int tm_distance_bias(const void *distances, int distance_dtype, int64_t batch, int64_t positions, const void *table,
                     int table_dtype, int buckets, int64_t heads, const float *edges, const void *add, void *out,
                     int out_dtype, hipStream_t stream);

/*
 * tm_relative_bias -- the same bias by the distance between a query's and a
 * key's position on a grid:
 *
 *   out[b][h][q][k] = add[b][h][q][k] + table[bucket(D(q, k))][h]
 *
 * Queries and keys are the positions of grids of ndim <= 8 axes with extents
 * query_shape and key_shape, in row-major order; queries begin at query_offset
 * (NULL: 0).  With delta_a = key_a - query_a, D is the signed delta_0
 * (TM_METRIC_OFFSET, ndim 1 only), sqrt(sum (s_a delta_a)^2), sum |s_a delta_a|
 * or max |s_a delta_a|, in float32 with every operation rounded, axes in
 * order.  sampling: NULL (ones) or ndim spacings, each rounded to float32.
 * batch samples share the bias; add NULL needs batch <= 1 (else TM_ERR_SHAPE).
 * Errors: as tm_distance_bias, TM_ERR_NDIM, TM_ERR_METRIC, TM_ERR_SAMPLING;
 * TM_ERR_TOO_LARGE also for offsets or extents beyond 2^30.
 */
int tm_relative_bias(int ndim, const int64_t *query_shape, const int64_t *key_shape, const int64_t *query_offset,
                     int metric, const double *sampling, int64_t batch, const void *table, int table_dtype,
                     int buckets, int64_t heads, const float *edges, const void *add, void *out, int out_dtype,
                     hipStream_t stream);

/*
 * tm_distance_bias_grad, tm_relative_bias_grad -- the table's gradient:
 *
 *   out_grad[k][h] = sum of grad[b][h][p] over the b, p in bucket k
 *
 * grad: [batch][heads][positions] of grad_dtype; out_grad: [buckets][heads]
 * of table_dtype, summed in float32 and rounded once: some 4096 sums (512 for
 * 128 heads and more) over shares of b and p in series, added together.  An
 * infinity or NaN reaches its own bucket and head only.  workspace: at least
 * tm_bias_grad_workspace_size() bytes, 16-byte aligned, no initialisation.
 * Errors: as the forward calls, and TM_ERR_WORKSPACE.
 */
int tm_distance_bias_grad(const void *distances, int distance_dtype, int64_t batch, int64_t positions,
                          const void *grad, int grad_dtype, int buckets, int64_t heads, const float *edges,
                          void *out_grad, int table_dtype, void *workspace, size_t workspace_bytes,
                          hipStream_t stream);
int tm_relative_bias_grad(int ndim, const int64_t *query_shape, const int64_t *key_shape,
                          const int64_t *query_offset, int metric, const double *sampling, int64_t batch,
                          const void *grad, int grad_dtype, int buckets, int64_t heads, const float *edges,
                          void *out_grad, int table_dtype, void *workspace, size_t workspace_bytes,
                          hipStream_t stream);
size_t tm_bias_grad_workspace_size(int buckets, int64_t heads);

#ifdef __cplusplus
}
#endif

#endif /* TM_TRAIN_H */
