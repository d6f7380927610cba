/*
 * gns_learn.h -- C ABI of what training and answering need next to the update step of Algorithm 1 (gns_sage_dense in
 * gns.h): the update step in 8-bit integers, its backward pass from activation checkpoints in 8 bits, and log
 * probabilities over the classes with their gradient.
 *
 *   gns_quantize_rows, gns_dense_int8, gns_sage_dense_int8     the update step with 8-bit rows and weights
 *   gns_checkpoint_save, gns_checkpoint_load                   activations kept in 8 bits for the backward pass
 *   gns_sage_dense_backward                                    gradients of weights, bias and input, from checkpoints
 *   gns_log_probs, gns_log_probs_backward                      the loss on given classes, entropy, best classes
 *
 * The general rules of gns.h hold: device pointers unless named host_, the caller owns every buffer, all work is
 * enqueued on hip_stream and no call synchronises or allocates, errors are gns_status codes with a message in
 * gns_last_error(ctx).  From the context these calls take the device's properties, the place for errors, the stage
 * timer and, for num_rows < 0, the counts of its last mini-batch: num_rows may be GNS_DEVICE_COUNTS(i), the dst rows of
 * layer index i, read on the device (buffers must then hold that layer's cap_dst rows; what lies behind the count is
 * not written).  num_rows may be 0, and buffers of rows NULL then.  A workspace for some num_rows serves calls of fewer rows too.  Calls on one context
 * may be enqueued on several streams as long as they do not share a workspace.  Inputs and outputs of a call must not
 * overlap unless the call says so.  Results do not depend on timing: a repeated call gives the same bits.
 */
#ifndef GNS_LEARN_H_
#define GNS_LEARN_H_

#include "gns.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { GNS_FP32 = 0, GNS_BF16 = 1 };
#define GNS_MAX_WIDTH (1 << 22)
#define GNS_MAX_STRIDE (1 << 24)

/* Rows of a matrix on the device: element (r, c) is data[r * stride + c], 0 <= c < width <= GNS_MAX_WIDTH.  width <= stride <=
 * GNS_MAX_STRIDE, in elements; data aligned to the element.  Any width, stride and alignment is taken; rows that begin at
 * multiples of 16 bytes are read and written a little faster. */
typedef struct {
    void* data;
    int64_t stride;
    int32_t width;
    int32_t type; /* GNS_FP32 / GNS_BF16 */
} gns_rows;

/* ---- the update step in 8-bit integers ----------------------------------------------------------------------------
 * Rows in 8 bits: int8[num_rows x GNS_INT8_STRIDE(k)], 16-byte aligned, columns k and beyond zero, with an fp32 scale
 * per row: x[r, c] ~ scale[r] * q[r, c]. */
#define GNS_INT8_STRIDE(k) (((int64_t) (k) + 63) / 64 * 64)
#define GNS_INT8_MAX_K 131072 /* 127 * 127 * k stays below 2^31 */

/* Quantises rows [x1 | x2] (x2 may be NULL; both of one type) of together k <= GNS_INT8_MAX_K columns: a = max |x[r, :]|,
 * scale[r] = a / 127, q[r, c] = x[r, c] * (127 * (1 / a)) rounded to nearest, ties to even, each operation in fp32: half a
 * step off and two roundings at most (halfway between two steps it may be either).  A row whose a is below 2^-120 gets
 * scale 0 and zeros; one with an infinity or NaN gets scale NaN and zeros.  Also the way to quantise weights, given as
 * hdim rows of k (one scale per output channel). */
gns_status gns_quantize_rows(gns_ctx* ctx, const gns_rows* x1, const gns_rows* x2, int8_t* q_dev, float* scale_dev,
                             int32_t num_rows, void* hip_stream);

/* out[r, n] = g( scale[r] * w_scale[n] * sum_c q[r, c] * wq[n, c] + bias[n] ), g = max(0, .) if relu != 0 (a NaN stays
 * one), identity otherwise.  The sum is exact (int32); q and wq are rows in 8 bits as above, wq of out->width rows (its
 * columns k and beyond may hold anything); bias may be NULL; out of either type.  Enqueue only. */
gns_status gns_dense_int8(gns_ctx* ctx, const int8_t* q_dev, const float* scale_dev, int32_t k, const int8_t* wq_dev,
                          const float* w_scale_dev, const float* bias_dev, int32_t relu, const gns_rows* out,
                          int32_t num_rows, void* hip_stream);

/* Both in one call: the update step of gns_sage_dense with rows quantised as they come (x2 may be NULL).  workspace:
 * gns_sage_dense_int8_workspace_bytes(ctx, k, num_rows) bytes, 256-byte aligned, for this call alone while it runs. */
size_t gns_sage_dense_int8_workspace_bytes(const gns_ctx* ctx, int32_t k, int32_t num_rows);
gns_status gns_sage_dense_int8(gns_ctx* ctx, const gns_rows* x1, const gns_rows* x2, const int8_t* wq_dev,
                               const float* w_scale_dev, const float* bias_dev, int32_t relu, const gns_rows* out,
                               int32_t num_rows, void* workspace, size_t workspace_bytes, void* hip_stream);

/* ---- activation checkpoints in 8 bits -----------------------------------------------------------------------------
 * 32 columns of a row share a power of two 2^e, the smallest with which the largest magnitude rounds to 127 steps or
 * fewer:
 *   q_dev          int8[num_rows x 32 * G], G = (width + 31) / 32, 16-byte aligned; columns from width on are zero
 *   exponents_dev  uint8[num_rows x G]: e + 127.  0: all values are zero (magnitudes below 2^-100 are taken as zero);
 *                  255: the group held an infinity or NaN, and all its values are NaN when loaded
 * A value is q * 2^e, rounded to nearest (ties to even), at most half a step off; it is exactly a bf16 value.
 * Magnitudes of 127.5 * 2^121 and more are kept as 127 * 2^121.
 * positive_dev (may be NULL): uint32[num_rows x G], bit j of word g set iff x[r, 32 g + j] > 0: the mask of a ReLU whose
 * output x is. */
gns_status gns_checkpoint_save(gns_ctx* ctx, const gns_rows* x, int8_t* q_dev, uint8_t* exponents_dev,
                               uint32_t* positive_dev, int32_t num_rows, void* hip_stream);
gns_status gns_checkpoint_load(gns_ctx* ctx, const int8_t* q_dev, const uint8_t* exponents_dev, const gns_rows* x,
                               int32_t num_rows, void* hip_stream);

/* The backward pass of gns_sage_dense, out = g([x1 | x2] . W + bias), with x1 (f1 columns) and x2 (f2 columns; f2 may be
 * 0 and its pointers NULL) from their checkpoints:
 *   dz = d_out where bit n of the row's `positive` words (of the output, as gns_checkpoint_save writes them) is set, zero
 *        elsewhere, whatever d_out holds there; positive_dev NULL: dz = d_out
 *   dw[k, n] = sum_r x[r, k] * dz[r, n]     fp32[(f1 + f2) x hdim]
 *   db[n]    = sum_r dz[r, n]               fp32[hdim], or NULL; comes with dw only
 *   dx[r, k] = sum_n dz[r, n] * w[k, n]     rows of f1 + f2 columns, in d_out's type, or NULL; w fp32[(f1 + f2) x hdim]
 * hdim = d_out->width.  dw may be NULL (then neither checkpoint is read).  Products have fp32's precision (fp32 values are
 * split into three bf16 terms), sums are fp32; subnormal bf16 values of d_out may count as zero in them.  Infinities and
 * NaN go where these formulas take them: an infinity stays one unless it meets a zero or its opposite (each such result
 * is summed by a thread alone; a call with very many takes long).  With no rows dw and db are zero.  workspace:
 * gns_sage_dense_backward_workspace_bytes(...) bytes, 256-byte aligned. */
size_t gns_sage_dense_backward_workspace_bytes(const gns_ctx* ctx, int32_t f1, int32_t f2, int32_t hdim, int32_t num_rows);
gns_status gns_sage_dense_backward(gns_ctx* ctx, const gns_rows* d_out, const uint32_t* positive_dev,
                                   const int8_t* q1_dev, const uint8_t* exponents1_dev, int32_t f1,
                                   const int8_t* q2_dev, const uint8_t* exponents2_dev, int32_t f2, const float* w_dev,
                                   float* dw_dev, float* db_dev, const gns_rows* dx, int32_t num_rows, void* workspace,
                                   size_t workspace_bytes, void* hip_stream);

/* ---- log probabilities --------------------------------------------------------------------------------------------
 * For row r of the logits z (C = logits->width classes), p = softmax(z), m = max z, L = log sum_j exp(z_j - m):
 *   logp[r]    = log p of class labels[r]; 0 where labels[r] < 0 (no label); NaN where labels[r] >= C
 *   entropy[r] = -sum_j p_j log p_j
 *   stats[2 r], stats[2 r + 1] = m, L
 *   top_index[r, i], top_logp[r, i], i < top <= GNS_MAX_TOP: the classes of highest log p, highest first, ties to the
 *                lowest index; where fewer than `top` classes are left, -1 and -infinity
 * A class with z = -infinity is masked: p = 0, it adds nothing to the entropy and is no alternative.  A row without any
 * class left has logp = -infinity (if labelled), entropy 0, stats (-infinity, 0) and no alternatives.  A row with a NaN
 * or +infinity has NaN in all fp32 outputs and index -1.  logp and labels go together (both NULL: not wanted); entropy, stats may be
 * NULL; top = 0 with NULL pointers: no alternatives.  Sums are fp32.  workspace: gns_log_probs_workspace_bytes(...) bytes,
 * 256-byte aligned (NULL if that is 0). */
#define GNS_MAX_TOP 32
size_t gns_log_probs_workspace_bytes(const gns_ctx* ctx, int32_t num_classes, int32_t top, int32_t num_rows);
gns_status gns_log_probs(gns_ctx* ctx, const gns_rows* logits, const int32_t* labels_dev, float* logp_dev,
                         float* entropy_dev, float* stats_dev, int32_t top, int32_t* top_index_dev, float* top_logp_dev,
                         int32_t num_rows, void* workspace, size_t workspace_bytes, void* hip_stream);

/* The gradient of sum_r g_logp[r] * logp[r] + g_entropy[r] * entropy[r] with respect to the logits:
 *   d_logits[r, j] = g_logp[r] * ([j = labels[r]] - p_j) - g_entropy[r] * p_j * (log p_j + entropy[r])
 * from the stats and entropy that gns_log_probs wrote.  A row without a label has no first term; rows without any class
 * left get zeros; rows of NaN, or with a label >= C, get NaN; p_j below 2^-126 counts as zero.  Either term may be left
 * out (g_logp or g_entropy NULL; what else the term needs is then not read), not both.  d_logits has the width of the
 * logits, either type, and may be the logits' own rows (same data, stride and type). */
gns_status gns_log_probs_backward(gns_ctx* ctx, const gns_rows* logits, const int32_t* labels_dev, const float* stats_dev,
                                  const float* entropy_dev, const float* g_logp_dev, const float* g_entropy_dev,
                                  const gns_rows* d_logits, int32_t num_rows, void* hip_stream);

/* Stages of gns_profile_begin (see gns.h) for the calls above. */
#define GNS_STAGE_INT8 22       /* gns_quantize_rows, gns_dense_int8, gns_sage_dense_int8 */
#define GNS_STAGE_CHECKPOINT 23 /* gns_checkpoint_save, gns_checkpoint_load               */
#define GNS_STAGE_BACKWARD 24   /* gns_sage_dense_backward                                */
#define GNS_STAGE_LOG_PROBS 25  /* gns_log_probs, gns_log_probs_backward                  */

#ifdef __cplusplus
}
#endif
#endif /* GNS_LEARN_H_ */
