/*
 * pase_operators.h - the layers of the computation graphs as operators on one
 * MI355X (gfx950): residual add + layer norm, matrix products grouped by
 * ragged row ranges (one range: a plain product), and the softmax loss over a
 * vocabulary, each with its backward pass.
 *
 * They run a vertex of a graph, or the shard of it that a configuration gives
 * one device, whatever sizes the split leaves; layer costs can be measured with
 * them and passed to pase_override_costs.
 *
 * Conventions:
 *  - Return value: PASE_OK or a pase_status of pase.h; pase_operator_error()
 *    then holds the reason.  On an error other than PASE_ERR_HIP nothing has been
 *    enqueued.
 *  - Every array is device memory of the current device, owned by the caller;
 *    inputs are only read.  Work is enqueued on `stream` (a hipStream_t, NULL =
 *    the null stream) and the call returns without waiting for it.  Nothing is
 *    allocated, copied to the host or kept between calls, so every call can be
 *    captured in a HIP graph.
 *  - Matrices are row major, elements of a row adjacent; ld* is the distance
 *    between rows in elements, at least the row's length.  Pointers need the
 *    alignment of one element only (16 bytes and an ld that keeps it are
 *    faster).
 *  - An array that is both read and written is named in/out; no other input
 *    may overlap an output, except where a function allows it.
 *  - Sums, statistics and products are accumulated in fp32; results are rounded
 *    once to the output's type.  Results do not depend on scheduling: no
 *    floating-point atomics.
 *  - Any row count including 0 is valid.  Sizes beyond a limit: TOO_LARGE.
 */
#ifndef PASE_OPERATORS_H
#define PASE_OPERATORS_H

#include "pase.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { PASE_BF16 = 0, PASE_FP16 = 1, PASE_FP32 = 2 } pase_dtype;

#define PASE_NORM_MAX_WIDTH 16384   /* columns of a layer norm */
#define PASE_MAX_GROUPS 65536       /* groups of a grouped product */

/* Reason of this thread's last failed operator call ("" if none yet). */
const char *pase_operator_error(void);

/* Layer norm of x + residual: z = x + residual, mean and variance (divided by
 * width) of each row of z in fp32, rstd = 1 / sqrt(variance + eps),
 * y = (z - mean) * rstd * gain + bias.
 * dtype: type of x, residual, y and z; param_dtype: type of gain and bias[width],
 * dtype or PASE_FP32.  residual: NULL = none, and z may then be NULL.
 * bias: NULL = none.  mean, rstd: fp32 [rows], written for the backward pass.
 * y and the statistics are those of the sum before z is rounded. */
pase_status pase_layer_norm_forward(int dtype, int param_dtype, uint64_t rows, uint64_t width,
                                    const void *x, uint64_t ldx, const void *residual, uint64_t ldr,
                                    const void *gain, const void *bias, float eps, void *y, uint64_t ldy,
                                    void *z, uint64_t ldz, float *mean, float *rstd, void *stream);

/* Bytes of workspace pase_layer_norm_backward needs. */
pase_status pase_layer_norm_workspace(int dtype, uint64_t rows, uint64_t width, uint64_t *bytes);

/* Backward pass, with h = (z - mean) * rstd and dh = dy * gain:
 * dx = rstd * (dh - avg(dh) - h * avg(dh * h)) + dz, the gradient of both x and
 * residual; dgain = sum over rows of dy * h, dbias = sum over rows of dy, both in
 * param_dtype (either may be NULL).  dz: the gradient that reaches z other than
 * through the norm, or NULL.  dx may be dy or dz.  Rows are summed in a fixed
 * order.  workspace: pase_layer_norm_workspace() bytes, 16-byte aligned. */
pase_status pase_layer_norm_backward(int dtype, int param_dtype, uint64_t rows, uint64_t width,
                                     const void *dy, uint64_t lddy, const void *z, uint64_t ldz,
                                     const void *dz, uint64_t lddz, const void *gain, const float *mean,
                                     const float *rstd, void *dx, uint64_t lddx, void *dgain, void *dbias,
                                     void *workspace, uint64_t workspace_bytes, void *stream);

/* Products grouped by row ranges: group e owns rows offsets[e] .. offsets[e + 1] - 1
 * of x and one matrix w[e] (n x k, row major, all groups adjacent), and
 * y[t] = w[e] x[t] for its rows.  dtype: PASE_BF16 or PASE_FP16, the type of x and
 * w; out_dtype: dtype or PASE_FP32.  offsets: device array of groups + 1 entries,
 * int32 (offsets_64 = 0) or int64 (1), not decreasing, within 0..rows.  They are
 * read on the device only: rows below offsets[0] and from offsets[groups] on
 * belong to no group and get y = 0.  An offset outside 0..rows or below an earlier
 * one is taken as the nearest that keeps the rule. */
pase_status pase_grouped_matmul_forward(int dtype, int out_dtype, uint64_t rows, uint32_t groups,
                                        uint64_t n, uint64_t k, const void *x, uint64_t ldx, const void *w,
                                        const void *offsets, int offsets_64, void *y, uint64_t ldy,
                                        void *stream);

/* Bytes of workspace pase_grouped_matmul_backward needs (0 is possible). */
pase_status pase_grouped_matmul_workspace(int dtype, int grad_dtype, uint64_t rows, uint32_t groups,
                                          uint64_t n, uint64_t k, uint64_t *bytes);

/* Backward pass: dx[t] = w[e]^T dy[t] in dtype (0 for rows of no group) and
 * dw[e] = sum over the rows t of group e of dy[t] x[t]^T in grad_dtype (dtype or
 * PASE_FP32; 0 for a group without rows).  Either output may be NULL and is then
 * not computed; x is read for dw only, w for dx only.  dw: groups x n x k, adjacent.
 * workspace: pase_grouped_matmul_workspace() bytes, 16-byte aligned. */
pase_status pase_grouped_matmul_backward(int dtype, int grad_dtype, uint64_t rows, uint32_t groups,
                                         uint64_t n, uint64_t k, const void *dy, uint64_t lddy,
                                         const void *x, uint64_t ldx, const void *w, const void *offsets,
                                         int offsets_64, void *dx, uint64_t lddx, void *dw, void *workspace,
                                         uint64_t workspace_bytes, void *stream);

/* Softmax loss of rows of logits: lse = log sum_j exp(logits[j]), loss =
 * lse - logits[target], both fp32 [rows].  targets: device array, int32
 * (targets_64 = 0) or int64 (1).  A row whose target is ignore_index has loss 0
 * and lse 0, and its logits are not read.  A logit of -inf masks its class.  A
 * row with every class masked has lse -inf and loss +inf.  A target outside
 * 0..classes-1 that is not ignore_index gives loss NaN.  The loss is formed from the
 * differences to the row's maximum: it does not carry the rounding of lse. */
pase_status pase_softmax_loss_forward(int dtype, uint64_t rows, uint64_t classes, const void *logits,
                                      uint64_t ldl, const void *targets, int targets_64, int64_t ignore_index,
                                      float *loss, float *lse, void *stream);

/* The same, with lse_low [rows]: what the rounding of lse to fp32 left of it (lse + lse_low
 * is the log-sum-exp; 0 for ignored rows and rows with every class masked). */
pase_status pase_softmax_loss_forward_parts(int dtype, uint64_t rows, uint64_t classes, const void *logits,
                                            uint64_t ldl, const void *targets, int targets_64, int64_t ignore_index,
                                            float *loss, float *lse, float *lse_low, void *stream);

/* Loss and gradient in one pass over the logits, for a loss gradient that is
 * known beforehand: dlogits[j] = (exp(logits[j] - lse) - [j = target]) * dloss.
 * dloss: fp32, one a row (dloss_stride 1) or one for all (0).  Ignored rows and
 * rows with every class masked get 0, rows with a target out of range NaN.
 * dlogits may be logits (same ld): each row is read before it is written. */
pase_status pase_softmax_loss_grad(int dtype, uint64_t rows, uint64_t classes, const void *logits,
                                   uint64_t ldl, const void *targets, int targets_64, int64_t ignore_index,
                                   const float *dloss, uint64_t dloss_stride, float *loss, float *lse,
                                   void *dlogits, uint64_t lddl, void *stream);

/* The gradient alone, from the lse of pase_softmax_loss_forward; same rules.  It carries
 * the rounding of lse: exp(logits[j] - lse) is off by up to 2^-24 |lse| of itself. */
pase_status pase_softmax_loss_backward(int dtype, uint64_t rows, uint64_t classes, const void *logits,
                                       uint64_t ldl, const void *targets, int targets_64, int64_t ignore_index,
                                       const float *lse, const float *dloss, uint64_t dloss_stride,
                                       void *dlogits, uint64_t lddl, void *stream);

/* The same without that rounding, from the lse and lse_low of pase_softmax_loss_forward_parts. */
pase_status pase_softmax_loss_backward_parts(int dtype, uint64_t rows, uint64_t classes, const void *logits,
                                             uint64_t ldl, const void *targets, int targets_64, int64_t ignore_index,
                                             const float *lse, const float *lse_low, const float *dloss,
                                             uint64_t dloss_stride, void *dlogits, uint64_t lddl, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* PASE_OPERATORS_H */
