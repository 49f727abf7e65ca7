/*
 * p2_train.h -- the local ends of a planned reduction, on one GPU.
 *
 * p2.h plans how the sums over the axes of a training job are made on a hierarchical system.  The calls here
 * compute what a device contributes to such a sum and what it does with the result:
 *  - layer norm, forward and backward: the gradients of weight and bias are sums over the device's rows, the local
 *    stage of the reduction over the data axis;
 *  - the balance of a router over experts: counts and probability sums per expert are sums over the device's
 *    tokens; the loss of the whole batch and its gradient need them reduced in between, hence three calls;
 *  - orthogonalised updates: a reduced weight gradient goes through Newton-Schulz products, which need the whole
 *    matrix on the device.
 *
 * Conventions (those of p2.h, except where this says otherwise)
 *  - Every function returns an int32 status: P2_OK or a negative error; p2_last_error() returns the text.
 *  - Every pointer to data is a DEVICE pointer, aligned to its element type; `stream` is a hipStream_t or NULL.
 *    A call checks its arguments, queues its kernels on the stream and returns; it neither waits nor allocates,
 *    so it may be captured into a graph.  Outputs must not overlap inputs or each other, except where a call says so.
 *  - Workspaces are the caller's: *_workspace gives the bytes (0: NULL will do), the pointer is aligned to 256.  A workspace may be
 *    used again as soon as the call's kernels are done; two streams need two.  Nothing in it outlives a call.
 *  - Rows are contiguous; `*_stride` is the distance between rows in elements and may be larger than the row.
 *  - Element types: P2_F32, P2_BF16, P2_F16.  Sums, statistics and products are accumulated in 32 bits or more
 *    and rounded once, when a result is written; where that is not so the call says so.
 *  - The same inputs give the same bits on every call: no result depends on the order of atomic additions.
 */
#ifndef P2_TRAIN_H
#define P2_TRAIN_H

#include <stdint.h>

#include "p2.h"

#ifdef __cplusplus
extern "C" {
#endif

#define P2_F32 0
#define P2_BF16 1
#define P2_F16 2

#define P2_MAX_EXPERTS 1024   /* experts of one router                              */
#define P2_MAX_CHOSEN 64      /* experts that one token may choose                  */

/* y = (x - mean) * rstd * weight + bias for each row of `cols` values (>= 1): mean and variance over the row (the
 * variance of all `cols` values, from squares of what is centred on the mean before its rounding), rstd = 1 / sqrt(variance + eps), eps >= 0.  `type` is that of x
 * and y, `weight_type` that of weight and bias; either may be NULL (1 and 0).  mean and rstd (NULL, or [rows]) are what the
 * backward pass needs.  y may be x (same stride).  rows = 0 writes nothing. */
int32_t p2_layer_norm_forward(const void* x, int32_t type, int64_t x_stride, const void* weight, const void* bias,
                              int32_t weight_type, int64_t rows, int64_t cols, double eps, void* y, int64_t y_stride,
                              float* mean, float* rstd, void* stream);

int32_t p2_layer_norm_backward_workspace(int64_t rows, int64_t cols, int64_t* bytes);

/* With xh = (x - mean) * rstd and g = dy * weight:  dx = rstd * (g - mean(g) - xh * mean(g * xh)) over each row,
 * dweight = sum over rows of dy * xh, dbias = sum over rows of dy.  dy, x and dx have `type`; weight (NULL: 1), dweight
 * and dbias have `weight_type`.  dx, dweight and dbias may each be NULL: not asked for.  dx may be dy (same stride).
 * rows = 0 writes zeros to dweight and dbias.  workspace may be NULL when neither of these is asked for. */
int32_t p2_layer_norm_backward(const void* dy, int64_t dy_stride, const void* x, int64_t x_stride, int32_t type,
                               const void* weight, int32_t weight_type, const float* mean, const float* rstd, int64_t rows,
                               int64_t cols, void* dx, int64_t dx_stride, void* dweight, void* dbias, void* workspace,
                               int64_t workspace_bytes, void* stream);

int32_t p2_balance_forward_workspace(int64_t tokens, int32_t experts, int64_t* bytes);

/* Routes each token to the k experts with the largest logits (ties: the lowest index; NaN counts as larger than every
 * number; an expert whose logit is -inf is never chosen) and sums up what the balance loss needs.
 *   expert[t][i] = i-th best expert of token t, gate[t][i] = its probability under the softmax over all experts; where a
 *   token has fewer than k experts on offer the rest is -1 and 0.
 *   counts[e] = how often expert e was chosen, prob_sum[e] = its probability summed over tokens, kept[0] = tokens that
 *   count.  A token counts unless keep[t] is 0 (keep may be NULL) or all its logits are -inf: such a token chooses
 *   nothing and its logits are not looked at.
 *   loss[0] = experts / (k * kept^2) * sum_e counts[e] * prob_sum[e]; 0 where no token counts.  1 when the choices and
 *   the probabilities are spread evenly.
 * 1 <= k <= min(experts, P2_MAX_CHOSEN). */
int32_t p2_balance_forward(const void* logits, int32_t type, int64_t stride, const uint8_t* keep, int64_t tokens,
                           int32_t experts, int32_t k, int32_t* expert, float* gate, int64_t* counts, float* prob_sum,
                           int64_t* kept, float* loss, void* workspace, int64_t workspace_bytes, void* stream);

/* The loss above from statistics that have been summed over devices. */
int32_t p2_balance_loss(const int64_t* counts, const float* prob_sum, const int64_t* kept, int32_t experts, int32_t k,
                        float* loss, void* stream);

/* Gradient of  dloss * loss + sum dgate * gate  with respect to the logits (the choice itself has none):
 *   u_e = dloss * experts / (k * kept^2) * counts[e] + sum over i with expert[t][i] = e of dgate[t][i],
 *   dlogits[t][e] = p_e * (u_e - sum_j p_j u_j), p the softmax of the row.
 * counts and kept are those that the loss was computed from: summed over all devices where it is a loss over all of them.
 * dloss (one float on the device) may be NULL: 1.  dgate [tokens][k] may be NULL: 0; expert is only read with it and may
 * be NULL without.  Tokens that do not count get zeros.  dlogits has the logits' type and may be the logits themselves
 * (same stride). */
int32_t p2_balance_backward(const void* logits, int32_t type, int64_t stride, const uint8_t* keep, int64_t tokens,
                            int32_t experts, int32_t k, const int32_t* expert, const float* dgate, const int64_t* counts,
                            const int64_t* kept, const float* dloss, void* dlogits, int64_t dlogits_stride, void* stream);

int32_t p2_orthogonalize_workspace(int64_t count, int64_t rows, int64_t cols, int64_t* bytes);

/* Newton-Schulz products: X = G / (||G|| + eps) with the Frobenius norm, then `steps` times (1 to 64)
 *   A = X X^T,  X = a X + (b A + c A A) X        (a, b, c) = coefficients[0..2]
 * (for matrices with more rows than columns on their transposes), result = scale * X.  `count` matrices of rows x cols
 * lie `matrix_stride` elements apart.  type is that of G, out_type that of the result, which is written with its own
 * strides.  A zero matrix gives zeros; one that holds an infinity or a NaN gives NaN throughout.
 * The products take each operand as a pair of 16-bit floats (22 bits) and are summed in 32 bits; the result is rounded
 * to out_type once, at the end: for each type it is the P2_F32 result, rounded.
 * Coefficients under which singular values of X may pass 2^10 are refused (P2_EUNSUPPORTED): the bound is worked out from
 * the polynomial, starting from [0, 1].  rows and cols up to 2^17, the pairs' padded size below 2^40 bytes. */
int32_t p2_orthogonalize(const void* g, int32_t type, int64_t stride, int64_t matrix_stride, int64_t count, int64_t rows,
                         int64_t cols, int32_t steps, const double* coefficients, double eps, double scale, void* out,
                         int32_t out_type, int64_t out_stride, int64_t out_matrix_stride, void* workspace,
                         int64_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif
