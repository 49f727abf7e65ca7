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
 *    matrix on the device;
 *  - routing to experts by scores, biases and groups: counts per expert are sums over the device's tokens, and the biases
 *    that balance the experts follow from the counts of the whole batch;
 *  - AdamW over many tensors: the sum of the gradients' squares is a sum over the devices' shares, and the step is what is done with a
 *    reduced gradient, or with a device's part of it, whose new weights' copy is then gathered;
 *  - matrix products with bias, activation and residual: a weight's gradient is a sum over the device's rows, and a
 *    device's part of the inner dimension gives a part of the sum over the tensor axis.
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

#define P2_SOFTMAX 0
#define P2_SIGMOID 1
#define P2_MAX_GROUPS 64      /* groups that a router's experts are in */

int32_t p2_route_forward_workspace(int64_t tokens, int32_t experts, int32_t k, int32_t groups, int64_t* bytes);

/* Routes each token to k experts by scores: s = softmax of its logits, or their sigmoids; v = s + bias (NULL: 0), compared in 64 bits, is
 * what is chosen by, and s what the gates are made of.  An expert whose logit or bias is -inf is not on offer; NaN counts as larger
 * than every number.  (A softmax over a logit of NaN or +inf is NaN throughout.  Logits may differ whose scores are one in 64 bits, as sigmoids of more than 37 are: these tie.)
 *   The experts are in `groups` groups of equal size, one after the other.  A group's value is the sum of its group_best (1 or 2) largest
 *   v (of as many as are on offer), and the choice is made within the group_limit groups of the largest values.
 *   expert[t][i] = the i-th best of those; gate[t][i] = scale * s, or with `renormalise` scale * s / (sum of the chosen experts' s), which
 *   keeps its digits where all of them are tiny.  Ties, of groups and of experts: the lowest index.  Where a token has fewer than k
 *   experts on offer the rest is -1 and 0.
 *   counts[e] = how often expert e was chosen; kept[0] = tokens that count: those with a logit above -inf (or NaN) whose keep[t] is not 0 (keep may
 *   be NULL).  The others choose nothing, and their logits are not looked at.
 * 1 <= k <= min(experts, P2_MAX_CHOSEN), experts a multiple of groups, 1 <= group_limit <= groups. */
int32_t p2_route_forward(const void* logits, int32_t type, int64_t stride, const uint8_t* keep, const float* bias, int64_t tokens,
                         int32_t experts, int32_t k, int32_t score, int32_t groups, int32_t group_limit, int32_t group_best,
                         int32_t renormalise, double scale, int32_t* expert, float* gate, int64_t* counts, int64_t* kept,
                         void* workspace, int64_t workspace_bytes, void* stream);

/* Gradient of  sum dgate * gate  with respect to the logits (the choice itself has none); score, renormalise and scale are those of
 * the forward call.  Choices of -1 count for nothing, and a token of these alone gets zeros.  Where a token names an expert twice both count.
 * dlogits has the logits' type and may be the logits themselves (same stride). */
int32_t p2_route_backward(const void* logits, int32_t type, int64_t stride, int64_t tokens, int32_t experts, int32_t k, int32_t score,
                          int32_t renormalise, double scale, const int32_t* expert, const float* dgate, void* dlogits,
                          int64_t dlogits_stride, void* stream);

/* out[e] = bias[e] + rate * sign(mean(counts) - counts[e]): an expert that was chosen less often than the mean is liked better next
 * time.  counts are those of the whole batch.  out may be bias. */
int32_t p2_route_bias(const float* bias, const int64_t* counts, int32_t experts, double rate, float* out, void* stream);

int32_t p2_square_sum_workspace(int64_t n, int64_t* bytes);

/* out[0] = sum of the squares of all values of n tensors of one type, in 64 bits.  `tensors` and `counts` (values of each) are HOST arrays, which are
 * read before the call returns. */
int32_t p2_square_sum(const void* const* tensors, const int64_t* counts, int64_t n, int32_t type, double* out, void* workspace,
                      int64_t workspace_bytes, void* stream);

#define P2_STATE_BLOCK 256    /* values that share a scale of an 8-bit state */

/* One tensor of an AdamW step, `count` values one after the other.  copy: NULL, or where the new weights go in copy_type, too.
 * 32 bits: mean and square are float[count].  8 bits: int8_t[count] and uint8_t[count], with a scale for each P2_STATE_BLOCK values
 * (the last block may be shorter).  A block's scale is its largest absolute value; with q the stored number
 *   mean = scale * (q / 127) * |q / 127|,   square = scale * (q / 255)^4,
 * the nearest q is stored (of a square other than 0 at least 1), and a block that holds nothing of 2^-100 or more is held as zeros.  A block that
 * holds an infinity or a NaN becomes NaN throughout. */
typedef struct p2_adamw_tensor {
    void* param;
    const void* grad;
    void* copy;
    void* mean;
    void* square;
    float* mean_scale;
    float* square_scale;
    int64_t count;
} p2_adamw_tensor;

int32_t p2_adamw_workspace(int64_t* bytes);

/* One step over n tensors (a HOST array, read before the call returns), t = step[0] + 1 being its number (0 <= step[0] < 2^40 - 1):
 *   g = grad * grad_factor * min(1, max_norm / (grad_factor * sqrt(square_sum[0])))
 *   mean = beta1 mean + (1 - beta1) g,  square = beta2 square + (1 - beta2) g^2
 *   param = param (1 - lr weight_decay) - lr / (1 - beta1^t) * mean / (sqrt(square / (1 - beta2^t)) + eps)
 * with lr = lr * rate[0] (a float on the device; NULL: 1), so that a captured step may follow a schedule.  The new weights are worked out from
 * mean and square before these are rounded to 8 bits; without a 32-bit copy of its own a 16-bit param is rounded to nearest each step.
 * square_sum (device; NULL: no clipping, every step is made) is what p2_square_sum gave, of all devices' gradients where they share a norm.  Where it
 * is not finite, or step[0] is negative or 2^40 - 1, the step is left out: nothing is changed, step[0] neither.  Else step[0] (device) becomes t; in
 * between its upper bits may count what is done.  (Two calls of one step, for groups of other types or decays, have a step[0] each: a call counts it up.)
 * max_norm may be infinity: only this check.  state_bits: 32 or 8; 8 takes eps >= 1e-12 (smaller squares would be held as 0).  Nothing that is written,
 * step and workspace included, may overlap, nor what is read any of it; a gradient may
 * be its own tensor's copy (same type). */
int32_t p2_adamw(const p2_adamw_tensor* tensors, int64_t n, int32_t type, int32_t grad_type, int32_t copy_type, int32_t state_bits,
                 int64_t* step, const float* rate, double lr, double beta1, double beta2, double eps, double weight_decay,
                 double grad_factor, const double* square_sum, double max_norm, void* workspace, int64_t workspace_bytes, void* stream);

/* The values that 8-bit states stand for: of each tensor mean, mean_scale, square, square_scale and count are read (8 bits), and
 * mean_out[i], square_out[i] (HOST arrays of device pointers to float[count]; an entry may be NULL) written. */
int32_t p2_adamw_values(const p2_adamw_tensor* tensors, int64_t n, float* const* mean_out, float* const* square_out, void* stream);

#define P2_NO_ACTIVATION 0
#define P2_RELU 1
#define P2_GELU 2             /* z (1 + erf(z / sqrt 2)) / 2                                    */
#define P2_GELU_TANH 3        /* z (1 + tanh(sqrt(2 / pi) (z + 0.044715 z^3))) / 2              */
#define P2_SILU 4             /* z / (1 + e^-z)                                                 */

/* Takes the arguments of the call that it is for (pointers are looked at for their alignment alone). */
int32_t p2_linear_forward_workspace(const void* x, int64_t x_stride, const void* weight, int64_t weight_stride, int32_t type,
                                    int64_t rows, int64_t inner, int64_t outer, int64_t* bytes);

/* y = activation(z) + residual with z = x weight^T + bias:  x [rows][inner], weight [outer][inner], y, z and residual [rows][outer], bias
 * [outer], all of one type.  bias, residual and z (not kept) may be NULL.  y may be residual (same stride).  Products are summed, and
 * everything up to y worked out, in 32 bits: y goes by the z that has not been rounded yet.  What is written may lie between the rows of something
 * of the same stride (each has columns of its own in a buffer), else everything from its first to its last byte is its own; so for the gradients. */
int32_t p2_linear_forward(const void* x, int64_t x_stride, const void* weight, int64_t weight_stride, const void* bias,
                          const void* residual, int64_t residual_stride, int32_t type, int32_t activation, int64_t rows,
                          int64_t inner, int64_t outer, void* y, int64_t y_stride, void* z, int64_t z_stride, void* workspace,
                          int64_t workspace_bytes, void* stream);

/* What any call of these sizes takes; _for: what the call of these arguments takes, which may be far less (pointers are looked at for their alignment
 * alone; dx, dweight, dbias: whether they are asked for). */
int32_t p2_linear_backward_workspace(int32_t type, int64_t rows, int64_t inner, int64_t outer, int64_t* bytes);
int32_t p2_linear_backward_workspace_for(const void* dy, int64_t dy_stride, const void* x, int64_t x_stride, const void* weight, int64_t weight_stride,
                                         int32_t type, int32_t activation, int64_t rows, int64_t inner, int64_t outer, int32_t dx, int32_t dweight,
                                         int32_t dbias, int64_t* bytes);

/* With dz = dy * activation'(z):  dx = dz weight, dweight = dz^T x, dbias = sum over rows of dz; dx, dweight and dbias may each be NULL: not asked
 * for.  z is what the forward pass kept (NULL without an activation); at 0 the slope of P2_RELU is 0.  The residual's gradient is dy.  dweight and
 * dbias have `weight_type`, all else `type`.  Where the matrix units make the products, as they do of more than eight rows, dz is rounded to `type` for
 * them (in 16 bits with an activation: by half a step at most of each dz, which moves results by as much as rounding them does; a call in P2_F32 rounds
 * nothing); where they do not, and for dbias, dz is taken as it is.  rows = 0 writes zeros to dweight and dbias.  */
int32_t p2_linear_backward(const void* dy, int64_t dy_stride, const void* z, int64_t z_stride, const void* x, int64_t x_stride,
                           const void* weight, int64_t weight_stride, int32_t type, int32_t activation, int64_t rows, int64_t inner,
                           int64_t outer, void* dx, int64_t dx_stride, void* dweight, int64_t dweight_stride, void* dbias,
                           int32_t weight_type, void* workspace, int64_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif
