/*
 * som_dense.h -- dense rows on a map: part of the C ABI of libsom.so (conventions, status codes and
 * som_last_error as in som.h).
 *
 * A map whose rows are dense (document embeddings, hidden states) is used through these operators:
 *
 *   som_linear    products of rows with a feature-major matrix, with bias, activation and residual.
 *                 With a codebook W and the bias -|w|^2 / 2 it scores every unit: x.w - |w|^2 / 2
 *                 is largest for the best-matching unit.
 *   som_route     each row's best k units by such scores, and their weights.
 *   som_experts   each row through the experts (two-layer networks) of its units, by these weights.
 *   som_clip      the norm of all gradients together, and their scaling to a largest norm.
 *   som_layer_norm  rows to mean 0 and variance 1, in front of a layer.
 *   som_adamw     a step of all parameters along their gradients, with states in 32 bits or in 8.
 *   som_mx4_...   rows and matrices in 4 bits, and products with them.
 *
 * The first three and som_layer_norm have a backward pass. Matrices are feature-major as codebooks are: W[k * ldw + m]
 * is feature k of column m.
 *
 * Types. Rows, matrices, residuals and results are all fp16 or all bf16 (`type`, SOM_F16 or
 * SOM_BF16) where nothing else is said. Products are summed in fp32 and rounded once, to the type
 * of what is written; softmax statistics are fp32, the sum of squares of som_clip fp64. Activations
 * of 16-bit results and slopes are good to 2^-20 of max(|z|, 1), those of fp32 results to a few
 * units in the last place (gelu below zero to z^2 of them).
 *
 * Strides (ldx, ldw, ...) are in elements, between rows; elements of a row are adjacent. Any
 * alignment to the element's size and any sizes are taken; rows that start 16-byte aligned and
 * widths that are multiples of 8 run fastest. Outputs must not overlap inputs unless stated.
 */
#ifndef SOM_DENSE_H
#define SOM_DENSE_H

#include "som.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { SOM_F32 = 0, SOM_F16 = 1, SOM_BF16 = 2 } som_type;

/* none: z; relu: max(z, 0); gelu: z Phi(z), Phi the normal distribution; silu: z / (1 + exp(-z)). */
typedef enum { SOM_ACT_NONE = 0, SOM_ACT_RELU = 1, SOM_ACT_GELU = 2, SOM_ACT_SILU = 3 } som_act;

typedef enum { SOM_SCORE_SOFTMAX = 0, SOM_SCORE_SIGMOID = 1 } som_score;

#define SOM_ROUTE_MAX_UNITS 4096
#define SOM_ROUTE_MAX_TAKEN 32
#define SOM_ROUTE_MAX_GROUPS 64
#define SOM_MAX_EXPERTS 1024

/*
 * Y = residual + act(X W + bias).
 *   X         device [N, K], ldx >= K;   W device [K, M], ldw >= M.
 *   bias      device [M] or NULL; bias_type is SOM_F32 or `type`.
 *   residual  device [N, M], ldr >= M, or NULL. It may be Y's own buffer (with ldr == ldy and
 *             y_type == type).
 *   Y         device [N, M], ldy >= M, written; y_type is `type`, or SOM_F32 for scores.
 *   pre       device [N, M], ldp >= M, written, or NULL: X W + bias, rounded to `type`, which the
 *             backward pass of an activation needs.
 * 0 <= N < 2^30, 1 <= K, M < 2^30. N == 0 is a no-op.
 */
som_status som_linear(int32_t type, const void *X, int64_t ldx, const void *W, int64_t ldw, const void *bias,
                      int32_t bias_type, int32_t act, const void *residual, int64_t ldr, void *Y, int64_t ldy,
                      int32_t y_type, void *pre, int64_t ldp, int64_t N, int64_t K, int64_t M, void *stream);

/*
 * Its gradients, from dY (device [N, M], lddy >= M, of `type`), each written unless NULL:
 *   dX [N, K] = dz W^T, dW [K, M] = X^T dz, dbias [M] (bias_type) = the column sums of dz, where
 *   dz = dY act'(pre); the residual's gradient is dY itself.
 * `pre` is what som_linear wrote; it is not read when act is SOM_ACT_NONE (then NULL will do). The
 * slope is taken at this rounded value, and dz is held in `type`. The workspace, som_linear_bwd_workspace_bytes(N, K, M, act) bytes, 256-byte
 * aligned, holds dz (unless act is SOM_ACT_NONE) and, for many rows of a small dW, parts of it in
 * fp32 (where it needs neither the size is 0 and NULL will do). N == 0 writes zeros to dW, dbias.
 */
size_t som_linear_bwd_workspace_bytes(int64_t N, int64_t K, int64_t M, int32_t act);

som_status som_linear_bwd(int32_t type, const void *X, int64_t ldx, const void *W, int64_t ldw, const void *pre,
                          int64_t ldp, int32_t act, const void *dY, int64_t lddy, void *dX, int64_t lddx, void *dW,
                          int64_t lddw, void *dbias, int32_t bias_type, int64_t N, int64_t K, int64_t M,
                          void *workspace, size_t workspace_bytes, void *stream);

/*
 * How som_route chooses and weighs units.
 *   score      SOM_SCORE_SOFTMAX: a unit's score is its share of the softmax over the row's open
 *              units; SOM_SCORE_SIGMOID: 1 / (1 + exp(-logit)).
 *   renorm     1: a row's weights are divided by their sum.
 *   groups     the units form this many groups of neighbours (it divides the number of units, at
 *              most SOM_ROUTE_MAX_GROUPS); a row takes units of its group_top best groups only, a
 *              group being as good as its best unit. 0 stands for 1.
 *   group_top  1 ... groups; 0 stands for groups.
 */
typedef struct {
    int32_t score;
    int32_t renorm;
    int32_t groups;
    int32_t group_top;
    int32_t reserved[4]; /* must be zero */
} som_route_config;

/*
 * Each row's k best units and their weights.
 *   logits   device [N, E] of logit_type (SOM_F32, SOM_F16 or SOM_BF16), ldl >= E: a row's logits.
 *   bias     device fp32 [E] or NULL: added to the logits (in fp32, one rounding) where units are
 *            ranked, not where they are weighed: it balances the units' loads.
 *   idx      device int32 [N, k], written: the units by falling logit + bias, the lowest index
 *            first among equals.
 *   weights  device [N, k] of weight_type, written: the scores of these units, without the bias.
 *   counts   device int32 [E], written, or NULL: how many rows took each unit.
 * A unit is closed to a row whose logit, or logit + bias, is NaN or minus infinity: it is not
 * taken and has no share in the softmax. Plus infinity ranks above every number; where units are
 * weighed, an infinite logit counts as the largest fp32 value. Where fewer than k units are open the
 * last places hold index -1 and weight 0.
 * 0 <= N < 2^30; 1 <= E <= SOM_ROUTE_MAX_UNITS; 1 <= k <= min(E, SOM_ROUTE_MAX_TAKEN).
 */
som_status som_route(int32_t logit_type, const void *logits, int64_t ldl, const float *bias, int64_t N, int64_t E,
                     int32_t k, const som_route_config *config, int32_t *idx, int32_t weight_type, void *weights,
                     int32_t *counts, void *stream);

/*
 * dlogits (device [N, E] of logit_type, lddl >= E, written whole) from dweights (device [N, k] of
 * weight_type) and the units som_route took. The choice itself has no gradient; bias has none.
 * Closed units get 0. Entries of idx outside [0, E) are skipped.
 */
som_status som_route_bwd(int32_t logit_type, const void *logits, int64_t ldl, const float *bias, const int32_t *idx,
                         int32_t weight_type, const void *dweights, int64_t N, int64_t E, int32_t k,
                         const som_route_config *config, void *dlogits, int64_t lddl, void *stream);

/*
 * out[n] = residual[n] + sum over j of w[n, j] (act(x[n] W1[e] + b1[e]) W2[e] + b2[e]), e = idx[n, j].
 *   X         device [N, D], ldx >= D.
 *   idx, w    device int32 [N, k] and [N, k] of `type`. Entries of idx outside [0, E) are skipped.
 *   W1, b1    device [E, D, F] and [E, F];   W2, b2 device [E, F, D] and [E, D]; dense. b1, b2 or
 *             both may be NULL.
 *   residual  device [N, D], ldr >= D, or NULL.
 *   out       device [N, D], ldo >= D, written; it may be the residual's buffer (with ldo == ldr).
 *   keep      1: the workspace is laid out for the backward pass and keeps what it needs.
 *   workspace device, som_experts_workspace_bytes(N, k, E, D, F, keep) bytes, 256-byte aligned.
 * act(...) is rounded to `type` between the two products; the experts' results are weighted and
 * added in fp32, in a fixed order.
 * 0 <= N; 1 <= k <= SOM_ROUTE_MAX_TAKEN; 1 <= E <= SOM_MAX_EXPERTS; N k < 2^30; 1 <= D, F < 2^24.
 */
size_t som_experts_workspace_bytes(int64_t N, int32_t k, int64_t E, int64_t D, int64_t F, int32_t keep);

som_status som_experts(int32_t type, const void *X, int64_t ldx, const int32_t *idx, const void *w, const void *W1,
                       const void *b1, const void *W2, const void *b2, int32_t act, const void *residual, int64_t ldr,
                       void *out, int64_t ldo, int64_t N, int32_t k, int64_t E, int64_t D, int64_t F, int32_t keep,
                       void *workspace, size_t workspace_bytes, void *stream);

/*
 * Its gradients from dout (device [N, D], lddo >= D): dX [N, D] (lddx >= D), dw [N, k], and dW1,
 * db1, dW2, db2 shaped as the weights, each written whole unless NULL (an expert without rows gets
 * zeros). The workspace is the one that som_experts (keep = 1, the same arguments) left, and that no
 * other call has been given since (nothing in it tells); it serves any number of backward passes. The residual's gradient is dout itself. N == 0 writes zeros.
 * dz = w dout W2^T act'(x W1 + b1) is rounded to `type` before the products that follow, and
 * w act(...) for dW2; act' is taken at x W1 + b1 rounded to `type`.
 */
som_status som_experts_bwd(int32_t type, const void *X, int64_t ldx, const int32_t *idx, const void *w, const void *W1,
                           const void *W2, const void *b2, int32_t act, const void *dout, int64_t lddo, void *dX,
                           int64_t lddx, void *dw, void *dW1, void *db1, void *dW2, void *db2, int64_t N, int32_t k,
                           int64_t E, int64_t D, int64_t F, void *workspace, size_t workspace_bytes, void *stream);

/*
 * The norm of `count` tensors together, norm = sqrt(sum of all squares), and the tensors scaled by
 * min(1, max_norm / norm).
 *   tensors, outs  host arrays of device pointers: tensor i has sizes[i] elements of types[i]
 *                  (SOM_F32, SOM_F16 or SOM_BF16) and is written, scaled, to outs[i], which may be
 *                  the tensor itself. The arrays are read during the call.
 *   norm           device fp32 [1], written: the norm before scaling.
 *   workspace      device, som_clip_workspace_bytes(sizes, count) bytes, 256-byte aligned.
 * Squares are summed in fp64 in a fixed order. A norm that is infinite (also by its rounding to
 * fp32) or NaN scales nothing: outputs equal their tensors, and the caller sees it in `norm`.
 * max_norm > 0 and finite.
 */
size_t som_clip_workspace_bytes(const int64_t *sizes, int64_t count);

som_status som_clip(const void *const *tensors, void *const *outs, const int64_t *sizes, const int32_t *types,
                    int64_t count, float max_norm, float *norm, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Y = (X - mean) / sqrt(var + eps) * weight + bias, mean and variance (divided by D) over each row.
 *   X         device [N, D] of `type` (SOM_F32, SOM_F16 or SOM_BF16), ldx >= D.
 *   weight    device [D] or NULL (ones);   bias  device [D] or NULL (zeros); both of weight_type,
 *             SOM_F32 or y_type.
 *   Y         device [N, D], ldy >= D, written; y_type is `type`, or any where that is SOM_F32. It may be
 *             X's own buffer (with ldy == ldx and y_type == type).
 *   stats     device fp64 [N, 2], written, or NULL: each row's mean and 1 / sqrt(var + eps), which the
 *             backward pass reads.
 * Mean and variance are formed in fp64. A row with an infinity or a NaN is all NaN. eps is at least
 * 2^-126, and finite. 0 <= N < 2^30, 1 <= D < 2^20. N == 0 is a no-op.
 */
som_status som_layer_norm(int32_t type, const void *X, int64_t ldx, const void *weight, const void *bias,
                          int32_t weight_type, double eps, void *Y, int64_t ldy, int32_t y_type, double *stats,
                          int64_t N, int64_t D, void *stream);

/*
 * Its gradients, from dY (device [N, D] of y_type, lddy >= D) and the stats that som_layer_norm wrote,
 * each written unless NULL:
 *   dX [N, D] of `type` (lddx >= D): add + (t - mean(t) - h mean(t h)) / std, where t = dY weight and
 *     h = (X - mean) / std;  dweight [D] = the sum over rows of dY h;  dbias [D] = the sum of dY.
 *   add       device [N, D] of `type`, ldadd >= D, or NULL: the gradient that reaches X by another way (round the
 *             layer). It may be dX's own buffer (with ldadd == lddx); so may dY (with lddy == lddx and y_type ==
 *             type).
 * Sums are fp32, in a fixed order. The workspace is som_layer_norm_bwd_workspace_bytes(N, D) bytes,
 * 256-byte aligned. N == 0 writes zeros to dweight and dbias.
 */
size_t som_layer_norm_bwd_workspace_bytes(int64_t N, int64_t D);

som_status som_layer_norm_bwd(int32_t type, const void *X, int64_t ldx, const void *weight, int32_t weight_type,
                              const void *dY, int64_t lddy, int32_t y_type, const double *stats, const void *add,
                              int64_t ldadd, void *dX, int64_t lddx, void *dweight, void *dbias, int64_t N, int64_t D,
                              void *workspace, size_t workspace_bytes, void *stream);

/*
 * One tensor of a step: `size` elements (at most 2^38), none of which another tensor of the call holds.
 *   param     device, of `type` (SOM_F32, SOM_F16 or SOM_BF16), updated.
 *   grad      device, of grad_type (any of the three).
 *   m, v      device, updated: the running means of the gradient and of its square, fp32 [size]; or,
 *             with 8-bit states, one code each, uint8 [size].
 *   m_scales, v_scales  device uint8 [ceil(size / 256)], updated: the scales of 8-bit states' blocks.
 *   master    device fp32 [size] or NULL: the parameter in fp32. It is what the step reads and updates; param gets its
 *             value, rounded.
 * 8-bit states start as zeros, scales too. A block of 256 values has the scale s of a power of two,
 * 2^(s - 127), at which its largest magnitude is at most 1.875. A code of m is a sign, 4 bits of exponent and 3 behind
 * the point, exponents from 2^-14 on; one of v 5 bits of exponent and 3 behind the point, from 2^-30 on; the lowest
 * exponent's codes are subnormal. Scale 0: all are zero (magnitudes below 2^-100 are held so). Scale 255: the block
 * held an infinity, a NaN or a magnitude above 1.875 * 2^127, and all of it stands for NaN.
 */
typedef struct {
    void *param;
    const void *grad;
    void *m, *v;
    uint8_t *m_scales, *v_scales;
    float *master;
    int64_t size;
    int32_t type, grad_type;
} som_adamw_tensor;

/*
 * How som_adamw steps. lr, weight_decay: finite, >= 0; 0 <= beta1, beta2 < 1; eps: >= 2^-126 and
 * finite; grad_scale: finite; step: this step's number, 1 ... 2^31 - 1.
 *   bits      32 or 8: the states.
 *   seed      for 8-bit states: with the step, the tensor's number in the call and the element's in the tensor it
 *             decides their rounding.
 *   lr_at, step_at  device fp32 [1] and int32 [1], or NULL: read instead of lr and step (a captured step's rate
 *             and number can so change from replay to replay). A *step_at below 1 counts as 1.
 *   norm      device fp32 [1] or NULL: where it is infinite or NaN (som_clip's norm) nothing is written.
 */
typedef struct {
    double lr, beta1, beta2, eps, weight_decay, grad_scale;
    int64_t step;
    int32_t bits;
    uint32_t seed;
    const float *lr_at;
    const int32_t *step_at;
    const float *norm;
    int64_t reserved[4]; /* must be zero */
} som_adamw_config;

/*
 * A step of AdamW (decoupled weight decay) over `count` tensors, with g = grad_scale * grad:
 *   m = beta1 m + (1 - beta1) g,   v = beta2 v + (1 - beta2) g^2,
 *   p = p (1 - lr weight_decay) - lr / (1 - beta1^step) * m / (sqrt(v) / sqrt(1 - beta2^step) + eps),
 * in fp32 (v below 2^-126 with its absolute error, 2^-149; root and reciprocal to a unit in the last place). Of 8-bit
 * states the step uses the new values before they are rounded. They are rounded to either of the codes beside them, by
 * the seed, so that their mean is kept; a v above zero is never rounded to zero but in a block that is all below 2^-100:
 * eps should be well above the root of that, 2^-50. The same arguments give the same bits.
 * tensors is a host array, read during the call.
 */
som_status som_adamw(const som_adamw_tensor *tensors, int64_t count, const som_adamw_config *config, void *stream);

/*
 * What 8-bit states stand for: m and v of tensor i as fp32 [size] to m_out[i] and v_out[i] (host arrays of device
 * pointers). Of the tensors m, v, their scales and the size are read.
 */
som_status som_adamw_values(const som_adamw_tensor *tensors, int64_t count, float *const *m_out, float *const *v_out,
                            void *stream);

/*
 * Values in 4 bits, microscaled: blocks of 32 features share a power of two.
 *   codes     device uint8 [n, 16 * ceil(K / 32)], 16-byte aligned, dense: a row's codes, two to a byte, the lower
 *             feature in the low half; zeros past feature K. A code is a sign (8) and 0 ... 7 for 0, 0.5, 1, 1.5, 2,
 *             3, 4, 6.
 *   scales    device uint8 [n, ceil(K / 32)], dense: block b's scale s stands for 2^(s - 127); 255 for NaN.
 * som_mx4_quantise writes both for X of `type` (SOM_F32, SOM_F16 or SOM_BF16): columns == 0, rows X [n, K]
 * (ldx >= K); columns == 1, the columns of a feature-major matrix X [K, n] (ldx >= n). s is the exponent of the
 * block's largest magnitude, less 2, plus 127, at least 0; values are rounded to the nearest, ties to the even code,
 * and those above 6 to 6. A block with an infinity or a NaN gets 255. som_mx4_values writes what codes and scales
 * stand for, rounded to `type`, to Y, laid out as X. Scales of 253 and 254 are not made here; magnitudes beyond
 * fp32 are infinite in values, and in products where they do not fit.
 * 0 <= n < 2^30, 1 <= K < 2^30.
 */
som_status som_mx4_quantise(int32_t type, const void *X, int64_t ldx, int32_t columns, uint8_t *codes, uint8_t *scales,
                            int64_t n, int64_t K, void *stream);

som_status som_mx4_values(int32_t type, const uint8_t *codes, const uint8_t *scales, int32_t columns, void *Y,
                          int64_t ldy, int64_t n, int64_t K, void *stream);

/*
 * Y = residual + act(X W + bias), as som_linear, with W in 4 bits by its columns: w_codes, w_scales [M, ...] as
 * som_mx4_quantise (columns == 1) writes them.
 *   X         device [N, K] of `type` (SOM_F16 or SOM_BF16), ldx >= K, with x_scales NULL; or the rows in
 *             4 bits: X the codes (ldx is not read), x_scales their scales.
 *   bias, bias_type, residual, Y, y_type  as in som_linear.
 * The values that codes stand for are multiplied as they are, without a further rounding, and summed in fp32.
 * Results that a block of NaN takes part in are NaN. The workspace is som_mx4_linear_workspace_bytes(N, K, M, packed)
 * bytes, packed 1 for rows in 4 bits, 256-byte aligned.
 * 0 <= N < 2^30, 1 <= K, M < 2^30. N == 0 is a no-op.
 */
size_t som_mx4_linear_workspace_bytes(int64_t N, int64_t K, int64_t M, int32_t packed);

som_status som_mx4_linear(int32_t type, const void *X, int64_t ldx, const uint8_t *x_scales, const uint8_t *w_codes,
                          const uint8_t *w_scales, const void *bias, int32_t bias_type, int32_t act,
                          const void *residual, int64_t ldr, void *Y, int64_t ldy, int32_t y_type, int64_t N, int64_t K,
                          int64_t M, void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif
