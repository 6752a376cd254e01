/*
 * eb_train.h -- what trains a mixture of experts over pooled lookups, for AMD
 * Instinct MI355X (gfx950).
 *
 * include/eb_experts.h runs a layer of experts.  Its training step takes, beside
 * those calls,
 *
 *   eb_layer_norm, eb_layer_norm_backward
 *                       the pooled vectors normalised, and the gradients of that;
 *   eb_activation, eb_activation_backward
 *                       the experts' activation of values that wait in 8 bits,
 *                       and its gradient from the same;
 *   eb_dispatch, eb_combine, eb_combine_backward
 *                       the tokens' rows sorted by expert, the experts' rows
 *                       joined per token with the router's weights, and the
 *                       gradients of both;
 *   eb_weight_gradient  the gradients of the experts' weights, from inputs and
 *                       output gradients in 16 or 8 bits.
 *
 * The gradient of a layer's input is eb_quantize_fp8 and eb_expert_product with
 * the transposed weights.  An "8-bit matrix" is what eb_quantize_fp8 writes with
 * block_rows 1: e4m3 values, 16-byte aligned, rows a multiple of 16 bytes apart,
 * and fp32 scales [ceil(columns/128)][lds], the scale of row r's block b at
 * b * lds + r.  A row is read up to the next multiple of 16 columns.  Where a
 * call writes one, the quotients are rounded to fp32 before they are to e4m3,
 * and the bytes of a row past its columns are zero up to the next multiple of 16.
 *
 * The conventions of include/eb.h hold: return codes, eb_last_error, no
 * exceptions, no allocation, no host synchronisation, borrowed device buffers,
 * all work enqueued on `stream`.  Contents of device buffers are not validated:
 * any values are safe.  Matrices in floating point are aligned to their elements
 * and may have any row stride from their width on.  An output must not overlap
 * an input or another output.  Every call may be captured into a graph; equal
 * calls give equal bits.  Calls that share a workspace, two captured graphs among
 * them, must not overlap.
 */
#ifndef EB_TRAIN_H
#define EB_TRAIN_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/*
 * eb_layer_norm -- rows to mean 0 and variance 1, scaled and shifted.
 *
 *   rows, cols   the matrix; rows >= 0, cols 1 .. 2^30.
 *   x            device, `dtype` EB_F32, EB_F16 or EB_BF16, rows ldx apart.
 *   weight, bias device fp32 [cols] each, or NULL (1; 0).
 *   eps          >= 0, added to the variance.
 *   out_type     EB_F32, EB_F16, EB_BF16 or EB_FP8.
 *   y            device [rows, cols] of out_type, rows ldy apart; EB_FP8: an
 *                8-bit matrix with y_scales, ldys >= rows.
 *   kept         device 8-bit matrix of the normalised values n (below), with
 *                kept_scales, ldks >= rows; or NULL.
 *   mean, rstd   device fp32 [rows] each, or NULL.
 *
 *   m = mean of a row's x, r = 1 / sqrt(mean of (x - m)^2 + eps),
 *   n = (x - m) * r,  y = n * weight + bias
 *
 * in fp32, y rounded once to its type.  Errors: EB_ERR_INVALID for an argument
 * outside the above, EB_ERR_UNSUPPORTED for sizes past the above or past one
 * launch (2^24 rows), EB_ERR_HIP when a launch fails.
 */
int eb_layer_norm(int64_t rows, int64_t cols, const void *x, int32_t dtype, int64_t ldx, const float *weight,
                  const float *bias, float eps, int32_t out_type, void *y, int64_t ldy, float *y_scales, int64_t ldys,
                  void *kept, int64_t ldk, float *kept_scales, int64_t ldks, float *mean, float *rstd, void *stream);

/* eb_layer_norm_backward_workspace -- device workspace, in bytes, of
 * eb_layer_norm_backward where it writes dweight or dbias.  EB_ERR_INVALID for
 * NULL bytes or bad sizes, EB_ERR_UNSUPPORTED past eb_layer_norm's limits. */
int eb_layer_norm_backward_workspace(int64_t rows, int64_t cols, size_t *bytes);

/*
 * eb_layer_norm_backward -- the gradients of eb_layer_norm.
 *
 *   dy           device [rows, cols], `dy_type` EB_F32, EB_F16 or EB_BF16, rows
 *                lddy apart: the gradient of y.
 *   x            device, x_type EB_F32, EB_F16 or EB_BF16: forward's x; or EB_FP8:
 *                what forward kept, an 8-bit matrix with x_scales, ldxs >= rows.
 *   mean, rstd   device fp32 [rows], as forward wrote them.  mean is NULL for
 *                EB_FP8, and only then.
 *   weight       forward's.
 *   dx           device [rows, cols] of dy_type, rows lddx apart.
 *   dweight, dbias
 *                device fp32 [cols] each, or NULL.
 *   workspace    device scratch of eb_layer_norm_backward_workspace() bytes,
 *                16-byte aligned, contents not kept; may be NULL where dweight
 *                and dbias are.
 *
 *   n = (x - mean) * rstd, or the values kept;  g = dy * weight
 *   dx = rstd * (g - mean of the row's g - n * mean of the row's g * n)
 *   dweight = sum over the rows of dy * n,  dbias = sum over the rows of dy
 *
 * in fp32, dx rounded once.  No rows: dweight and dbias are zeros.  Errors as
 * eb_layer_norm.
 */
int eb_layer_norm_backward(int64_t rows, int64_t cols, const void *dy, int32_t dy_type, int64_t lddy, const void *x,
                           int32_t x_type, int64_t ldx, const float *x_scales, int64_t ldxs, const float *mean,
                           const float *rstd, const float *weight, void *dx, int64_t lddx, float *dweight, float *dbias,
                           void *workspace, size_t workspace_bytes, void *stream);

/*
 * eb_activation -- an expert's activation, of values before it.
 *
 *   rows, cols   the output; rows >= 0, cols 1 .. 2^29.
 *   act          EB_ACT_RELU: v is [rows, cols], h = max(v, 0).  EB_ACT_SILU_GATE:
 *                v is [rows, 2 * cols], h[c] = g / (1 + exp(-g)) * u with
 *                g = v[c], u = v[cols + c].
 *   v            device, v_type EB_F32, EB_F16, EB_BF16, rows ldv apart; or EB_FP8:
 *                an 8-bit matrix with v_scales, ldvs >= rows (as eb_expert_product
 *                writes it with EB_ACT_NONE).
 *   h            device [rows, cols] of out_type EB_F32, EB_F16, EB_BF16, rows
 *                ldh apart; or EB_FP8: an 8-bit matrix with h_scales, ldhs >= rows.
 *
 * In fp32, rounded once; the gate's quotient within 4 + |g| ulp of fp32, or
 * 2^-119.  A NaN of v gives NaN, infinities what the formula gives.  Errors:
 * EB_ERR_INVALID for an argument outside the above, EB_ERR_UNSUPPORTED for sizes
 * past the above or past one launch (2^24 strips of 16 rows by 256 columns),
 * EB_ERR_HIP when a launch fails.
 */
int eb_activation(int64_t rows, int64_t cols, int32_t act, const void *v, int32_t v_type, int64_t ldv,
                  const float *v_scales, int64_t ldvs, int32_t out_type, void *h, int64_t ldh, float *h_scales,
                  int64_t ldhs, void *stream);

/*
 * eb_activation_backward -- the gradient of eb_activation.
 *
 *   rows, cols, act, v ...
 *                as forward's.
 *   dh           device [rows, cols], dh_type EB_F32, EB_F16 or EB_BF16, rows lddh
 *                apart: the gradient of h.
 *   dv           device, of v's shape, in out_type EB_F32, EB_F16, EB_BF16, rows
 *                lddv apart; or EB_FP8: an 8-bit matrix with dv_scales, lddvs >=
 *                rows (blocks of 128 columns from g's first to u's last).
 *
 *   EB_ACT_RELU: dv = dh where v > 0, else 0.  EB_ACT_SILU_GATE, with
 *   p = 1 / (1 + exp(-g)):  dg = dh * p * u * (1 + g * (1 - p)),  du = dh * p * g
 *
 * In fp32, rounded once; p as in eb_activation.  What p or dh * p holds below 2^-126 may
 * be lost.  Errors as eb_activation.
 */
int eb_activation_backward(int64_t rows, int64_t cols, int32_t act, const void *dh, int32_t dh_type, int64_t lddh,
                           const void *v, int32_t v_type, int64_t ldv, const float *v_scales, int64_t ldvs,
                           int32_t out_type, void *dv, int64_t lddv, float *dv_scales, int64_t lddvs, void *stream);

/*
 * eb_dispatch -- rows sorted by expert: out[m] = x[tokens[m]].
 *
 *   M, cols      slots (0 .. 2^31 - 1) and columns (1 .. 2^30).
 *   x            device [x_rows, cols] of dtype EB_F32, EB_F16, EB_BF16, rows ldx
 *                apart; or EB_FP8: an 8-bit matrix with x_scales, ldxs >= x_rows,
 *                whose bytes past cols up to the next multiple of 16 go along.
 *   tokens       device int32 [M], as eb_route_experts writes them.  A slot whose
 *                token is outside [0, x_rows) is not written.
 *   out          device [M, cols] of dtype, rows ldo apart, with out_scales, ldos
 *                >= M, for EB_FP8.
 *
 * Its gradient is eb_combine without weights.  Errors: EB_ERR_INVALID for an
 * argument outside the above, EB_ERR_UNSUPPORTED for sizes past the above or past one
 * launch (2^26 rows of more than 256 bytes or 128 columns, more of shorter ones),
 * EB_ERR_HIP when a launch fails.
 */
int eb_dispatch(int64_t M, int64_t cols, const void *x, int32_t dtype, int64_t ldx, int64_t x_rows, const float *x_scales,
                int64_t ldxs, const int32_t *tokens, void *out, int64_t ldo, float *out_scales, int64_t ldos, void *stream);

/*
 * eb_combine -- the experts' rows joined: out[t] = sum over k of
 * weights[t, k] * y[slots[t, k]].
 *
 *   N, K, cols   tokens (0 .. 2^31 - 1), pairs of a token (1 .. 64), columns
 *                (1 .. 2^30); N * K < 2^31.
 *   y            device [y_rows, cols] of y_type EB_F32, EB_F16, EB_BF16, rows ldy
 *                apart.
 *   slots        device int32 [N, K], as eb_route_experts writes them.  A pair whose
 *                slot is outside [0, y_rows) adds nothing.
 *   weights      device fp32 [N, K], or NULL (1).
 *   out          device [N, cols] of out_type EB_F32, EB_F16, EB_BF16, rows ldo
 *                apart.  Every element is written.
 *
 * Sums are fp32 in the order of k, rounded once.  Errors as eb_dispatch.
 */
int eb_combine(int64_t N, int32_t K, int64_t cols, const void *y, int32_t y_type, int64_t ldy, int64_t y_rows,
               const int32_t *slots, const float *weights, int32_t out_type, void *out, int64_t ldo, void *stream);

/*
 * eb_combine_backward -- the gradients of eb_combine.
 *
 *   N, K, cols, y, slots, weights
 *                as forward's, but that no two pairs may have the same slot of y
 *                (eb_route_experts gives each its own): else which of them dy has
 *                is not specified.  y may be NULL where dweights is.
 *   dout         device [N, cols], dout_type EB_F32, EB_F16 or EB_BF16, rows lddo
 *                apart: the gradient of out.
 *   dy           device [y_rows, cols] of dy_type EB_F32, EB_F16, EB_BF16, rows lddy
 *                apart; or EB_FP8: an 8-bit matrix with dy_scales, lddys >= y_rows.
 *                Rows that are no pair's slot are not written.  May be NULL.
 *   dweights     device fp32 [N, K] or NULL; 0 for a pair without a slot.
 *
 *   dy[slots[t, k]] = weights[t, k] * dout[t]
 *   dweights[t, k] = sum over the columns of dout[t] * y[slots[t, k]]
 *
 * In fp32, rounded once.  Errors as eb_dispatch.
 */
int eb_combine_backward(int64_t N, int32_t K, int64_t cols, const void *dout, int32_t dout_type, int64_t lddo,
                        const void *y, int32_t y_type, int64_t ldy, int64_t y_rows, const int32_t *slots,
                        const float *weights, int32_t dy_type, void *dy, int64_t lddy, float *dy_scales, int64_t lddys,
                        float *dweights, void *stream);

/* eb_weight_gradient_workspace -- device workspace, in bytes, of
 * eb_weight_gradient: 0 where its tiles fill the GPU.  EB_ERR_INVALID for NULL
 * bytes or bad sizes, EB_ERR_UNSUPPORTED past eb_weight_gradient's limits. */
int eb_weight_gradient_workspace(int64_t M, int32_t E, int64_t N, int64_t K, size_t *bytes);

/*
 * eb_weight_gradient -- the gradients of the weights of eb_expert_product.
 *
 *   M, E         slots (0 .. 2^31 - 1) and experts (1 .. 2^30).
 *   N, K         rows and columns of a weight matrix, each 1 .. 2^30.
 *   dy           device [M, N], dy_type EB_F16, EB_BF16, rows lddy apart; or EB_FP8:
 *                an 8-bit matrix with dy_scales, lddys >= M.  The gradient of the
 *                product's output before its activation.
 *   x            device [x_rows, K], x_type EB_F16, EB_BF16, rows ldx apart; or
 *                EB_FP8: an 8-bit matrix with x_scales, ldxs >= x_rows.
 *   tokens       device int32 [M] or NULL: slot m's input is row tokens[m] of x; a
 *                slot whose token is outside [0, x_rows) adds nothing.  NULL: row m
 *                (x_rows >= M).
 *   offsets      device int32 [E + 1], as eb_route_experts writes them: expert e has
 *                the slots [offsets[e], offsets[e + 1]) (clamped into [0, M]).
 *                NULL for E == 1: all M slots.
 *   out_type     EB_F32, EB_F16 or EB_BF16.
 *   accumulate   0: dw is written, zeros for an expert without slots.  1: it is
 *                added to.
 *   dw           device [E][N, K] of out_type, rows lddw (>= K) apart, matrices
 *                N * lddw apart.
 *   workspace    device scratch of eb_weight_gradient_workspace() bytes, 16-byte
 *                aligned, contents not kept; may be NULL where that is 0.
 *
 *   dw[e][n, k] = sum over e's slots m of dy[m, n] * x[tokens[m], k]
 *
 * Sums are fp32, in an order that depends on the sizes and offsets alone, rounded
 * once (with accumulate after dw is added).  Products are within 2^-20 of exact; where
 * neither operand is bfloat16 and one has scales, also within 2^-34 of the largest that
 * the scales of the expert's slots allow; for a bfloat16 output of a bfloat16 operand and
 * one with scales within 2^-16.  An infinite operand gives
 * infinities or NaNs.  Errors: EB_ERR_INVALID for an argument outside the
 * above, EB_ERR_UNSUPPORTED for sizes past the above or past one launch (2^24
 * tiles of 128 x 128), EB_ERR_HIP when a launch fails.
 */
int eb_weight_gradient(int64_t M, int32_t E, int64_t N, int64_t K, const void *dy, int32_t dy_type, int64_t lddy,
                       const float *dy_scales, int64_t lddys, const void *x, int32_t x_type, int64_t ldx, int64_t x_rows,
                       const float *x_scales, int64_t ldxs, const int32_t *tokens, const int32_t *offsets,
                       int32_t out_type, int32_t accumulate, void *dw, int64_t lddw, void *workspace,
                       size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* EB_TRAIN_H */
