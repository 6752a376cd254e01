/*
 * eb_experts.h -- a mixture of experts over pooled lookups, for AMD Instinct
 * MI355X (gfx950).
 *
 * What follows the pooled lookups of include/eb.h in a ranking model is its
 * dense part.  Where that is a mixture of experts, one batch takes four steps:
 *
 *   eb_route_experts    every token's best experts from its scores, their
 *                       weights, and the chosen (token, expert) pairs grouped
 *                       by expert (the "slots");
 *   eb_quantize_fp8     the tokens' vectors in 8 bits, with a scale for each
 *                       block of 128;
 *   eb_expert_product   every slot's vector times its expert's weights (once
 *                       or more; also a plain product with one weight matrix);
 *   eb_forward_ex       the slots' results joined again per token: a weighted
 *                       pooled lookup whose ids are the pairs' slots.
 *
 * The conventions of include/eb.h hold: return codes, eb_last_error, no
 * exceptions, no allocation, no host synchronisation, borrowed device buffers,
 * all work enqueued on `stream`.  Contents of device buffers are not validated:
 * any values are safe.  Every call may be captured into a graph.
 */
#ifndef EB_EXPERTS_H
#define EB_EXPERTS_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* 8-bit floating point e4m3 (1 sign, 4 exponent, 3 mantissa bits; largest
 * value 448, a NaN, no infinities), beside EB_F32, EB_F16 and EB_BF16. */
enum { EB_FP8 = 3 };

/* How a router's outputs become scores, for eb_route_experts' `mode`. */
enum { EB_SOFTMAX = 0, EB_SIGMOID = 1 };
/* OR-ed into it: divide a token's weights by their sum; judge a group by the
 * sum of its two best experts instead of its best. */
enum { EB_RENORMALIZE = 0x100, EB_GROUP_PAIR = 0x200 };

/* What eb_expert_product applies to its sums. */
enum { EB_ACT_NONE = 0, EB_ACT_RELU = 1, EB_ACT_SILU_GATE = 2 };
/* OR-ed into it: 16-bit outputs from sums as exact as those of other types,
 * whatever the call's size. */
enum { EB_EXACT_SUMS = 0x100 };

/*
 * eb_route_experts_workspace -- device workspace, in bytes, of eb_route_experts
 * for N tokens, K of E experts per token and the shard [shard_lo, shard_hi): 0
 * for few pairs.  Returns EB_ERR_INVALID for NULL bytes or bad sizes,
 * EB_ERR_UNSUPPORTED beyond eb_route_experts' limits on E, K and N * K.  Touches
 * no device state.
 */
int eb_route_experts_workspace(int64_t N, int32_t E, int32_t K, int32_t shard_lo, int32_t shard_hi, size_t *bytes);

/*
 * eb_route_experts -- choose K of E experts for each of N tokens, and group the
 * chosen pairs by expert.
 *
 *   N, E, K      tokens (>= 0), experts (1 .. 1024), experts per token
 *                (1 .. 64, <= E); N * K < 2^31.
 *   scores       device [N, E] of `dtype` (EB_F32, EB_F16, EB_BF16), rows
 *                `ld` (>= E) elements apart, element-aligned: the router's
 *                outputs x.  An expert whose x is -infinity or NaN cannot be
 *                chosen; +infinity counts as the largest finite float.
 *   bias         device fp32 [E] added to the scores for the choice only, or
 *                NULL.  NaN and -infinity keep their expert from being chosen.
 *   mode         EB_SOFTMAX (s = softmax of a token's x) or EB_SIGMOID
 *                (s = 1 / (1 + exp(-x))), optionally | EB_RENORMALIZE
 *                | EB_GROUP_PAIR.
 *   groups, top_groups
 *                experts are judged in `groups` (1 .. 32, dividing E) groups
 *                of consecutive experts; only those of the top_groups
 *                (1 .. groups) best groups are chosen from.  A group's
 *                worth is its best expert's, or with EB_GROUP_PAIR (groups of
 *                two or more) the sum of s + bias of its two best (minus
 *                infinity where fewer can be chosen).  1, 1: no groups.
 *   scale        every weight is multiplied by it.
 *   shard_lo, shard_hi
 *                the experts [lo, hi) of this GPU, 0 <= lo <= hi <= E: only
 *                pairs of these get slots.  0, E for all of them.
 *   ids          device int32 [N, K]: the experts of largest s + bias (without
 *                a bias: of largest x), best first, the lower id first where
 *                two are equal.  -1 where no expert is left to choose.
 *   weights      device fp32 [N, K]: s of those experts (without the bias);
 *                with EB_RENORMALIZE divided by their sum; times scale.  0 where the id is -1.
 *   offsets      device int32 [hi - lo + 1], or NULL (then tokens and slots
 *                must be NULL too and only ids and weights are written): the
 *                slots of expert lo + j are [offsets[j], offsets[j + 1]).
 *   tokens       device int32 [N * K]: the token of each slot, in token order
 *                within an expert; -1 at and past offsets[hi - lo].
 *   slots        device int32 [N, K]: the slot of each pair, or -1.
 *   workspace    device scratch of at least eb_route_experts_workspace()
 *                bytes, 4-byte aligned, owned by the caller; contents not
 *                kept.  May be NULL where that is 0, or offsets NULL.
 *
 * Scores, sums and weights are fp32 whatever the type of x; a softmax's
 * exponentials are within 2 ulp, and 0 below 2^-126.  Equal calls give equal bits.
 * Errors: EB_ERR_INVALID for an argument outside the above,
 * EB_ERR_UNSUPPORTED for E, K, groups or N * K beyond the limits or 2^28 tokens
 * and more, EB_ERR_HIP when a launch fails.  N == 0 writes zero offsets.
 */
int eb_route_experts(int64_t N, int32_t E, int32_t K, const void *scores, int32_t dtype, int64_t ld,
                     const float *bias, int32_t mode, int32_t groups, int32_t top_groups, float scale,
                     int32_t shard_lo, int32_t shard_hi, int32_t *ids, float *weights, int32_t *offsets,
                     int32_t *tokens, int32_t *slots, void *workspace, size_t workspace_bytes, void *stream);

/*
 * eb_quantize_fp8 -- values to 8 bits, with a scale for each block.
 *
 *   matrices, rows, cols
 *                `matrices` matrices of rows x cols, stacked: row r of matrix m
 *                is row m * rows + r of x and q.  rows >= 0, cols >= 1.
 *   x            device, `dtype` EB_F32, EB_F16 or EB_BF16, element-aligned,
 *                rows ldx (>= cols) elements apart.
 *   block_rows   1: a scale for each 1 x 128 of a row (vectors);
 *                128: for each 128 x 128 of a matrix (weights).  Blocks at the
 *                end of a row or a matrix are smaller.
 *   q            device e4m3, 16-byte aligned, rows ldq (>= cols, a multiple
 *                of 16) bytes apart.  Bytes of a row past cols are zero up to
 *                the next multiple of 16.
 *   scales       device fp32.  block_rows 1: [ceil(cols/128)][lds], the scale
 *                of row r's block b at b * lds + r, lds >= matrices * rows.
 *                block_rows 128: [matrices][ceil(rows/128)][ceil(cols/128)],
 *                lds unused.
 *
 * scale = max(largest |x| of the block / 448, 2^-126), rounded to fp32; q =
 * x / the scale before its rounding, the exact quotient rounded once, to nearest
 * even.  The value held is q * scale.  A block with an infinity or a NaN has the
 * scale NaN and only NaNs.  Errors:
 * EB_ERR_INVALID for an argument outside the above, EB_ERR_UNSUPPORTED for
 * sizes one launch does not hold (2^24 strips of 16 rows by 256 columns, or of
 * 128 x 128), EB_ERR_HIP when a launch fails.
 */
int eb_quantize_fp8(int32_t matrices, int64_t rows, int64_t cols, const void *x, int32_t dtype, int64_t ldx,
                    int32_t block_rows, void *q, int64_t ldq, float *scales, int64_t lds, void *stream);

/*
 * eb_expert_product -- rows times the weights of their experts, both in 8 bits
 * with a scale for each block of 128.
 *
 *   M            slots (output rows), >= 0, < 2^31.
 *   E            experts, 1 .. 2^30.
 *   N, K         rows of a weight matrix (outputs before EB_ACT_SILU_GATE) and
 *                its columns (inputs), each 1 .. 2^30.
 *   x            device e4m3 [x_rows, K], 16-byte aligned, rows ldx (>= K, a
 *                multiple of 16) bytes apart; read up to K's next multiple
 *                of 16, bytes past K may be anything.
 *   x_scales     device fp32 [ceil(K/128)][ldxs], ldxs >= x_rows: as
 *                eb_quantize_fp8 writes them with block_rows 1.
 *   tokens       device int32 [M] or NULL: slot m multiplies row tokens[m] of
 *                x.  A slot whose token is outside [0, x_rows) is not written.
 *                NULL: row m (x_rows >= M).
 *   w            device e4m3 [E][N, K], 16-byte aligned, rows ldw (>= K, a
 *                multiple of 16) bytes apart, matrices N * ldw apart.
 *   w_scales     device fp32 [E][ceil(N/128)][ceil(K/128)]: as eb_quantize_fp8
 *                writes them with block_rows 128.  With EB_ACT_SILU_GATE the
 *                two halves of the rows are blocked each on its own:
 *                [E][2][ceil(N/2/128)][ceil(K/128)].
 *   offsets      device int32 [E + 1], as eb_route_experts writes them: expert
 *                e takes the slots [offsets[e], offsets[e + 1]) (clamped into
 *                [0, M]; they must not decrease, or outputs are unspecified).
 *                Slots of no expert are not written.  NULL for E == 1: all M
 *                slots.
 *   bias         device fp32 [E, N] added to the sums, or NULL.
 *   act          EB_ACT_NONE; EB_ACT_RELU: max(v, 0); EB_ACT_SILU_GATE (even
 *                N): with g = v[n], u = v[N/2 + n], n < N/2, the output is
 *                g / (1 + exp(-g)) * u, N/2 wide, the quotient within 4 + |g|
 *                ulp of fp32, or 2^-119.  Optionally | EB_EXACT_SUMS.
 *   out_type     EB_F32, EB_F16, EB_BF16 or EB_FP8.
 *   out          device, rows ldo elements (>= the output's width) apart,
 *                element-aligned.  EB_FP8: e4m3, 16-byte aligned, ldo a
 *                multiple of 16, scaled as by eb_quantize_fp8 with block_rows 1
 *                from the fp32 values, the quotients within 2 ulp of fp32.
 *   out_scales   device fp32 [ceil(width/128)][ldos], ldos >= M, for EB_FP8;
 *                else unused.
 *
 *   v[m, n] = bias[e, n] + sum over the blocks b of 128 inputs of
 *             x_scales[b, row] * w_scales[e, n/128, b] * (sum over b's inputs k
 *             of x[row, k] * w[e, n, k])
 *
 * in fp32, rounded once to the output's type.  For fp32 and 8-bit outputs, and
 * with EB_EXACT_SUMS for all, the products and sums are exact to fp32's rounding.
 * For 16-bit outputs all but small calls otherwise use the 8-bit matrix unit, at
 * up to twice the rate.  It adds the products of eight neighbouring inputs with
 * what lies more than 13 bits below the largest of them cut off, so a sum is off
 * by less than 2^-10 of the largest product of each eight: about 1.5e-5 of the
 * size of a sum of normal values, but all of what small products add beside one
 * 2^13 times as large, also where large ones cancel.  Equal calls give equal bits;
 * the same row in calls of other sizes need not.
 * Errors: EB_ERR_INVALID for an argument outside the above, EB_ERR_UNSUPPORTED
 * for M, E, N or K past their ends and sizes one launch does not hold (2^23
 * tiles), EB_ERR_HIP when a launch fails.
 */
int eb_expert_product(int64_t M, int32_t E, int64_t N, int64_t K, const void *x, int64_t ldx, int64_t x_rows,
                      const float *x_scales, int64_t ldxs, const int32_t *tokens, const void *w, int64_t ldw,
                      const float *w_scales, const int32_t *offsets, const float *bias, int32_t act,
                      int32_t out_type, void *out, int64_t ldo, float *out_scales, int64_t ldos, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* EB_EXPERTS_H */
