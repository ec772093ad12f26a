/*
 * tuna_moe.h -- what a mixture of experts needs around the all-to-all of tuna.h: the router that makes the call's
 * arrays, rows packed as 8-bit records, the experts' products, the weighted sum of what comes back, and the whole layer
 * for a few tokens in two kernels.  Kernels for gfx950, the same library, the same error codes.
 *
 * The rows of a mixture of experts travel like this (rank = expert, n_experts virtual ranks, the tokens cut into as many
 * shards of ceil(tokens / n_experts) neighbours; `ranks_per_node` of the all-to-all = experts of one device):
 *     tuna_moe_route       logits -> experts, weights, slots, and the all-to-all's counts and displacements
 *     tuna_fp8_quantize    rows -> records [8-bit values | scales] at their slots in the send buffer
 *     tuna_alltoallv       records -> the experts; an expert's rows lie back to back, expert_rows says where
 *     tuna_fp8_matmul      the experts' first product; tuna_fp8_quantize(TUNA_ACT_SWIGLU); the second product
 *     tuna_alltoallv       back, with the two sides' arrays exchanged (their counts are those of other record sizes)
 *     tuna_moe_combine     the sum over a token's experts
 * The same way in 4 bits: tuna_fp4_quantize and tuna_fp4_matmul in the places of the 8-bit ones (half the bytes on the way), and
 * tuna_moe_few with weights of TUNA_F4.  tuna_moe_balance is the loss that keeps the router's experts evenly used, beside tuna_moe_route.
 *
 * Conventions
 *   - Pointers are DEVICE pointers unless a comment says HOST; `stream` is a hipStream_t as void* (NULL = the default
 *     stream).  Every call enqueues kernels on `stream` and returns: nothing is allocated, copied to the host or waited
 *     for, so every call may be captured in a HIP graph.  Memory a call needs besides its arguments is a workspace of the
 *     caller's, 16-byte aligned, whose contents need not outlive the call; two calls in flight need two.
 *   - `ld...` is the distance between rows in elements of the array (scales: in scales; values in 4 bits: in BYTES, of which a row of
 *     n values has ceil(n / 2)); it is at least the row's length.
 *   - The arguments are checked on the host; TUNA_ERR_ARG, TUNA_ERR_TOO_LARGE or TUNA_ERR_WORKSPACE_TOO_SMALL comes
 *     back before anything is enqueued.  Indices that live on the device (slots, expert numbers, group_rows) are held
 *     inside their arrays by the kernels: a slot or an expert outside its range counts as -1 (absent), a group bound
 *     counts as the largest of all bounds up to it, inside [0, m], so that groups never overlap.
 *   - Rows, columns and (token, expert) pairs number at most 2^31 - 1 each, groups of rows (experts, packed sequences) 1 to
 *     TUNA_MOE_MAX_EXPERTS in every call that has them.  With b = 2^24 - 1, what a launch has threads for:
 *     the router and its gradient take 4 b tokens, the sum's gradient b tokens, tuna_fp8_quantize 32 b blocks of 128 values,
 *     its form by columns b blocks of rows and 128 * 65535 columns; products of rows off 16 bytes 64 b rows; y has up to
 *     64 * 65535 columns (dw: its k); the sum and the gate's gradient take 2^31 - 2^15 rows.  In 4 bits the blocks of 32 of all rows
 *     number at most 2^31 - 1, the rest is as in 8 bits.  More is TUNA_ERR_TOO_LARGE.
 *   - Values: TUNA_F32, TUNA_BF16, TUNA_F8 (e4m3, largest 448, no infinity), TUNA_F4 (e2m1: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their
 *     negatives, two to a byte, the first in the low half; a row starts on a byte, and the high half behind an odd row's last value is
 *     written as 0 and not read).  Pointers are aligned to their elements; operands whose rows start on 16 bytes (and have such a
 *     distance) run wider loads.
 *   - The products in 4 bits go by their scales too.  Their tiles want rows and groups of values AND of scales on 16 bytes (the distances as
 *     well): a row of ceil(k / 32) scales is then held in the next multiple of 16.  The form for few rows wants values on 16 and scales on 4 bytes.
 *     All else runs a simple form: right, and slow.  20011 rows of 32 groups: 2048 x 1792 77 us, with rows of 56 scales 195; 5632 x 2880 0.37 ms,
 *     with rows of 92 scales 1.2, of 90 scales 6.8; 60 rows of 4096 x 2880 6 us, with rows of 90 scales 75.
 *   - Sums, softmax statistics and products are accumulated in 32 bits and rounded once, to the type of the output, but for two
 *     places.  (1) The products of tuna_fp8_matmul(_grad_w) with an output of TUNA_BF16 run on the 8-bit matrix cores, which
 *     add eight neighbouring products at a time, each cut at 2^-13 of the largest one's power of two: off by at most 2^-10 of
 *     the sum of the products' MAGNITUDES.  Where little cancels that is some 1.5e-5 of the result, below its rounding; where
 *     large products cancel, the small ones beside them are lost and the result shows it.  With an output of TUNA_F32
 *     products are exact and sums are in 32 bits, at half the rate: for those who need that.  (2) tuna_moe_few keeps its
 *     activations between its two kernels as two bf16 parts, 2^-16 of each, for either type of the output.  The 4-bit matrix cores add
 *     exact products in 32 bits, so the products of tuna_fp4_matmul(_grad_w) are as good for either type of the output.
 *   - Results do not depend on what runs beside the call: there are no floating-point atomics.
 */
#ifndef TUNA_MOE_H
#define TUNA_MOE_H

#include "tuna.h"

#ifdef __cplusplus
extern "C" {
#endif

#define TUNA_F32 0
#define TUNA_BF16 1
#define TUNA_F8 2
#define TUNA_F4 4

#define TUNA_SCALE_F32 0             /* scales are 32-bit values (quantisers: largest magnitude / 448) */
#define TUNA_SCALE_E8 1              /* scales are powers of two 2^(s - 127), kept as the byte s (quantisers: the smallest not below
                                        largest magnitude / 448); the matrix cores apply them for free */

#define TUNA_ACT_NONE 0
#define TUNA_ACT_SWIGLU 1            /* the row holds 2 * cols values, gate then up: silu(gate) * up is what is quantised */

#define TUNA_ROUTE_RENORM 1          /* the weights of a token's chosen experts sum to one */

#define TUNA_BALANCE_ADD 1           /* the gradient is added to what dlogits holds */

#define TUNA_MOE_MAX_EXPERTS 1024
#define TUNA_MOE_MAX_K 16
#define TUNA_MOE_FEW_TOKENS 64       /* the most tokens of tuna_moe_few */

/*
 * The router: softmax over a token's logits, the k largest, and where every (token, expert) pair goes.
 *   logits    [n_tokens, n_experts], TUNA_F32 or TUNA_BF16.  A logit of -inf or NaN is not eligible: its expert has no
 *             share.  Logits of +inf share the whole weight equally.
 *   experts   [n_tokens, k] in descending order of their logits, equal ones by index; -1 where a token has fewer than k
 *             eligible experts (all of them, if a mask leaves nothing).
 *   weights   [n_tokens, k]: the softmax over all eligible experts, or over the chosen ones (TUNA_ROUTE_RENORM); 0 at -1.
 *   slots     [n_tokens, k]: the pair's row, -1 at -1.  Without a plan: rows in order (expert, token).  With a plan: rows
 *             of the send buffer, in order (shard of the token, expert, token).
 *   expert_rows [n_experts + 1]: expert e's rows are expert_rows[e] .. expert_rows[e + 1] - 1, in order of the token
 *             (with a plan: in the receive buffer, after the all-to-all).
 *   sendcounts, sdispls, recvcounts, rdispls: the plan, [n_experts, n_experts] each, for records of row_bytes bytes
 *             that lie back to back on both sides; all four or none.  For the way back call the all-to-all with
 *             (received rows, recvcounts, rdispls, buffer, sendcounts, sdispls), made for that way's row_bytes.
 */
int tuna_moe_route(const void* logits, int type, int64_t ld, int64_t n_tokens, int n_experts, int k, int flags,
                   int32_t* experts, float* weights, int32_t* slots, int32_t* expert_rows,
                   int64_t row_bytes, int32_t* sendcounts, int64_t* sdispls, int32_t* recvcounts, int64_t* rdispls,
                   void* workspace, size_t workspace_bytes, void* stream);
/* HOST only: the workspace of tuna_moe_route, with (1) or without (0) a plan; what is enough for n_tokens is enough for fewer. */
int tuna_moe_route_workspace(int64_t n_tokens, int n_experts, int k, int with_plan, size_t* bytes);
/* The gradient of the weights with respect to the logits (the choice itself has none): dlogits has the logits' type and
 * is written whole, 0 for experts that are not eligible.  `weights` and `experts` as tuna_moe_route left them. */
int tuna_moe_route_grad(const void* logits, int type, int64_t ld, int64_t n_tokens, int n_experts, int k, int flags,
                        const int32_t* experts, const float* weights, const float* dweights,
                        void* dlogits, int64_t ld_dlogits, void* stream);

/*
 * The loss that is least when a router uses its experts evenly, for every sequence of a packed batch:
 *     loss[s] = n_experts * sum over e of (counts[s, e] / C) * shares[s, e],   C = sum over e of counts[s, e]
 * 1 where counts or shares are even, n_experts where one expert has everything, 0 where a sequence has no pairs or no tokens.
 *   logits    as tuna_moe_route takes them, with the same rule for the eligible ones.
 *   experts   [n_tokens, k], as tuna_moe_route left them; a number outside [0, n_experts) is absent.
 *   group_rows [groups + 1]: the sequences' bounds in the tokens, or NULL for one sequence of all tokens.  Tokens outside every
 *             sequence count nowhere.
 *   counts    [groups, n_experts]: how many of the sequence's (token, expert) pairs the expert has.
 *             More than TUNA_MOE_MAX_EXPERTS sequences: a call for each so many of them (group_rows, counts, tokens, shares and loss from
 *             there on), and the gradient with TUNA_BALANCE_ADD to zeros.
 *   tokens    [groups]: how many of its tokens have an eligible expert.
 *   shares    [groups, n_experts]: the mean over those tokens of the softmax over all eligible logits.
 *   loss      [groups].  All four are written whole.
 */
int tuna_moe_balance(const void* logits, int type, int64_t ld, int64_t n_tokens, int n_experts, const int32_t* experts, int k,
                     const int32_t* group_rows, int groups, int32_t* counts, int32_t* tokens, float* shares, float* loss,
                     void* workspace, size_t workspace_bytes, void* stream);
/* HOST only: the workspace of tuna_moe_balance; what is enough for n_tokens is enough for fewer. */
int tuna_moe_balance_workspace(int64_t n_tokens, int n_experts, int groups, size_t* bytes);
/* The gradient of the losses with respect to the logits, dloss [groups] the losses' own (counts have none); counts and tokens as
 * tuna_moe_balance left them.  dlogits has the logits' type and is written whole, 0 for tokens outside every sequence and experts
 * that are not eligible; with TUNA_BALANCE_ADD it is added to what is there (tuna_moe_route_grad's, for the whole of the router). */
int tuna_moe_balance_grad(const void* logits, int type, int64_t ld, int64_t n_tokens, int n_experts,
                          const int32_t* group_rows, int groups, const int32_t* counts, const int32_t* tokens, const float* dloss,
                          int flags, void* dlogits, int64_t ld_dlogits, void* stream);

/*
 * Rows in 8 bits: every 128 neighbours of a row (the last block of a row may be shorter) share a scale.  With a = the largest finite
 * magnitude of the block: scale = a / 448 rounded to 32 bits and at least 2^-126, or the smallest power of two that is not
 * less (TUNA_SCALE_E8); 1 for a block of zeros.  Values are x / scale, to nearest, ties to even; infinities and NaN
 * become NaN.  The gradient of a quantisation is taken as the identity.
 *   x         [rows, cols] (TUNA_ACT_SWIGLU: [rows, 2 cols]) of TUNA_F32 or TUNA_BF16.
 *   slots     NULL: row r goes to row r of q and scales (copies = 1).  Else [rows, copies]: row r goes to each of its
 *             slots in [0, out_rows); others are skipped.  Two pairs must not have one slot.
 *   q, scales [out_rows, cols] and [out_rows, ceil(cols / 128)]; both may lie in one record (q at its start, scales behind).
 */
int tuna_fp8_quantize(const void* x, int type, int64_t ldx, int64_t rows, int64_t cols, int act,
                      const int32_t* slots, int copies, int64_t out_rows,
                      void* q, int64_t ldq, void* scales, int64_t ld_scales, int scale_type, void* stream);
/*
 * Columns in 8 bits, transposed: every 128 rows of a group share one scale in each column.  q is [cols, ldq], scales
 * [cols, ld_scales]; group g's rows start at a multiple of 128, behind those of the groups before it, each rounded up to
 * 128; the rest of its last block is zeros.  ldq >= 128 * (ceil(rows / 128) + groups - 1), ld_scales >= ldq's blocks.
 *   group_rows [groups + 1]: the groups' bounds in the rows, or NULL for one group of all rows.
 */
int tuna_fp8_quantize_columns(const void* x, int type, int64_t ldx, int64_t rows, int64_t cols,
                              const int32_t* group_rows, int groups, void* q, int64_t ldq, void* scales, int64_t ld_scales,
                              int scale_type, void* stream);
/* The gradient of silu(gate) * up: x [rows, 2 cols], dh [rows, cols], dx [rows, 2 cols], all of `type`. */
int tuna_moe_swiglu_grad(const void* x, int type, int64_t ldx, const void* dh, int64_t ld_dh, int64_t rows, int64_t cols,
                         void* dx, int64_t ld_dx, void* stream);

/*
 * y[r, j] = sum over blocks b of 128 columns: xs[r, b] * ws[g, j / 128, b] * sum over i in b: x[r, i] * w[g, j, i]
 * for the rows r of group g.  x [m, k], w [groups, n, k] in TUNA_F8; xs [m, ceil(k / 128)], ws [groups, ceil(n / 128),
 * ceil(k / 128)]; y [m, n] in TUNA_F32 or TUNA_BF16.  w_group, ws_group: the distance of two groups' w and ws, in elements.
 *   group_rows [groups + 1]: the groups' bounds in the rows of x and y, or NULL for one group of all rows.  Rows outside
 *   every group are not written.
 * The gradient of x is the same product of dy in 8 bits with w transposed (kept beside w: 128 x 128 scales transpose with it).
 */
int tuna_fp8_matmul(const void* x, int64_t ldx, const void* xs, int64_t ld_xs,
                    const void* w, int64_t ldw, int64_t w_group, const void* ws, int64_t ld_ws, int64_t ws_group, int scale_type,
                    const int32_t* group_rows, int groups, void* y, int y_type, int64_t ldy,
                    int64_t m, int64_t n, int64_t k, void* stream);
/*
 * The gradient of the weights: dw[g, i, j] = sum over the rows r of group g: dy[r, i] * x[r, j], with both sides as
 * tuna_fp8_quantize_columns lays them out: dyt [n, ...], xt [k, ...], scales for every 128 rows.  dw [groups, n, k] in
 * TUNA_F32 or TUNA_BF16 is written whole (zeros for a group without rows).  m = the rows of all groups, as above.
 */
int tuna_fp8_matmul_grad_w(const void* dyt, int64_t ld_dyt, const void* dyt_scales, int64_t ld_dyt_scales,
                           const void* xt, int64_t ld_xt, const void* xt_scales, int64_t ld_xt_scales, int scale_type,
                           const int32_t* group_rows, int groups, void* dw, int dw_type, int64_t ld_dw, int64_t dw_group,
                           int64_t m, int64_t n, int64_t k, void* stream);

/*
 * Rows in 4 bits: every 32 neighbours of a row (the last block of a row may be shorter) share a scale, a power of two 2^(s - 127) kept
 * as the byte s: the smallest that is not below largest magnitude / 6, at least 2^-126; 1 for a block of zeros.  Values are x / scale, to
 * nearest, ties to even.  A block that holds an infinity or a NaN has the scale NaN (s = 255): all of it reads as NaN.  The gradient of a
 * quantisation is taken as the identity.  Arguments as in tuna_fp8_quantize; ldq in bytes.
 *   q, scales [out_rows, ceil(cols / 2)] and [out_rows, ceil(cols / 32)] bytes; both may lie in one record.
 */
int tuna_fp4_quantize(const void* x, int type, int64_t ldx, int64_t rows, int64_t cols, int act,
                      const int32_t* slots, int copies, int64_t out_rows,
                      void* q, int64_t ldq, void* scales, int64_t ld_scales, void* stream);
/*
 * Columns in 4 bits, transposed: every 32 rows of a group share one scale in each column.  q is [cols, ldq] bytes, scales
 * [cols, ld_scales]; group g's rows start at a multiple of 128, behind those of the groups before it, each rounded up to 128; the
 * rest of its last 128 is zeros, with scales of 1.  With nb = ceil(rows / 128) + groups - 1: ldq >= 64 nb, ld_scales >= 4 nb.
 *   group_rows [groups + 1]: the groups' bounds in the rows, or NULL for one group of all rows.
 */
int tuna_fp4_quantize_columns(const void* x, int type, int64_t ldx, int64_t rows, int64_t cols,
                              const int32_t* group_rows, int groups, void* q, int64_t ldq, void* scales, int64_t ld_scales,
                              void* stream);
/* Rows in 4 bits read back: x[r, i] = value * scale, in TUNA_F32 or TUNA_BF16, either of which holds it
 * exactly, or is infinite from 2^128 on (magnitudes of 1.75 * 2^127 and more are rounded to that when they are quantised). */
int tuna_fp4_dequantize(const void* q, int64_t ldq, const void* scales, int64_t ld_scales, int64_t rows, int64_t cols,
                        void* x, int type, int64_t ldx, void* stream);

/*
 * y[r, j] = sum over blocks b of 32 columns: xs[r, b] * ws[g, j, b] * sum over i in b: x[r, i] * w[g, j, i]
 * for the rows r of group g.  x [m, k], w [groups, n, k] in TUNA_F4; xs [m, ceil(k / 32)], ws [groups, n, ceil(k / 32)] bytes; y [m, n]
 * in TUNA_F32 or TUNA_BF16.  ldx, ldw in bytes; w_group, ws_group: the distance of two groups' w and ws, in bytes.
 *   group_rows [groups + 1]: the groups' bounds in the rows of x and y, or NULL for one group of all rows.  Rows outside
 *   every group are not written.
 * The gradient of x is the same product of dy in 4 bits with w in 4 bits along its other axis: tuna_fp4_quantize_columns of w as
 * [groups * n, k] with the bounds 0, n, 2 n, ... leaves it so, with w_group = 64 ceil(n / 128) and ws_group = 4 ceil(n / 128), which is
 * a multiple of 16 where ceil(n / 128) is one of 4.  A call for each group leaves any distance, and so scales on 16 bytes for every n (10007
 * rows of 8 groups, 2816 x 2048: the product 64 us in place of 154, the calls 70 in place of 35 once for each new w).
 */
int tuna_fp4_matmul(const void* x, int64_t ldx, const void* xs, int64_t ld_xs,
                    const void* w, int64_t ldw, int64_t w_group, const void* ws, int64_t ld_ws, int64_t ws_group,
                    const int32_t* group_rows, int groups, void* y, int y_type, int64_t ldy,
                    int64_t m, int64_t n, int64_t k, void* stream);
/*
 * The gradient of the weights: dw[g, i, j] = sum over the rows r of group g: dy[r, i] * x[r, j], with both sides as
 * tuna_fp4_quantize_columns lays them out: dyt [n, ...], xt [k, ...], scales for every 32 rows.  dw [groups, n, k] in
 * TUNA_F32 or TUNA_BF16 is written whole (zeros for a group without rows).  m = the rows of all groups, as above.
 */
int tuna_fp4_matmul_grad_w(const void* dyt, int64_t ld_dyt, const void* dyt_scales, int64_t ld_dyt_scales,
                           const void* xt, int64_t ld_xt, const void* xt_scales, int64_t ld_xt_scales,
                           const int32_t* group_rows, int groups, void* dw, int dw_type, int64_t ld_dw, int64_t dw_group,
                           int64_t m, int64_t n, int64_t k, void* stream);

/*
 * out[t] = sum over j of weights[t, j] * y[slots[t, j]]; a slot outside [0, y_rows) adds nothing.  y and out in TUNA_F32
 * or TUNA_BF16, each with its own type.
 */
int tuna_moe_combine(const void* y, int y_type, int64_t ldy, int64_t y_rows, const int32_t* slots, const float* weights,
                     int64_t n_tokens, int k, int64_t cols, void* out, int out_type, int64_t ld_out, void* stream);
/* dy[slots[t, j]] = weights[t, j] * dout[t] (y's type; rows without a slot are not written; no two pairs may have one slot),
 * dweights[t, j] = <dout[t], y[slots[t, j]]> (0 where there is no slot). */
int tuna_moe_combine_grad(const void* dout, int out_type, int64_t ld_dout, const void* y, int y_type, int64_t ldy, int64_t y_rows,
                          const int32_t* slots, const float* weights, int64_t n_tokens, int k, int64_t cols,
                          void* dy, int64_t ld_dy, float* dweights, void* stream);

/*
 * The whole layer for at most TUNA_MOE_FEW_TOKENS tokens, in two kernels, for serving:
 *     out[t] = sum over the chosen experts e: weight(t, e) * w2[e] (silu(gate) * up),   [gate | up] = w1[e] x[t]
 * with the choice and the weights of tuna_moe_route.  A chosen expert's weights are read once for up to 16 of its tokens, w1 for up
 * to 32 where the experts have more than 8 pairs on average, w2 in 4 bits whose rows start on 16 bytes for up to 4, and again for as many more.
 *   x  [n_tokens, hidden] TUNA_BF16;  logits [n_tokens, n_experts] TUNA_F32 or TUNA_BF16
 *   w1 [n_experts, 2 inner, hidden], w2 [n_experts, hidden, inner], dense: TUNA_F8 with s1 [n_experts, ceil(2 inner / 128),
 *      ceil(hidden / 128)], s2 [n_experts, ceil(hidden / 128), ceil(inner / 128)], or TUNA_BF16 (s1 = s2 = NULL), or TUNA_F4 (rows of
 *      ceil(hidden / 2) and ceil(inner / 2) bytes) with scale_type TUNA_SCALE_E8, s1 [n_experts, 2 inner, ceil(hidden / 32)], s2
 *      [n_experts, hidden, ceil(inner / 32)], as tuna_fp4_quantize makes them of the rows of w1 and w2
 *   out [n_tokens, hidden] TUNA_F32 or TUNA_BF16
 */
int tuna_moe_few(const void* x, int64_t ldx, int64_t n_tokens, int64_t hidden, const void* logits, int logits_type, int64_t ld_logits,
                 int n_experts, int k, int flags, const void* w1, const void* s1, const void* w2, const void* s2, int64_t inner,
                 int weight_type, int scale_type, void* out, int out_type, int64_t ld_out,
                 void* workspace, size_t workspace_bytes, void* stream);
/* HOST only */
int tuna_moe_few_workspace(int64_t n_tokens, int64_t hidden, int64_t inner, int n_experts, int k, size_t* bytes);

#ifdef __cplusplus
}
#endif
#endif /* TUNA_MOE_H */
