/*
 * ep_layer.h -- operators of a MoE layer around dispatch and combine (libep.so).
 *
 * ep.h moves a layer's token rows; the calls below compute what stands before and after
 * the movement on the same GPU, forward and backward:
 *
 *   ep_rmsnorm          residual addition and RMS norm; bf16 rows and 8-bit rows
 *   ep_route            top-k experts, gates, counts per expert, balance loss
 *   ep_expert_product   y = act(x W_e^T + b_e) + residual over the rows packed by expert
 *   ep_combine_grad     the gradient of the gate-weighted combine
 *   ..._grad            their backward passes
 *
 * A training step's forward is: ep_rmsnorm, ep_expert_product (one expert: the router's
 * logits), ep_route, ep_dispatch_layout and ep_pack (or ep_dispatch), ep_expert_product
 * (up, then down), ep_combine_rows.  Its backward is: ep_combine_grad, ep_expert_product_grad
 * (down, then up), ep_combine_rows with unit gates (the gradient of the dispatch),
 * ep_route_grad, ep_expert_product_grad (the router's), ep_rmsnorm_grad.
 *
 * The conventions of ep.h hold: device pointers on the current device, calls that only
 * enqueue on `stream`, argument errors reported before anything is enqueued, no call throws.
 * No call keeps state or allocates.  Further:
 *   - Rows are contiguous ([T][H], no gaps) and 16-byte aligned, row lengths are multiples
 *     of 8 elements (of 16 for 8-bit rows).
 *   - No output may overlap an input or another output, except where stated.
 *   - Workspaces need no initial contents and hold nothing between calls; two calls that may
 *     run at once need two.
 *   - Sums, softmax statistics and accumulators are fp32; a result of 16 or 8 bits is rounded
 *     once, to nearest-even.  The same inputs give the same bits.
 *   - NaN and infinities go through as the formulas say; they change no other row.
 *
 * 8-bit rows (EP_ROWS_8BIT): a row of H values is H bytes of e4m3 (OCP, largest value 448),
 * then the row's fp32 scale, then 12 bytes of zero: H + 16 bytes.  Value i is byte i's value
 * times the scale.  Dispatch moves such a row as any other, as a bf16 row of (H + 16) / 2
 * elements.
 */
#ifndef EP_LAYER_H
#define EP_LAYER_H

#include "ep.h"

#ifdef __cplusplus
extern "C" {
#endif

#define EP_ROWS8_EXTRA 16       /* bytes of an 8-bit row behind its values */
#define EP_NORM_MAX_HIDDEN 65536 /* longest row of the norm */
#define EP_PRODUCT_MAX_LENGTH 262144 /* largest K and largest number of weight rows */

typedef enum {
    EP_ROWS_BF16 = 0,
    EP_ROWS_8BIT = 1,
} ep_rows_kind;

typedef enum {
    EP_ACT_NONE = 0,
    EP_ACT_RELU = 1,   /* max(z, 0) */
    EP_ACT_SILU = 2,   /* z / (1 + exp(-z)) */
    EP_ACT_GELU = 3,   /* z Phi(z), Phi the normal distribution function (by erf) */
    EP_ACT_SWIGLU = 4, /* silu(gate) * up: W_e has 2N rows, the gates' N first, then the ups' */
} ep_activation;

/* --------------------------------------------------------------------------- norm */

/* Residual addition and RMS norm of each row (before a MoE layer's router and dispatch):
 *   s = x + residual            (s = x without a residual)
 *   y = s / sqrt(mean(s^2) + eps) * weight
 *   x, residual  bf16 [T][H]; residual may be NULL
 *   weight       bf16 [H], or NULL for ones
 *   total        bf16 [T][H] or NULL: s, the residual stream; may be x or residual itself
 *   out          bf16 [T][H] or NULL: y
 *   rows8        [T][H + 16] bytes or NULL: y as 8-bit rows, scale = max(max|y|, 2^-100) / 448
 * y is computed from the unrounded sum s and rounded once.  A row with a NaN has a NaN scale.
 * Requires H % 8 == 0 (16 with rows8), 8 <= H <= EP_NORM_MAX_HIDDEN, eps >= 0, an output. */
ep_status ep_rmsnorm(const void *x_dev, const void *residual_dev, const void *weight_dev, int64_t num_tokens,
                     int32_t hidden, float eps, void *total_dev, void *out_dev, void *rows8_dev,
                     hipStream_t stream);

/* Bytes of workspace ep_rmsnorm_grad needs for its weight gradient (0 bytes without one). */
ep_status ep_rmsnorm_grad_workspace_bytes(int64_t num_tokens, int32_t hidden, size_t *bytes /* host out */);

/* Gradient of the norm at s = total (bf16, as ep_rmsnorm wrote it):
 *   n = s / sqrt(mean(s^2) + eps);  g = d_out * weight
 *   dx = (g - n mean(g n)) / sqrt(mean(s^2) + eps) + d_total
 *   d_weight = sum over tokens of d_out * n
 *   total, d_out  bf16 [T][H];  d_total  bf16 [T][H] or NULL: the residual stream's gradient
 *   dx            bf16 [T][H]: the gradient of x and of the residual; may be d_out or d_total
 *   d_weight      fp32 [H] or NULL (then no workspace is needed)
 * Requires what ep_rmsnorm requires. */
ep_status ep_rmsnorm_grad(const void *total_dev, const void *weight_dev, const void *d_out_dev,
                          const void *d_total_dev, int64_t num_tokens, int32_t hidden, float eps, void *dx_dev,
                          float *d_weight, void *workspace, size_t workspace_bytes, hipStream_t stream);

/* ------------------------------------------------------------------------- router */

/* Bytes of workspace ep_route needs. */
ep_status ep_route_workspace_bytes(int64_t num_tokens, int32_t num_experts, size_t *bytes /* host out */);

/* Routing of T tokens from their logits z (softmax gates, balance loss):
 *   p[t] = softmax(z[t]);  topk_idx[t] = the k largest logits, largest first, the lowest
 *   index first among equals (+0 equals -0; a NaN ranks below every number)
 *   topk_w[t][j] = p[t][topk_idx[t][j]], or with `normalize` the softmax over the k chosen
 *   counts[e] = slots that chose e;  prob_sums[e] = sum over tokens of p[t][e]
 *   loss = balance * E * sum_e counts[e] / (N k) * prob_sums[e] / N,  N = live tokens
 *   (0 without live tokens)
 *   logits    fp32 [T][E], or bf16 with logits_bf16 != 0
 *   mask      uint8 [T] or NULL: 0 marks a token that is not live (padding): its gates are 0,
 *             it counts nowhere, its logits are not looked at, and its ids are
 *             (t*k + j) % E, so that the layout gets k different valid experts for it
 *   topk_idx  int32 [T][k], topk_w fp32 [T][k]: what ep_dispatch_layout and ep_combine read
 *   counts    int32 [E], prob_sums fp32 [E], loss fp32 [1]: all three, or all three NULL
 *             where the routing alone is wanted (then no workspace is needed)
 * A logit of -inf is a masked expert: probability and gate 0 (chosen only when fewer than k
 * others are left); a row of -inf alone has no probability anywhere.  A NaN or +inf makes its
 * own row's p NaN, and prob_sums and loss with it; normalized gates look at the chosen logits
 * alone (a NaN is chosen only when fewer than k numbers are left).
 * Requires T >= 0, T*k < 2^31, 1 <= k <= E <= EP_MAX_EXPERTS. */
ep_status ep_route(const void *logits_dev, int32_t logits_bf16, const uint8_t *mask, int64_t num_tokens,
                   int32_t num_experts, int32_t topk, int32_t normalize, float balance, int32_t *topk_idx,
                   float *topk_w, int32_t *counts, float *prob_sums, float *loss, void *workspace,
                   size_t workspace_bytes, hipStream_t stream);

/* Gradient of ep_route with respect to the logits:
 *   d_topk_w  fp32 [T][k] or NULL: the gates' gradient
 *   d_loss    device fp32 [1] or NULL: the balance loss's gradient
 *   topk_idx  as ep_route wrote it;  counts  int32 [E] as ep_route wrote it (only with d_loss):
 *             a group of ranks that balances over all its tokens sums the counts and gives the
 *             sum; N is then the sum's number of tokens (the counts together may pass 2^31)
 *   d_logits  [T][E] in the logits' type; may be the logits themselves
 * The counts are constants of the loss, as usual.  A token that is not live gets zeros. */
ep_status ep_route_grad(const void *logits_dev, int32_t logits_bf16, const uint8_t *mask, const int32_t *topk_idx,
                        const int32_t *counts, const float *d_topk_w, const float *d_loss, int64_t num_tokens,
                        int32_t num_experts, int32_t topk, int32_t normalize, float balance, void *d_logits_dev,
                        hipStream_t stream);

/* ------------------------------------------------------------------------ combine */

/* Gradient of ep_combine_rows (out[t] = sum_j w[t][j] y[slot_pos[t*k + j]]):
 *   dy[slot_pos[t*k + j]] = bf16(w[t][j] * d_out[t]);  d_topk_w[t][j] = <d_out[t], y[slot_pos[t*k+j]]>
 *   d_out     bf16 [T][H];  y  bf16 [max_rows][H];  slot_pos int32 [T*k];  topk_w fp32 [T][k]
 *   dy        bf16 [max_rows][H] or NULL;  d_topk_w fp32 [T][k] or NULL
 * A slot without a row (slot_pos outside [0, max_rows)) writes no row and gets 0.  Rows that
 * no slot names are left as they are.  No two slots may name one row. */
ep_status ep_combine_grad(const void *d_out_dev, const void *y_dev, int64_t max_rows, const int32_t *slot_pos,
                          const float *topk_w, int64_t num_tokens, int32_t hidden, int32_t topk, void *dy_dev,
                          float *d_topk_w, hipStream_t stream);

/* ----------------------------------------------------------------- experts' product */

/* Bytes of workspace ep_expert_product needs (0 for most sizes). */
ep_status ep_expert_product_workspace_bytes(int64_t rows, int32_t num_experts, int32_t in_length, int32_t out_length,
                                            ep_rows_kind kind, ep_activation act, size_t *bytes /* host out */);

/* The experts' matrix product over rows packed by expert: for row r of expert e,
 * offsets[e] <= r < offsets[e+1],
 *   z = x[r] W_e^T (+ bias_e);  y[r] = act(z) (+ residual[r])
 *   x         kind EP_ROWS_BF16: bf16 [rows][K];  EP_ROWS_8BIT: 8-bit rows [rows][K + 16 bytes]
 *   offsets   device int32 [E+1], not decreasing, within [0, rows] (expert_offsets or
 *             local_offsets of a layout); NULL with E = 1: all rows.  Rows outside
 *             [offsets[0], offsets[E]) are left as they are.  Offsets outside [0, rows]
 *             are taken as the nearest of the two
 *   w         [E][Nw][K], Nw = N (2N with EP_ACT_SWIGLU): bf16, or e4m3 bytes with 8-bit rows
 *   w_scale   fp32 [E][Nw], only with 8-bit rows: weight = e4m3 value * w_scale of its row
 *   bias      bf16 [E][Nw] or NULL;  residual  bf16 [rows][N] or NULL
 *   pre       bf16 [rows][Nw] or NULL: z, which the gradient of an activation needs
 *   y         [rows][N], bf16 or fp32
 * bf16 products are exact in the fp32 accumulators.  So are those of 8-bit values where y is
 * fp32 or K < 512; longer sums that end in bf16 go through the 8-bit matrix instruction, which
 * drops the bits of a product that lie 2^13 below the largest one it adds at a time.
 * Requires rows >= 0, 1 <= E <= EP_MAX_EXPERTS, K and N positive multiples of 8 (K of 16 with
 * 8-bit rows), K and Nw <= EP_PRODUCT_MAX_LENGTH, an expert's weights < 2^31 bytes. */
ep_status ep_expert_product(const void *x_dev, ep_rows_kind kind, int64_t rows, const int32_t *offsets,
                            int32_t num_experts, const void *w_dev, const float *w_scale, int32_t in_length,
                            int32_t out_length, const void *bias_dev, ep_activation act, const void *residual_dev,
                            void *pre_dev, void *y_dev, ep_out_dtype out_dtype, void *workspace,
                            size_t workspace_bytes, hipStream_t stream);

/* Bytes of workspace ep_expert_product_grad needs for the results named: EP_GRAD_DBIAS or 0, and
 * what is not wanted.  (1 and 0, with a bias and without, stand for a call for dx and dw.) */
#define EP_GRAD_DBIAS 1
#define EP_GRAD_WITHOUT_DX 2
#define EP_GRAD_WITHOUT_DW 4
ep_status ep_expert_product_grad_workspace_bytes(int64_t rows, int32_t num_experts, int32_t in_length,
                                                 int32_t out_length, ep_activation act, int32_t results,
                                                 size_t *bytes /* host out */);

/* Gradient of ep_expert_product with bf16 rows:
 *   dz = d_y * act'(pre);  dx[r] = dz[r] W_e;  dw_e = sum_r dz[r]^T x[r];  dbias_e = sum_r dz[r]
 *   (the residual's gradient is d_y itself)
 *   x, offsets, w  as in the forward;  d_y  bf16 [rows][N]
 *   pre     bf16 [rows][Nw] as the forward wrote it; NULL with EP_ACT_NONE
 *   dx      bf16 [rows][K] or NULL;  dw  bf16 [E][Nw][K] or NULL;  dbias  fp32 [E][Nw] or NULL
 * dz is rounded to bf16 for the two products (dbias sums it unrounded).  An expert without
 * rows gets zeros in dw and dbias.  Requires what the forward requires, rows < 2^31. */
ep_status ep_expert_product_grad(const void *x_dev, int64_t rows, const int32_t *offsets, int32_t num_experts,
                                 const void *w_dev, int32_t in_length, int32_t out_length, ep_activation act,
                                 const void *pre_dev, const void *d_y_dev, void *dx_dev, void *dw_dev, float *dbias,
                                 void *workspace, size_t workspace_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* EP_LAYER_H */
