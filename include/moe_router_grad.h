/*
 * moe_router_grad.h -- C ABI of what trains the router of an Expert module (gfx950): the auxiliary losses on its logits with the
 * per-expert counts they need, and the gradients from the layer's output back to the router's weights.
 *
 *   moe_combine_backward   dy -> the gates' gradient d_topk_w, and that of the shared expert's gate
 *   moe_route_backward     d_topk_w (moe_route_topk's gates) and the auxiliary losses -> d_logits
 *   moe_router_backward    d_logits -> the router's weights' gradient, and its part of dx
 *
 * The experts' own matrices are taken as frozen: no gradient of moe_expert_ffn is computed, and dx holds the router's part only.
 *
 * Conventions as in moe_shard.h: status codes (MOE_OK / MOE_ERR_*), validation on the host before any HIP call, no allocation, no
 * synchronisation, work enqueued on `stream`; all pointers are DEVICE pointers owned by the caller.  With T == 0 the buffers of T rows
 * may be NULL.  bf16 tensors, y_perm, y_shared, w_shared_gate, d_w_router and workspaces are 16-byte aligned.  A call writes all of its
 * workspace that it reads, so nothing has to start at zero; calls that overlap on one GPU each bring their own.  Sums are taken in a fixed
 * order: the same call gives the same bits.
 */
#ifndef MOE_ROUTER_GRAD_H
#define MOE_ROUTER_GRAD_H

#include "moe_shard.h"

#define MOE_ROUTER_GRAD_MAX_HIDDEN 262144

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Balance loss, z loss and per-expert counts of one batch.  With p = softmax(logits) over all E experts and Tv the number of tokens
 * that count (token_mask != 0; all without a mask):
 *   counts[e]    = assignments (t,j) of counting tokens with topk_idx[t,j] == e;  counts[E] = Tv
 *   mean_prob[e] = mean over the counting tokens of p[t,e]
 *   losses[0]    = E / (k Tv) * sum_e counts[e] * mean_prob[e]         (1 when both are even)
 *   losses[1]    = mean over the counting tokens of (log sum_e exp logits[t,e])^2
 * With Tv == 0 all of them are 0.
 * logits     [T,E] fp32; -inf excludes an expert for a token, which needs one finite logit; a row that does not count may hold anything
 * topk_idx   [T,k] int32; ids outside [0,E) are not counted
 * token_mask [T] bytes, or NULL
 * counts     [E+1] int32, mean_prob [E] fp32, losses [2] fp32
 * workspace  at least moe_balance_workspace_bytes(T, E) bytes
 * Requires T >= 0, 1 <= k <= E <= MOE_MAX_EXPERTS, k <= MOE_MAX_TOPK, T * k < 2^24.
 */
int moe_balance_loss(const float* logits, const int32_t* topk_idx, const uint8_t* token_mask, int32_t T, int32_t E, int32_t k,
                     int32_t* counts, float* mean_prob, float* losses, void* workspace, size_t workspace_bytes, void* stream);

/* Bytes of scratch moe_balance_loss needs; 0 on invalid sizes. */
size_t moe_balance_workspace_bytes(int32_t T, int32_t E);

/*
 * Gradient with respect to the logits of  sum_{t,j} d_topk_w[t,j] * topk_w[t,j] + coef_balance * losses[0] + coef_z * losses[1],
 * where the selection itself (topk_idx, counts) is constant, as it has no derivative.
 * topk_idx   [T,k] as moe_route_topk selected (distinct ids in [0,E))
 * d_topk_w   [T,k] fp32: gradient with respect to moe_route_topk's gate weights; NULL: zeros
 * token_mask [T] bytes or NULL: tokens that do not count get no part of the auxiliary losses; their gates' gradient stays
 * counts     [E+1] int32 as moe_balance_loss wrote them; NULL only if both coefficients are 0.  Data-parallel devices
 *            may pass the sums of their counts: the losses are then those of the whole batch, and the devices' gradients add up
 * coef_*     finite
 * flags      0 or MOE_RENORM_TOPK, as in the forward call
 * d_logits   [T,E] fp32, written whole
 * With d_topk_w == NULL a row that does not count may hold anything (its gradient is 0).  Sizes as above.
 */
int moe_route_backward(const float* logits, const int32_t* topk_idx, const float* d_topk_w, const uint8_t* token_mask,
                       const int32_t* counts, int32_t T, int32_t E, int32_t k, float coef_balance, float coef_z, uint32_t flags,
                       float* d_logits, void* stream);

/*
 * Gradients of the router's product logits = x W_r:
 *   d_w_router[h,e] = sum_t x[t,h] * d_logits[t,e];  dx[t,h] = dx_in[t,h] + sum_e d_logits[t,e] * w_router[h,e]
 * x_bf16     [T,H] bf16, w_router [H,E] fp32 (unused, may be NULL, without dx), d_logits [T,E] fp32; finite values
 * dx_in      [T,H] bf16, what other branches that read x contribute; may be dx itself; NULL: zeros
 * dx         [T,H] bf16, rounded once by each call that adds to it; NULL: not computed (dx_in must be NULL too)
 * d_w_router [H,E] fp32, written whole
 * workspace  at least moe_router_backward_workspace_bytes(T, H, E) bytes
 * The shared expert's gate (moe_combine's w_shared_gate) is the case E = 1 with d_logits = d_shared_gate.
 * Requires T >= 0, T < 2^24, 1 <= E <= MOE_MAX_EXPERTS, H % 8 == 0, 8 <= H <= MOE_ROUTER_GRAD_MAX_HIDDEN.
 */
int moe_router_backward(const void* x_bf16, const float* w_router, const float* d_logits, int32_t T, int32_t H, int32_t E,
                        const void* dx_in, void* dx, float* d_w_router, void* workspace, size_t workspace_bytes, void* stream);

/* Bytes of scratch moe_router_backward needs; 0 on invalid sizes. */
size_t moe_router_backward_workspace_bytes(int32_t T, int32_t H, int32_t E);

/*
 * Gradients of moe_combine with respect to its gates, for dy, the loss's gradient with respect to y_out:
 *   d_topk_w[t,j]    = sum_h dy[t,h] * y_perm[slot_row[t*k+j],h]       (0 where slot_row is negative)
 *   d_shared_gate[t] = gate_t (1 - gate_t) * sum_h dy[t,h] * y_shared[t,h], the gradient with respect to x[t,:] . w_shared_gate
 * dy_bf16       [T,H] bf16
 * y_perm, slot_row, y_shared, x_bf16, w_shared_gate as in moe_combine; the last three and d_shared_gate: all NULL or none
 * d_topk_w      [T,k] fp32, d_shared_gate [T] fp32
 * flags         0 or MOE_Y_PERM_BF16, as in the forward call
 * Requires T >= 0, T < 2^24, 1 <= k <= MOE_MAX_TOPK, H % 8 == 0, 8 <= H <= MOE_ROUTER_GRAD_MAX_HIDDEN.
 */
int moe_combine_backward(const void* dy_bf16, const void* y_perm, const int32_t* slot_row, int32_t T, int32_t k, int32_t H,
                         const void* y_shared, const void* x_bf16, const float* w_shared_gate, float* d_topk_w,
                         float* d_shared_gate, uint32_t flags, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* MOE_ROUTER_GRAD_H */
