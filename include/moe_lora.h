/*
 * moe_lora.h -- C ABI of low-rank adapters of many requests beside one shared projection (gfx950).
 *
 * A server keeps one set of weights for all requests and a small correction for each tenant: where the projection computes
 * y = x W^T, a request with adapter a gets y + scale_a (x A_a^T) B_a^T as well, with A_a of `rank` rows and B_a of `rank` columns.
 * One call serves a batch whose rows have adapters in any order, or none.  The projection's own result is an input (y_in): it comes
 * from whatever computed it (moe_expert_ffn's down projection, moe_combine, a library).
 *
 * A tensor-parallel device whose projection is sliced along K (a down projection) passes its columns of A, whole B, and adds its
 * partial result to its partial y; beside a module whose input every device has whole, a device takes its share of the rank
 * (rows of A, columns of B).  Either way the devices' results add up to the unsharded one, as those of the experts do.
 *
 * Conventions as in moe_shard.h: status codes (MOE_OK / MOE_ERR_*), validation on the host before any HIP call, no allocation, no
 * synchronisation, work enqueued on `stream`; all pointers are DEVICE pointers owned by the caller, 16-byte aligned (adapter_idx and
 * scale: 4-byte).  With T == 0 the buffers of T rows may be NULL.  Values must be finite, except in the rows of x, dy and v whose
 * request has no adapter, and in lora_a, lora_b and scale of an adapter that no row has: those are not used.
 * A call writes all of its workspace that it reads, so nothing has to start at zero; calls that overlap on one GPU (different
 * streams, graphs replayed concurrently) each bring their own.
 */
#ifndef MOE_LORA_H
#define MOE_LORA_H

#include "moe_shard.h"

#ifdef __cplusplus
extern "C" {
#endif

#define MOE_LORA_MAX_ADAPTERS 256
#define MOE_LORA_MAX_RANK 128
#define MOE_LORA_MAX_COLUMNS 262144

/*
 * v[t,:] = x[t,:] A_a^T (fp32, a = adapter_idx[t]),  y_out[t,:] = y_in[t,:] + scale[a] * v[t,:] B_a^T
 * x_bf16       [T,K] bf16
 * adapter_idx  [T] int32: the row's adapter; outside [0, n_adapters): none, y_out[t,:] = y_in[t,:] and v[t,:] = 0
 * lora_a       [n_adapters][rank][K] bf16
 * lora_b       [n_adapters][N][rank] bf16
 * scale        [n_adapters] fp32
 * y_in         [T,N] bf16 (fp32 with MOE_OUT_F32); may be y_out itself; NULL: zeros
 * y_out        [T,N] of the same type; rounded once
 * v            [T,rank] fp32, kept for moe_lora_backward; NULL: not kept
 * workspace    at least moe_lora_workspace_bytes(..., 0) bytes
 * flags        0 or MOE_OUT_F32
 * Requires T >= 0, T < 2^24, 1 <= n_adapters <= MOE_LORA_MAX_ADAPTERS, rank % 8 == 0, 8 <= rank <= MOE_LORA_MAX_RANK,
 * K % 8 == 0, N % 8 == 0, 8 <= K, N <= MOE_LORA_MAX_COLUMNS.  Apart from y_in and y_out no two buffers may overlap.
 */
int moe_lora_forward(const void* x_bf16, const int32_t* adapter_idx, int32_t T, int32_t K, int32_t N, int32_t rank,
                     int32_t n_adapters, const void* lora_a, const void* lora_b, const float* scale, const void* y_in,
                     void* y_out, float* v, void* workspace, size_t workspace_bytes, uint32_t flags, void* stream);

/*
 * Gradients of moe_lora_forward for dy, the loss's gradient with respect to y_out (that with respect to y_in is dy itself):
 *   u[t,:] = scale[a] * dy[t,:] B_a;  dx[t,:] = dx_in[t,:] + u[t,:] A_a
 *   grad_a[a] = sum over the rows t of adapter a of u[t,:]^T x[t,:];  grad_b[a] = scale[a] * sum of dy[t,:]^T v[t,:]
 * dy_bf16      [T,N] bf16
 * v            [T,rank] fp32 as moe_lora_forward left it
 * dx_in        [T,K] bf16, what other branches that read x contribute; may be dx itself; NULL: zeros
 * dx           [T,K] bf16, rounded once by each call that adds to it; NULL: not computed (dx_in must be NULL too)
 * grad_a       [n_adapters][rank][K] fp32, grad_b [n_adapters][N][rank] fp32: written whole, zeros for an adapter without rows
 * workspace    at least moe_lora_workspace_bytes(..., 1) bytes
 * Sums over rows are taken in a fixed order: the same call gives the same bits.  Sizes as above.
 */
int moe_lora_backward(const void* x_bf16, const void* dy_bf16, const int32_t* adapter_idx, int32_t T, int32_t K, int32_t N,
                      int32_t rank, int32_t n_adapters, const void* lora_a, const void* lora_b, const float* scale,
                      const float* v, const void* dx_in, void* dx, float* grad_a, float* grad_b, void* workspace,
                      size_t workspace_bytes, void* stream);

/* Bytes of scratch of moe_lora_forward (backward == 0) or moe_lora_backward; 0 on invalid sizes. */
size_t moe_lora_workspace_bytes(int32_t T, int32_t K, int32_t N, int32_t rank, int32_t n_adapters, int32_t backward);

#ifdef __cplusplus
}
#endif
#endif /* MOE_LORA_H */
