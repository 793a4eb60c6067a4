// What trains the router: balance and z loss with per-expert counts, and the gradients from the combine's gates to the
// router's weights.
#include <cmath>

#include "moe_internal.hpp"
#include "moe_router_grad.h"

namespace moe {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kSlots = MOE_MAX_EXPERTS / kWave;

// softmax of one token's row: expert lane + 64 s in slot s; returns log sum exp
__device__ __forceinline__ float row_softmax(const float* __restrict__ row, int lane, int E, float (&p)[kSlots]) {
  float top = -INFINITY;
#pragma unroll
  for (int s = 0; s < kSlots; ++s) {
    const int e = lane + s * kWave;
    p[s] = e < E ? row[e] : -INFINITY;
    top = fmaxf(top, p[s]);
  }
  top = wave_max(top);
  float sum = 0.f;
#pragma unroll
  for (int s = 0; s < kSlots; ++s) {
    p[s] = lane + s * kWave < E ? expf(p[s] - top) : 0.f;
    sum += p[s];
  }
  sum = wave_sum(sum);
#pragma unroll
  for (int s = 0; s < kSlots; ++s) p[s] /= sum;
  return top + logf(sum);
}

__global__ __launch_bounds__(kThreads) void balance_kernel(const float* __restrict__ logits, const int32_t* __restrict__ idx,
                                                           const uint8_t* __restrict__ mask, int T, int E, int k,
                                                           int32_t* __restrict__ counts, float* __restrict__ mean_prob,
                                                           float* __restrict__ losses) {
  __shared__ int32_t cnt[MOE_MAX_EXPERTS + 1];
  __shared__ float prob[kWaves][MOE_MAX_EXPERTS], zsum[kWaves], part[kWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  for (int e = tid; e <= E; e += kThreads) cnt[e] = 0;
  __syncthreads();
  float mine[kSlots] = {}, z = 0.f;
  for (int t = wave; t < T; t += kWaves) {
    if (mask != nullptr && mask[t] == 0) continue;
    float p[kSlots];
    const float lse = row_softmax(logits + (size_t)t * E, lane, E, p);
#pragma unroll
    for (int s = 0; s < kSlots; ++s) mine[s] += p[s];
    z = fmaf(lse, lse, z);
    if (lane < k) {
      const int e = idx[(size_t)t * k + lane];
      if ((unsigned)e < (unsigned)E) atomicAdd(&cnt[e], 1);
    }
    if (lane == 0) atomicAdd(&cnt[E], 1);
  }
#pragma unroll
  for (int s = 0; s < kSlots; ++s) prob[wave][lane + s * kWave] = mine[s];
  if (lane == 0) zsum[wave] = z;
  __syncthreads();
  const float many = fmaxf((float)cnt[E], 1.f);
  float b = 0.f;
  if (tid <= E) counts[tid] = cnt[tid];
  if (tid == 0) counts[E] = cnt[E];
  if (tid < E) {
    float sum = 0.f;
    for (int w = 0; w < kWaves; ++w) sum += prob[w][tid];
    mean_prob[tid] = sum / many;
    b = sum / many * ((float)cnt[tid] / many);
  }
  b = wave_sum(b);
  if (lane == 0) part[wave] = b;
  __syncthreads();
  if (tid == 0) {
    float sum = 0.f, zs = 0.f;
    for (int w = 0; w < kWaves; ++w) sum += part[w], zs += zsum[w];
    losses[0] = sum * ((float)E / k);
    losses[1] = zs / many;
  }
}

// a wavefront per token
__global__ __launch_bounds__(kThreads) void route_backward_kernel(const float* __restrict__ logits, const int32_t* __restrict__ idx,
                                                                  const float* __restrict__ d_topk_w,
                                                                  const uint8_t* __restrict__ mask,
                                                                  const int32_t* __restrict__ counts, int T, int E, int k,
                                                                  float coef_balance, float coef_z, bool renorm,
                                                                  float* __restrict__ d_logits) {
  const int lane = threadIdx.x & 63, t = blockIdx.x * kWaves + (threadIdx.x >> 6);
  if (t >= T) return;
  const bool counts_in = mask == nullptr || mask[t] != 0;
  float d[kSlots] = {};
  if (counts_in || d_topk_w != nullptr) {
    float p[kSlots];
    const float lse = row_softmax(logits + (size_t)t * E, lane, E, p);
    if (d_topk_w != nullptr) {
      float w[kSlots], dw[kSlots], sum = 0.f;
#pragma unroll
      for (int s = 0; s < kSlots; ++s) {
        dw[s] = 0.f;
        bool picked = false;
        for (int j = 0; j < k; ++j)
          if (idx[(size_t)t * k + j] == lane + s * kWave) picked = true, dw[s] += d_topk_w[(size_t)t * k + j];
        w[s] = renorm && !picked ? 0.f : p[s];
        sum += w[s];
      }
      sum = renorm ? wave_sum(sum) : 1.f;
      float dot = 0.f;
#pragma unroll
      for (int s = 0; s < kSlots; ++s) w[s] /= sum, dot = fmaf(w[s], dw[s], dot);
      dot = wave_sum(dot);
#pragma unroll
      for (int s = 0; s < kSlots; ++s) d[s] = w[s] * (dw[s] - dot);
    }
    if (counts_in && counts != nullptr) {
      const float many = fmaxf((float)counts[E], 1.f), even = (float)k * many / (float)E;
      const float c = coef_balance * E / k / many / many, cz = 2.f * coef_z / many * lse;
      float g[kSlots], dot = 0.f;
#pragma unroll
      for (int s = 0; s < kSlots; ++s) {
        const int e = lane + s * kWave;
        g[s] = e < E ? c * ((float)counts[e] - even) : 0.f;  // (the gradient is the same with any constant taken off)
        dot = fmaf(p[s], g[s], dot);
      }
      dot = wave_sum(dot);
#pragma unroll
      for (int s = 0; s < kSlots; ++s) d[s] += p[s] * (g[s] - dot + cz);
    }
  }
#pragma unroll
  for (int s = 0; s < kSlots; ++s)
    if (lane + s * kWave < E) d_logits[(size_t)t * E + lane + s * kWave] = d[s];
}

__global__ __launch_bounds__(kThreads) void router_weight_grad_kernel(const uint16_t* __restrict__ x,
                                                                      const float* __restrict__ d_logits, int T, int H, int E,
                                                                      float* __restrict__ d_w) {
  const int e = blockIdx.x, h = blockIdx.y * kThreads + threadIdx.x;
  if (h >= H) return;
  float sum = 0.f;
  for (int t = 0; t < T; ++t) sum = fmaf(bf16_bits_to_f32(x[(size_t)t * H + h]), d_logits[(size_t)t * E + e], sum);
  d_w[(size_t)h * E + e] = sum;
}

__global__ __launch_bounds__(kThreads) void router_input_grad_kernel(const float* __restrict__ w_router,
                                                                     const float* __restrict__ d_logits, int H, int E,
                                                                     const uint16_t* dx_in, uint16_t* dx) {
  const int t = blockIdx.x, h = blockIdx.y * kThreads + threadIdx.x;
  if (h >= H) return;
  float sum = 0.f;
  for (int e = 0; e < E; ++e) sum = fmaf(d_logits[(size_t)t * E + e], w_router[(size_t)h * E + e], sum);
  if (dx_in != nullptr) sum += bf16_bits_to_f32(dx_in[(size_t)t * H + h]);
  dx[(size_t)t * H + h] = (uint16_t)f32_to_bf16_bits(sum);
}

__device__ __forceinline__ float at(const float* p, size_t i) { return p[i]; }
__device__ __forceinline__ float at(const uint16_t* p, size_t i) { return bf16_bits_to_f32(p[i]); }

// a wavefront per (token, slot); slot k is the shared expert's gate
template <typename YT>
__global__ __launch_bounds__(kThreads) void combine_backward_kernel(const uint16_t* __restrict__ dy, const YT* __restrict__ y_perm,
                                                                    const int32_t* __restrict__ slot_row, int T, int k, int H,
                                                                    const YT* __restrict__ y_shared,
                                                                    const uint16_t* __restrict__ x,
                                                                    const float* __restrict__ w_shared_gate,
                                                                    float* __restrict__ d_topk_w,
                                                                    float* __restrict__ d_shared_gate) {
  const int t = blockIdx.x, lane = threadIdx.x & 63;
  for (int j = threadIdx.x >> 6; j < k + (y_shared != nullptr); j += kWaves) {
    const int row = j < k ? slot_row[(size_t)t * k + j] : t;
    const YT* y = j < k ? y_perm : y_shared;
    float sum = 0.f, z = 0.f;
    if (row >= 0)
      for (int h = lane; h < H; h += kWave) {
        sum = fmaf(at(dy, (size_t)t * H + h), at(y, (size_t)row * H + h), sum);
        if (j == k) z = fmaf(at(x, (size_t)t * H + h), w_shared_gate[h], z);
      }
    sum = wave_sum(sum);
    if (j < k) {
      if (lane == 0) d_topk_w[(size_t)t * k + j] = sum;
    } else {
      const float gate = 1.f / (1.f + expf(-wave_sum(z)));
      if (lane == 0) d_shared_gate[t] = gate * (1.f - gate) * sum;
    }
  }
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int losses_status(int32_t T, int32_t E, int32_t k) {
  if (T < 0 || E < 1 || E > MOE_MAX_EXPERTS || k < 1 || k > E || k > MOE_MAX_TOPK || (int64_t)T * k >= (1 << 24))
    return MOE_ERR_INVALID_ARG;
  return MOE_OK;
}

int router_status(int32_t T, int32_t H, int32_t E) {
  if (T < 0 || T >= (1 << 24) || E < 1 || E > MOE_MAX_EXPERTS || H < 8) return MOE_ERR_INVALID_ARG;
  return H % 8 != 0 ? MOE_ERR_UNSUPPORTED_SHAPE : MOE_OK;
}

int blocks(int n) { return (n + kThreads - 1) / kThreads; }

}  // namespace
}  // namespace moe

extern "C" {

size_t moe_balance_workspace_bytes(int32_t T, int32_t E) {
  return moe::losses_status(T, E, 1) == MOE_OK ? 256 : 0;
}

int moe_balance_loss(const float* logits, const int32_t* topk_idx, const uint8_t* token_mask, int32_t T, int32_t E, int32_t k,
                     int32_t* counts, float* mean_prob, float* losses, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace moe;
  const int st = losses_status(T, E, k);
  if (st != MOE_OK) return st;
  if (T > 0 && (logits == nullptr || topk_idx == nullptr)) return MOE_ERR_INVALID_ARG;
  if (counts == nullptr || mean_prob == nullptr || losses == nullptr) return MOE_ERR_INVALID_ARG;
  if (workspace == nullptr || !aligned16(workspace) || workspace_bytes < moe_balance_workspace_bytes(T, E)) return MOE_ERR_WORKSPACE;
  hipLaunchKernelGGL(balance_kernel, dim3(1), dim3(kThreads), 0, static_cast<hipStream_t>(stream), logits, topk_idx, token_mask, T,
                     E, k, counts, mean_prob, losses);
  return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

int moe_route_backward(const float* logits, const int32_t* topk_idx, const float* d_topk_w, const uint8_t* token_mask,
                       const int32_t* counts, int32_t T, int32_t E, int32_t k, float coef_balance, float coef_z, uint32_t flags,
                       float* d_logits, void* stream) {
  using namespace moe;
  const int st = losses_status(T, E, k);
  if (st != MOE_OK) return st;
  if (flags & ~(uint32_t)MOE_RENORM_TOPK) return MOE_ERR_INVALID_ARG;
  if (T > 0 && (logits == nullptr || topk_idx == nullptr || d_logits == nullptr)) return MOE_ERR_INVALID_ARG;
  if (!std::isfinite(coef_balance) || !std::isfinite(coef_z)) return MOE_ERR_INVALID_ARG;
  if (counts == nullptr && (coef_balance != 0.f || coef_z != 0.f)) return MOE_ERR_INVALID_ARG;
  if (T == 0) return MOE_OK;
  hipLaunchKernelGGL(route_backward_kernel, dim3((T + kWaves - 1) / kWaves), dim3(kThreads), 0, static_cast<hipStream_t>(stream),
                     logits, topk_idx, d_topk_w, token_mask, counts, T, E, k, coef_balance, coef_z,
                     (flags & MOE_RENORM_TOPK) != 0, d_logits);
  return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

size_t moe_router_backward_workspace_bytes(int32_t T, int32_t H, int32_t E) {
  return moe::router_status(T, H, E) == MOE_OK ? 256 : 0;
}

int moe_router_backward(const void* x_bf16, const float* w_router, const float* d_logits, int32_t T, int32_t H, int32_t E,
                        const void* dx_in, void* dx, float* d_w_router, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace moe;
  const int st = router_status(T, H, E);
  if (st != MOE_OK) return st;
  if (T > 0 && (x_bf16 == nullptr || d_logits == nullptr)) return MOE_ERR_INVALID_ARG;
  if (d_w_router == nullptr || (dx == nullptr ? dx_in != nullptr : w_router == nullptr)) return MOE_ERR_INVALID_ARG;
  if (!aligned16(x_bf16) || !aligned16(dx_in) || !aligned16(dx)) return MOE_ERR_INVALID_ARG;
  if (workspace == nullptr || !aligned16(workspace) || workspace_bytes < moe_router_backward_workspace_bytes(T, H, E))
    return MOE_ERR_WORKSPACE;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  hipLaunchKernelGGL(router_weight_grad_kernel, dim3(E, blocks(H)), dim3(kThreads), 0, s, static_cast<const uint16_t*>(x_bf16),
                     d_logits, T, H, E, d_w_router);
  if (dx != nullptr && T > 0)
    hipLaunchKernelGGL(router_input_grad_kernel, dim3(T, blocks(H)), dim3(kThreads), 0, s, w_router, d_logits, H, E,
                       static_cast<const uint16_t*>(dx_in), static_cast<uint16_t*>(dx));
  return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

int moe_combine_backward(const void* dy_bf16, const void* y_perm, const int32_t* slot_row, int32_t T, int32_t k, int32_t H,
                         const void* y_shared, const void* x_bf16, const float* w_shared_gate, float* d_topk_w,
                         float* d_shared_gate, uint32_t flags, void* stream) {
  using namespace moe;
  if (T < 0 || k < 1 || k > MOE_MAX_TOPK || H < 8) return MOE_ERR_INVALID_ARG;
  if (flags & ~(uint32_t)MOE_Y_PERM_BF16) return MOE_ERR_INVALID_ARG;
  const bool gate = w_shared_gate != nullptr;
  if (T > 0) {
    if (dy_bf16 == nullptr || y_perm == nullptr || slot_row == nullptr || d_topk_w == nullptr) return MOE_ERR_INVALID_ARG;
    if ((y_shared != nullptr) != gate || (x_bf16 != nullptr) != gate || (d_shared_gate != nullptr) != gate)
      return MOE_ERR_INVALID_ARG;
  }
  if (H % 8 != 0) return MOE_ERR_UNSUPPORTED_SHAPE;
  if (!aligned16(dy_bf16) || !aligned16(y_perm) || !aligned16(y_shared) || !aligned16(x_bf16) || !aligned16(w_shared_gate))
    return MOE_ERR_INVALID_ARG;
  if (T == 0) return MOE_OK;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const uint16_t *dy = static_cast<const uint16_t*>(dy_bf16), *x = static_cast<const uint16_t*>(x_bf16);
  if (flags & MOE_Y_PERM_BF16)
    hipLaunchKernelGGL(combine_backward_kernel<uint16_t>, dim3(T), dim3(kThreads), 0, s, dy, static_cast<const uint16_t*>(y_perm),
                       slot_row, T, k, H, static_cast<const uint16_t*>(y_shared), x, w_shared_gate, d_topk_w, d_shared_gate);
  else
    hipLaunchKernelGGL(combine_backward_kernel<float>, dim3(T), dim3(kThreads), 0, s, dy, static_cast<const float*>(y_perm),
                       slot_row, T, k, H, static_cast<const float*>(y_shared), x, w_shared_gate, d_topk_w, d_shared_gate);
  return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

}  // extern "C"
