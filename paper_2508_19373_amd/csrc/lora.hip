// Low-rank adapters of many requests beside one projection: y += scale_a (x A_a^T) B_a^T with the row's own adapter a, and the
// gradients of A, B and x.
#include "moe_internal.hpp"
#include "moe_lora.h"

namespace moe {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float load_f32(const uint16_t* p) { return bf16_bits_to_f32(*p); }
__device__ __forceinline__ float load_f32(const float* p) { return *p; }
__device__ __forceinline__ void store_f32(uint16_t* p, float v) { *p = (uint16_t)f32_to_bf16_bits(v); }
__device__ __forceinline__ void store_f32(float* p, float v) { *p = v; }

// v[t,j] = x[t,:] . A_a[j,:]: a workgroup per row, a wavefront per j.
__global__ __launch_bounds__(kThreads) void lora_shrink_kernel(const uint16_t* __restrict__ x, const int32_t* __restrict__ idx,
                                                               int K, int rank, int L, const uint16_t* __restrict__ lora_a,
                                                               float* __restrict__ v) {
  const int t = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int a = idx[t];
  for (int j = wave; j < rank; j += kThreads / kWave) {
    float sum = 0.f;
    if ((unsigned)a < (unsigned)L)
      for (int k = lane; k < K; k += kWave)
        sum = fmaf(bf16_bits_to_f32(x[(size_t)t * K + k]), bf16_bits_to_f32(lora_a[((size_t)a * rank + j) * K + k]), sum);
    sum = wave_sum(sum);
    if (lane == 0) v[(size_t)t * rank + j] = sum;
  }
}

// y_out[t,n] = y_in[t,n] + scale sum_j v[t,j] B_a[n,j]: a lane per n.
template <typename YT>
__global__ __launch_bounds__(kThreads) void lora_expand_kernel(const float* __restrict__ v, const int32_t* __restrict__ idx, int N,
                                                               int rank, int L, const uint16_t* __restrict__ lora_b,
                                                               const float* __restrict__ scale, const YT* y_in, YT* y_out) {
  const int t = blockIdx.x, n = blockIdx.y * kThreads + threadIdx.x;
  if (n >= N) return;
  const int a = idx[t];
  float sum = 0.f;
  if ((unsigned)a < (unsigned)L) {
    for (int j = 0; j < rank; ++j)
      sum = fmaf(v[(size_t)t * rank + j], bf16_bits_to_f32(lora_b[((size_t)a * N + n) * rank + j]), sum);
    sum *= scale[a];
  }
  const size_t at = (size_t)t * N + n;
  store_f32(y_out + at, y_in != nullptr ? load_f32(y_in + at) + sum : sum);
}

// u[t,j] = scale sum_n dy[t,n] B_a[n,j]
__global__ __launch_bounds__(kThreads) void lora_grad_v_kernel(const uint16_t* __restrict__ dy, const int32_t* __restrict__ idx,
                                                               int N, int rank, int L, const uint16_t* __restrict__ lora_b,
                                                               const float* __restrict__ scale, float* __restrict__ u) {
  const int t = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int a = idx[t];
  for (int j = wave; j < rank; j += kThreads / kWave) {
    float sum = 0.f;
    if ((unsigned)a < (unsigned)L)
      for (int n = lane; n < N; n += kWave)
        sum = fmaf(bf16_bits_to_f32(dy[(size_t)t * N + n]), bf16_bits_to_f32(lora_b[((size_t)a * N + n) * rank + j]), sum);
    sum = wave_sum(sum);
    if (lane == 0) u[(size_t)t * rank + j] = sum != 0.f ? sum * scale[a] : 0.f;
  }
}

// dx[t,k] = dx_in[t,k] + sum_j u[t,j] A_a[j,k]
__global__ __launch_bounds__(kThreads) void lora_grad_x_kernel(const float* __restrict__ u, const int32_t* __restrict__ idx, int K,
                                                               int rank, int L, const uint16_t* __restrict__ lora_a,
                                                               const uint16_t* dx_in, uint16_t* dx) {
  const int t = blockIdx.x, k = blockIdx.y * kThreads + threadIdx.x;
  if (k >= K) return;
  const int a = idx[t];
  float sum = 0.f;
  if ((unsigned)a < (unsigned)L)
    for (int j = 0; j < rank; ++j)
      sum = fmaf(u[(size_t)t * rank + j], bf16_bits_to_f32(lora_a[((size_t)a * rank + j) * K + k]), sum);
  const size_t at = (size_t)t * K + k;
  store_f32(dx + at, dx_in != nullptr ? load_f32(dx_in + at) + sum : sum);
}

// grad[a] = c_a * sum over the rows t of adapter a of w[t,j] z[t,c], at [j][c] or [c][j]
__global__ __launch_bounds__(kThreads) void lora_outer_kernel(const uint16_t* __restrict__ z, const float* __restrict__ w,
                                                              const int32_t* __restrict__ idx, int T, int C, int rank,
                                                              const float* __restrict__ scale, bool column_major,
                                                              float* __restrict__ grad) {
  const int a = blockIdx.x / rank, j = blockIdx.x % rank, c = blockIdx.y * kThreads + threadIdx.x;
  if (c >= C) return;
  float sum = 0.f;
  for (int t = 0; t < T; ++t)
    if (idx[t] == a) sum = fmaf(w[(size_t)t * rank + j], bf16_bits_to_f32(z[(size_t)t * C + c]), sum);
  if (scale != nullptr) sum *= scale[a];
  grad[(size_t)a * rank * C + (column_major ? (size_t)c * rank + j : (size_t)j * C + c)] = sum;
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int size_status(int32_t T, int32_t K, int32_t N, int32_t rank, int32_t L) {
  if (T < 0 || T >= (1 << 24) || K < 8 || N < 8 || rank < 1 || L < 1 || L > MOE_LORA_MAX_ADAPTERS) return MOE_ERR_INVALID_ARG;
  if (K % 8 != 0 || N % 8 != 0 || rank % 8 != 0 || rank > MOE_LORA_MAX_RANK) return MOE_ERR_UNSUPPORTED_SHAPE;
  return MOE_OK;
}

int blocks(int n) { return (n + kThreads - 1) / kThreads; }

}  // namespace
}  // namespace moe

extern "C" {

size_t moe_lora_workspace_bytes(int32_t T, int32_t K, int32_t N, int32_t rank, int32_t n_adapters, int32_t backward) {
  if (moe::size_status(T, K, N, rank, n_adapters) != MOE_OK) return 0;
  return 256 + (size_t)T * rank * sizeof(float);
}

int moe_lora_forward(const void* x_bf16, const int32_t* adapter_idx, int32_t T, int32_t K, int32_t N, int32_t rank,
                     int32_t n_adapters, const void* lora_a, const void* lora_b, const float* scale, const void* y_in,
                     void* y_out, float* v, void* workspace, size_t workspace_bytes, uint32_t flags, void* stream) {
  using namespace moe;
  const int st = size_status(T, K, N, rank, n_adapters);
  if (st != MOE_OK) return st;
  if (flags & ~(uint32_t)MOE_OUT_F32) return MOE_ERR_INVALID_ARG;
  if (lora_a == nullptr || lora_b == nullptr || scale == nullptr) return MOE_ERR_INVALID_ARG;
  if (T > 0 && (x_bf16 == nullptr || adapter_idx == nullptr || y_out == nullptr)) return MOE_ERR_INVALID_ARG;
  if (!aligned16(x_bf16) || !aligned16(lora_a) || !aligned16(lora_b) || !aligned16(y_in) || !aligned16(y_out) || !aligned16(v))
    return MOE_ERR_INVALID_ARG;
  if (workspace == nullptr || !aligned16(workspace) || workspace_bytes < moe_lora_workspace_bytes(T, K, N, rank, n_adapters, 0))
    return MOE_ERR_WORKSPACE;
  if (T == 0) return MOE_OK;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (v == nullptr) v = static_cast<float*>(workspace);
  hipLaunchKernelGGL(lora_shrink_kernel, dim3(T), dim3(kThreads), 0, s, static_cast<const uint16_t*>(x_bf16), adapter_idx, K, rank,
                     n_adapters, static_cast<const uint16_t*>(lora_a), v);
  if (flags & MOE_OUT_F32)
    hipLaunchKernelGGL(lora_expand_kernel<float>, dim3(T, blocks(N)), dim3(kThreads), 0, s, v, adapter_idx, N, rank, n_adapters,
                       static_cast<const uint16_t*>(lora_b), scale, static_cast<const float*>(y_in), static_cast<float*>(y_out));
  else
    hipLaunchKernelGGL(lora_expand_kernel<uint16_t>, dim3(T, blocks(N)), dim3(kThreads), 0, s, v, adapter_idx, N, rank,
                       n_adapters, static_cast<const uint16_t*>(lora_b), scale, static_cast<const uint16_t*>(y_in),
                       static_cast<uint16_t*>(y_out));
  return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

int moe_lora_backward(const void* x_bf16, const void* dy_bf16, const int32_t* adapter_idx, int32_t T, int32_t K, int32_t N,
                      int32_t rank, int32_t n_adapters, const void* lora_a, const void* lora_b, const float* scale,
                      const float* v, const void* dx_in, void* dx, float* grad_a, float* grad_b, void* workspace,
                      size_t workspace_bytes, void* stream) {
  using namespace moe;
  const int st = size_status(T, K, N, rank, n_adapters);
  if (st != MOE_OK) return st;
  if (lora_a == nullptr || lora_b == nullptr || scale == nullptr || grad_a == nullptr || grad_b == nullptr)
    return MOE_ERR_INVALID_ARG;
  if (T > 0 && (x_bf16 == nullptr || dy_bf16 == nullptr || adapter_idx == nullptr || v == nullptr)) return MOE_ERR_INVALID_ARG;
  if (dx == nullptr && dx_in != nullptr) return MOE_ERR_INVALID_ARG;
  if (!aligned16(x_bf16) || !aligned16(dy_bf16) || !aligned16(lora_a) || !aligned16(lora_b) || !aligned16(v) || !aligned16(dx_in) ||
      !aligned16(dx) || !aligned16(grad_a) || !aligned16(grad_b))
    return MOE_ERR_INVALID_ARG;
  if (workspace == nullptr || !aligned16(workspace) || workspace_bytes < moe_lora_workspace_bytes(T, K, N, rank, n_adapters, 1))
    return MOE_ERR_WORKSPACE;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const uint16_t *x = static_cast<const uint16_t*>(x_bf16), *dy = static_cast<const uint16_t*>(dy_bf16);
  const uint16_t *la = static_cast<const uint16_t*>(lora_a), *lb = static_cast<const uint16_t*>(lora_b);
  float* const u = static_cast<float*>(workspace);
  if (T > 0) {
    hipLaunchKernelGGL(lora_grad_v_kernel, dim3(T), dim3(kThreads), 0, s, dy, adapter_idx, N, rank, n_adapters, lb, scale, u);
    if (dx != nullptr)
      hipLaunchKernelGGL(lora_grad_x_kernel, dim3(T, blocks(K)), dim3(kThreads), 0, s, u, adapter_idx, K, rank, n_adapters, la,
                         static_cast<const uint16_t*>(dx_in), static_cast<uint16_t*>(dx));
  }
  hipLaunchKernelGGL(lora_outer_kernel, dim3(n_adapters * rank, blocks(K)), dim3(kThreads), 0, s, x, u, adapter_idx, T, K, rank,
                     nullptr, false, grad_a);
  hipLaunchKernelGGL(lora_outer_kernel, dim3(n_adapters * rank, blocks(N)), dim3(kThreads), 0, s, dy, v, adapter_idx, T, N, rank,
                     scale, true, grad_b);
  return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

}  // extern "C"
