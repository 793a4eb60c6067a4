// What trains the router: balance and z loss with per-expert counts, and the gradients from the combine's gates to the
// router's weights.
#include <cmath>

#include "moe_router_grad.h"
#include "skinny.hpp"

namespace moe {
namespace {

using namespace skinny;

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;

// ---- softmax rows ----------------------------------------------------------------------------------------------------------
// G lanes (8 to 64) share a token and its E experts, expert l + G s in slot s of the group's lane l: with 8 experts a wavefront holds
// eight tokens, with 60 one, and every load is of neighbouring words.  U tokens one after the other: their loads are in flight
// together, and with 64 lanes a token four tokens' reductions are one.
//
// op over the group's lanes for each of U values; every lane gets them.
template <int G, int U, typename Op>
__device__ __forceinline__ void group_reduce(float (&v)[U], Op op) {
#ifdef __HIP_DEVICE_COMPILE__
  if constexpr (G == 64 && U == 4) {
    // halves of two values side by side, quarters of four; then within 16 lanes all four at a time (row_ror:8, :4, quad_perm)
    const auto pair = [&](float a, float b) {
      const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
      return op(__uint_as_float(h[0]), __uint_as_float(h[1]));
    };
    const auto q = __builtin_amdgcn_permlane16_swap(__float_as_uint(pair(v[0], v[1])), __float_as_uint(pair(v[2], v[3])), false, false);
    float x = op(__uint_as_float(q[0]), __uint_as_float(q[1]));
    const auto move = [](float y, auto ctrl) {
      return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(y), decltype(ctrl)::value, 0xF, 0xF, true));
    };
    x = op(x, move(x, std::integral_constant<int, 0x128>{}));
    x = op(x, move(x, std::integral_constant<int, 0x124>{}));
    x = op(x, move(x, std::integral_constant<int, 0x4E>{}));
    x = op(x, move(x, std::integral_constant<int, 0xB1>{}));
    const int lane_of[4] = {0, 32, 16, 48};
#pragma unroll
    for (int u = 0; u < 4; ++u) v[u] = __int_as_float((int)__builtin_amdgcn_readlane(__float_as_int(x), lane_of[u]));
    return;
  }
#endif
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if constexpr (G == 64) {
      v[u] = wave_reduce(v[u], op);
    } else {
#pragma unroll
      for (int d = G / 2; d >= 1; d /= 2) v[u] = op(v[u], __shfl_xor(v[u], d));
    }
  }
}
template <int G, int U>
__device__ __forceinline__ void group_sum(float (&v)[U]) {
  group_reduce<G, U>(v, [](float a, float b) { return a + b; });
}

// p: the tokens' logits on entry, exp(logit - the largest) on return (0 past E), whose sum is `sum`; lse: log sum exp.
template <int G, int S, int U>
__device__ __forceinline__ void group_softmax(float (&p)[U][S], int l, int E, float (&sum)[U], float (&lse)[U]) {
  float top[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    top[u] = -INFINITY;
#pragma unroll
    for (int s = 0; s < S; ++s) top[u] = fmaxf(top[u], l + G * s < E ? p[u][s] : -INFINITY);
  }
  group_reduce<G, U>(top, [](float a, float b) { return fmaxf(a, b); });
#pragma unroll
  for (int u = 0; u < U; ++u) {
    sum[u] = 0.f;
#pragma unroll
    for (int s = 0; s < S; ++s) {
      p[u][s] = l + G * s < E ? expf(p[u][s] - top[u]) : 0.f;
      sum[u] += p[u][s];
    }
  }
  group_sum<G, U>(sum);
#pragma unroll
  for (int u = 0; u < U; ++u) lse[u] = top[u] + logf(sum[u]);
}

// ---- balance loss ----------------------------------------------------------------------------------------------------------
// A workgroup takes every gridDim.x-th run of tokens and leaves the sums of its probabilities, squared logarithms and counts; the
// counts are integers added in LDS, whose order does not matter, the rest is added in a fixed order.  One workgroup alone finishes by
// itself, several leave their sums to balance_join_kernel.  16384 tokens of 64 experts: 5.9 us (5.5 MB; a launch alone is 2.5) and 5.4 for the
// 256 parts that one compute unit reads to join them.
constexpr int kLossThreads = 512, kLossWaves = kLossThreads / kWave;

struct Balance {
  const float* logits;
  const int32_t* idx;
  const uint8_t* mask;
  int T, E, k;
  int32_t* counts;    // [E+1]
  float* mean_prob;   // [E]
  float* losses;      // [2]
  float* part_prob;   // [workgroups][E+1]: sums of p, of lse^2
  int32_t* part_cnt;  // [workgroups][E+1]
};

// cnt, prob: totals in LDS, [E] of prob being the sum of squares.
__device__ __forceinline__ void balance_finish(const Balance& b, const int32_t* cnt, const float* prob, float* s_red) {
  const int tid = threadIdx.x, E = b.E;
  const float many = fmaxf((float)cnt[E], 1.f);
  float sum = 0.f;
  for (int e = tid; e <= E; e += kLossThreads) {
    b.counts[e] = cnt[e];
    if (e < E) {
      const float mean = prob[e] / many;
      b.mean_prob[e] = mean;
      sum = fmaf(mean, (float)cnt[e] / many, sum);
    }
  }
  sum = wave_sum(sum);
  if ((tid & 63) == 0) s_red[tid >> 6] = sum;
  __syncthreads();
  if (tid == 0) {
    float total = 0.f;
#pragma unroll
    for (int w = 0; w < kLossWaves; ++w) total += s_red[w];
    b.losses[0] = total * ((float)E / b.k);
    b.losses[1] = prob[E] / many;
  }
}

template <int G, int S>
__global__ __launch_bounds__(kLossThreads) void balance_kernel(Balance b) {
  constexpr int kGroups = kLossThreads / G, U = G == 64 ? 4 : 2, PICKED = G < MOE_MAX_TOPK ? 2 : 1;
  __shared__ int32_t cnt[MOE_MAX_EXPERTS + 1];
  __shared__ float sums[kGroups][G * S], zsum[kGroups], total[MOE_MAX_EXPERTS + 1], red[kLossWaves];
  const int tid = threadIdx.x, l = tid & (G - 1), group = tid / G, E = b.E;
  for (int e = tid; e <= E; e += kLossThreads) cnt[e] = 0;
  __syncthreads();
  float mine[S], z = 0.f;
#pragma unroll
  for (int s = 0; s < S; ++s) mine[s] = 0.f;
  // (no load under a condition, which would be waited for at once)
  const uint8_t* const mask = b.mask != nullptr ? b.mask : reinterpret_cast<const uint8_t*>(b.logits);
  const int step = gridDim.x * kGroups;
  for (int t0 = blockIdx.x * kGroups + group; t0 < b.T; t0 += U * step) {
    float p[U][S], all[U], lse[U];
    int e[U][PICKED];
    bool in[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = min(t0 + u * step, b.T - 1);
      in[u] = mask[b.mask != nullptr ? t : 0] != 0 || b.mask == nullptr;
#pragma unroll
      for (int s = 0; s < S; ++s) p[u][s] = b.logits[(size_t)t * E + min(l + G * s, E - 1)];
#pragma unroll
      for (int i = 0; i < PICKED; ++i) e[u][i] = b.idx[(size_t)t * b.k + min(l + G * i, b.k - 1)];
    }
    group_softmax<G, S, U>(p, l, E, all, lse);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (!in[u] || t0 + u * step >= b.T) continue;
#pragma unroll
      for (int i = 0; i < PICKED; ++i)
        if (l + G * i < b.k && (unsigned)e[u][i] < (unsigned)E) atomicAdd(&cnt[e[u][i]], 1);
      if (l == 0) atomicAdd(&cnt[E], 1);
      z = fmaf(lse[u], lse[u], z);
#pragma unroll
      for (int s = 0; s < S; ++s) mine[s] += p[u][s] / all[u];
    }
  }
#pragma unroll
  for (int s = 0; s < S; ++s) sums[group][l + G * s] = mine[s];
  if (l == 0) zsum[group] = z;
  __syncthreads();
  for (int e = tid; e <= E; e += kLossThreads) {
    float sum = 0.f;
#pragma unroll 8
    for (int g = 0; g < kGroups; ++g) sum += e < E ? sums[g][e] : zsum[g];
    total[e] = sum;
  }
  __syncthreads();
  if (gridDim.x == 1) return balance_finish(b, cnt, total, red);
  for (int e = tid; e <= E; e += kLossThreads) {
    b.part_prob[(size_t)blockIdx.x * (E + 1) + e] = total[e];
    b.part_cnt[(size_t)blockIdx.x * (E + 1) + e] = cnt[e];
  }
}

// 64 columns at a time, an eighth of the parts a wavefront, sixteen of them in flight.
__global__ __launch_bounds__(kLossThreads) void balance_join_kernel(Balance b, int parts) {
  __shared__ int32_t cnt[MOE_MAX_EXPERTS + 1], s_cnt[kLossWaves][kWave];
  __shared__ float total[MOE_MAX_EXPERTS + 1], s_sum[kLossWaves][kWave], red[kLossWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, E1 = b.E + 1;
  for (int e0 = 0; e0 < E1; e0 += kWave) {
    const int e = e0 + lane, at = min(e, E1 - 1);
    float sum = 0.f;
    int c = 0;
    for (int p0 = wave; p0 < parts; p0 += 16 * kLossWaves) {
      float v[16];
      int n[16];
#pragma unroll
      for (int u = 0; u < 16; ++u) {
        const size_t from = (size_t)min(p0 + u * kLossWaves, parts - 1) * E1 + at;
        v[u] = b.part_prob[from];
        n[u] = b.part_cnt[from];
      }
#pragma unroll
      for (int u = 0; u < 16; ++u)
        if (p0 + u * kLossWaves < parts) sum += v[u], c += n[u];
    }
    s_sum[wave][lane] = sum;
    s_cnt[wave][lane] = c;
    __syncthreads();
    if (wave == 0 && e < E1) {
      float all = 0.f;
      int n = 0;
#pragma unroll
      for (int w = 0; w < kLossWaves; ++w) all += s_sum[w][lane], n += s_cnt[w][lane];
      total[e] = all;
      cnt[e] = n;
    }
    __syncthreads();
  }
  balance_finish(b, cnt, total, red);
}

// ---- gradient of the logits ------------------------------------------------------------------------------------------------
struct RouteBackward {
  const float *logits, *d_topk_w;
  const int32_t *idx, *counts;
  const uint8_t* mask;
  int T, E, k;
  float coef_balance, coef_z;
  bool renorm;
  float* d_logits;
};

// The gradients at the picked experts, k values of a token, come to the lanes of these experts through LDS (a group's own piece of
// it).  The losses' part is p (f - sum p f), that of the gates the same with their own softmax, which without renormalisation is p too:
// one dot product serves both then.  16384 tokens of 64 experts, 8 picked: 6.4 us for 9.4 MB; 64 of 8, 3.0, a launch's time.
template <int G, int S, int U>
__global__ __launch_bounds__(kThreads) void route_backward_kernel(RouteBackward b) {
  constexpr int PICKED = G < MOE_MAX_TOPK ? 2 : 1;  // a lane's share of a token's picked experts
  __shared__ float2 s_picked[kThreads / G][U][G * S];  // (1 if picked, gradient)
  const int l = threadIdx.x & (G - 1), group = threadIdx.x / G, E = b.E, k = b.k;
  const int t0 = (blockIdx.x * (kThreads / G) + group) * U;
  if (t0 >= b.T) return;
  // (no load under a condition, which would be waited for at once: what is not there is read from the logits and not used)
  const bool gates = b.d_topk_w != nullptr, losses = b.counts != nullptr;
  const uint8_t* const mask = b.mask != nullptr ? b.mask : reinterpret_cast<const uint8_t*>(b.logits);
  const float* const d_topk_w = gates ? b.d_topk_w : b.logits;
  float p[U][S], all[U], lse[U], load[S], grads[U][PICKED];
  int ids[U][PICKED];
  bool counted[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const size_t t = min(t0 + u, b.T - 1);
    counted[u] = (mask[b.mask != nullptr ? t : 0] != 0 || b.mask == nullptr) && losses;
#pragma unroll
    for (int s = 0; s < S; ++s) p[u][s] = b.logits[t * E + min(l + G * s, E - 1)];
#pragma unroll
    for (int i = 0; i < PICKED; ++i) {
      ids[u][i] = b.idx[t * k + min(l + G * i, k - 1)];
      grads[u][i] = d_topk_w[gates ? t * k + min(l + G * i, k - 1) : 0];
    }
  }
  // the load's gradient is the same with a constant taken off: off the even load, which leaves small numbers to subtract
  float cz = 0.f;
#pragma unroll
  for (int s = 0; s < S; ++s) load[s] = 0.f;
  if (losses) {
    const float many = fmaxf((float)b.counts[E], 1.f), even = (float)k * many / (float)E;
    const float c = b.coef_balance * (float)E / ((float)k * many * many);
    cz = 2.f * b.coef_z / many;
#pragma unroll
    for (int s = 0; s < S; ++s) load[s] = l + G * s < E ? c * ((float)b.counts[l + G * s] - even) : 0.f;
  }
  if (gates) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int s = 0; s < S; ++s) s_picked[group][u][l + G * s] = make_float2(0.f, 0.f);
    wave_fence();
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < PICKED; ++i)
        if (l + G * i < k && (unsigned)ids[u][i] < (unsigned)E) s_picked[group][u][ids[u][i]] = make_float2(1.f, grads[u][i]);
    wave_fence();
  }
  group_softmax<G, S, U>(p, l, E, all, lse);
  float f[U][S], w[U][S], gate_dot[U], gate_sum[U], dot[U];  // w: the picked experts' own softmax
  const bool renormed = b.renorm && gates;
  if (renormed) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      gate_sum[u] = 0.f;
#pragma unroll
      for (int s = 0; s < S; ++s) {
        w[u][s] = s_picked[group][u][l + G * s].x * p[u][s];
        gate_sum[u] += w[u][s];
      }
    }
    group_sum<G, U>(gate_sum);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    gate_dot[u] = dot[u] = 0.f;
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const float grad = gates ? s_picked[group][u][l + G * s].y : 0.f;
      p[u][s] /= all[u];
      f[u][s] = counted[u] ? load[s] : 0.f;
      if (renormed) {
        w[u][s] /= gate_sum[u] > 0.f ? gate_sum[u] : 1.f;  // (1 exactly where one expert is picked: its gradient is 0)
        gate_dot[u] = fmaf(grad, w[u][s], gate_dot[u]);
      } else {
        f[u][s] += grad;
      }
      dot[u] = fmaf(p[u][s], f[u][s], dot[u]);
    }
  }
  group_sum<G, U>(dot);
  if (renormed) group_sum<G, U>(gate_dot);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (t0 + u >= b.T) break;
    const float z = counted[u] ? cz * lse[u] : 0.f;
#pragma unroll
    for (int s = 0; s < S; ++s) {
      float d = counted[u] || (gates && !b.renorm) ? p[u][s] * (f[u][s] - dot[u] + z) : 0.f;
      if (renormed) d = fmaf(w[u][s], s_picked[group][u][l + G * s].y - gate_dot[u], d);
      if (l + G * s < E) b.d_logits[(size_t)(t0 + u) * E + l + G * s] = d;
    }
  }
}

// One kernel for each number of lanes a token needs.
template <template <int, int> class Launch, typename... Args>
void by_width(int E, Args... args) {
  if (E <= 8) Launch<8, 1>::run(args...);
  else if (E <= 16) Launch<16, 1>::run(args...);
  else if (E <= 32) Launch<32, 1>::run(args...);
  else if (E <= 64) Launch<64, 1>::run(args...);
  else if (E <= 128) Launch<64, 2>::run(args...);
  else Launch<64, 4>::run(args...);
}

// Two steps of two tokens for each group of lanes, at most a workgroup a compute unit (one kernel more joins them).
int loss_workgroups(int T, int E) {
  const int lanes = E <= 8 ? 8 : (E <= 16 ? 16 : (E <= 32 ? 32 : 64));
  const int n = ceil_div(T, 4 * (kLossThreads / lanes));
  return n < 1 ? 1 : (n > 256 ? 256 : n);
}

template <int G, int S>
struct LaunchBalance {
  static void run(const Balance& b, int groups, hipStream_t s) {
    hipLaunchKernelGGL((balance_kernel<G, S>), dim3(groups), dim3(kLossThreads), 0, s, b);
  }
};
template <int G, int S>
struct LaunchRoute {
  static void run(const RouteBackward& b, hipStream_t s) {
    // four tokens a group of lanes from a wavefront for each of the chip's places on
    if ((int64_t)b.T * G >= (int64_t)64 * 8192)
      hipLaunchKernelGGL((route_backward_kernel<G, S, 4>), dim3(ceil_div(b.T, 4 * (kThreads / G))), dim3(kThreads), 0, s, b);
    else
      hipLaunchKernelGGL((route_backward_kernel<G, S, 1>), dim3(ceil_div(b.T, kThreads / G)), dim3(kThreads), 0, s, b);
  }
};

// ---- gradient of the router's product --------------------------------------------------------------------------------------
// d_w_router is the outer product of skinny.hpp over all rows, dx its expansion, with W_r in three bf16 parts: rows [h][part][R] of R
// columns, E rounded up to a multiple of 32 by zeros.
int router_width(int E) { return ceil_div(E, 32) * 32; }

// In one launch: W_r's parts, 2048 values a workgroup, and d_logits' fragments, 32 rows a workgroup (8192 tokens of 3584, 64 experts:
// 5.6 us).
constexpr int kSplitValues = 4;
__global__ __launch_bounds__(kPackThreads) void router_prepare_kernel(const float* __restrict__ w, int64_t n, int E, int R,
                                                                      uint16_t* __restrict__ out, int split_blocks, Pack pack) {
  __shared__ __align__(16) float s_sum[32][kMaxGroups + 4];
  if (blockIdx.x >= (unsigned)split_blocks) return pack_block(pack, blockIdx.x - split_blocks, &s_sum[0][0], kMaxGroups + 4);
#pragma unroll
  for (int k = 0; k < kSplitValues; ++k) {
    const int64_t i = ((int64_t)blockIdx.x * kSplitValues + k) * kPackThreads + threadIdx.x;
    if (i >= n) break;
    const int64_t h = i / R;
    const int e = (int)(i - h * R);
    float v = e < E ? w[h * E + e] : 0.f;
#pragma unroll
    for (int p = 0; p < kParts; ++p) {
      const uint32_t bits = f32_to_bf16_bits(v);
      out[(h * kParts + p) * R + e] = (uint16_t)bits;
      v -= bf16_bits_to_f32(bits);  // exact
    }
  }
}

// Above 64 experts dx's workgroups take W_r's columns in several rounds.  While they are few, one after the other bound by a round's latency,
// they have half the columns and four rounds' loads on their way; else P, which each of them reads, counts (workgroups: us with half the
// columns / with all: 1024 columns, 256 experts 4: 18.8 / 25.1, 32: 21.7 / 28.1, 188: 40.6 / 37.4, 1024: 120 / 107; 2048, 128 experts
// 8: 12.3 / 15.6, 64: 14.4 / 17.3, 376: 34.3 / 35.9, 1024: 61.4 / 57.6).
constexpr int kFewF32 = 128;

struct RouterPlan {
  int chunk, pieces, slots, tiles;
  size_t split, packed, outer, partial, bytes;  // offsets in the workspace
};
RouterPlan plan_router(int T, int H, int E) {
  RouterPlan p = {};
  p.chunk = outer_chunk(T, 1, ceil_div(H, kOuterCols), E, 256);
  p.pieces = T > p.chunk ? ceil_div(T, p.chunk) : 1;
  p.slots = T > p.chunk ? p.pieces : 0;
  p.tiles = ceil_div(T, kTileRows);
  p.packed = padded((size_t)H * kParts * router_width(E) * 2);
  p.outer = p.packed + padded(packed_bytes(p.tiles, E));
  p.partial = p.outer + padded(outer_bytes(p.tiles, E));
  p.bytes = p.partial + padded((size_t)p.slots * H * E * sizeof(float));
  return p;
}

// ---- gradient of the combine's gates ---------------------------------------------------------------------------------------
// A workgroup per token: every lane holds 8 columns of dy and meets the token's rows of y one after the other, so dy is read once and
// each row of y once, 16 or 32 bytes a lane; the k + 1 sums are joined at the end.  Bound by y's bytes: 4096 tokens of 4096, 2 fp32 rows
// each, 31.2 us (5.4 TB/s).
template <typename YT, int KMAX>
__global__ __launch_bounds__(kThreads) void combine_backward_kernel(const uint16_t* __restrict__ dy, const YT* __restrict__ y_perm,
                                                                    const int32_t* __restrict__ slot_row, int k, int H,
                                                                    const YT* __restrict__ y_shared,
                                                                    const uint16_t* __restrict__ x,
                                                                    const float* __restrict__ w_shared_gate,
                                                                    float* __restrict__ d_topk_w,
                                                                    float* __restrict__ d_shared_gate) {
  __shared__ float red[kWaves][KMAX + 2];
  const int t = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  float acc[KMAX], shared = 0.f, z = 0.f;
  int row[KMAX];
#pragma unroll
  for (int j = 0; j < KMAX; ++j) {
    acc[j] = 0.f;
    row[j] = j < k ? slot_row[(size_t)t * k + j] : -1;
  }
  for (int h = tid * 8; h < H; h += kThreads * 8) {
    float g[8], v[8];
    load8(dy + (size_t)t * H + h, g);
#pragma unroll
    for (int j = 0; j < KMAX; ++j)
      if (row[j] >= 0) {
        load8(y_perm + (size_t)row[j] * H + h, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[j] = fmaf(g[i], v[i], acc[j]);
      }
    if (y_shared != nullptr) {
      load8(y_shared + (size_t)t * H + h, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) shared = fmaf(g[i], v[i], shared);
      float w[8];
      load8(x + (size_t)t * H + h, v);
      load8(w_shared_gate + h, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) z = fmaf(v[i], w[i], z);
    }
  }
#pragma unroll
  for (int j = 0; j < KMAX; ++j) {
    const float sum = wave_sum(acc[j]);
    if (lane == 0) red[wave][j] = sum;
  }
  if (y_shared != nullptr) {
    shared = wave_sum(shared);
    z = wave_sum(z);
    if (lane == 0) red[wave][KMAX] = shared, red[wave][KMAX + 1] = z;
  }
  __syncthreads();
  if (tid < k) {
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) sum += red[w][tid];
    d_topk_w[(size_t)t * k + tid] = sum;
  }
  if (tid == 64 && y_shared != nullptr) {
    float sum = 0.f, logit = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) sum += red[w][KMAX], logit += red[w][KMAX + 1];
    const float e = expf(-fabsf(logit));  // gate (1 - gate) without a difference: both ends keep their digits
    d_shared_gate[t] = e / ((1.f + e) * (1.f + e)) * sum;
  }
}

template <typename YT>
void launch_combine_backward(const uint16_t* dy, const void* y_perm, const int32_t* slot_row, int T, int k, int H,
                             const void* y_shared, const uint16_t* x, const float* w, float* d_topk_w, float* d_gate,
                             hipStream_t s) {
  const auto kernel = k <= 1   ? combine_backward_kernel<YT, 1>
                      : k <= 2 ? combine_backward_kernel<YT, 2>
                      : k <= 4 ? combine_backward_kernel<YT, 4>
                      : k <= 8 ? combine_backward_kernel<YT, 8>
                               : combine_backward_kernel<YT, 16>;
  hipLaunchKernelGGL(kernel, dim3(T), dim3(kThreads), 0, s, dy, static_cast<const YT*>(y_perm), slot_row, k, H,
                     static_cast<const YT*>(y_shared), x, w, d_topk_w, d_gate);
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int losses_status(int32_t T, int32_t E, int32_t k) {
  if (T < 0 || E < 1 || E > MOE_MAX_EXPERTS || k < 1 || k > E || k > MOE_MAX_TOPK || (int64_t)T * k >= (1 << 24))
    return MOE_ERR_INVALID_ARG;
  return MOE_OK;
}

int router_status(int32_t T, int32_t H, int32_t E) {
  if (T < 0 || T >= (1 << 24) || E < 1 || E > MOE_MAX_EXPERTS || H < 8 || H > MOE_ROUTER_GRAD_MAX_HIDDEN) return MOE_ERR_INVALID_ARG;
  return H % 8 != 0 ? MOE_ERR_UNSUPPORTED_SHAPE : MOE_OK;
}

}  // namespace
}  // namespace moe

extern "C" {

size_t moe_balance_workspace_bytes(int32_t T, int32_t E) {
  using namespace moe;
  if (losses_status(T, E, 1) != MOE_OK) return 0;
  return 2 * padded((size_t)loss_workgroups(T, E) * (E + 1) * 4);
}

int moe_balance_loss(const float* logits, const int32_t* topk_idx, const uint8_t* token_mask, int32_t T, int32_t E, int32_t k,
                     int32_t* counts, float* mean_prob, float* losses, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace moe;
  const int st = losses_status(T, E, k);
  if (st != MOE_OK) return st;
  if (T > 0 && (logits == nullptr || topk_idx == nullptr)) return MOE_ERR_INVALID_ARG;
  if (counts == nullptr || mean_prob == nullptr || losses == nullptr) return MOE_ERR_INVALID_ARG;
  if (workspace == nullptr || !aligned16(workspace) || workspace_bytes < moe_balance_workspace_bytes(T, E)) return MOE_ERR_WORKSPACE;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const int groups = loss_workgroups(T, E);
  const Balance b{logits, topk_idx, token_mask, T, E, k, counts, mean_prob, losses, static_cast<float*>(workspace),
                  reinterpret_cast<int32_t*>(static_cast<char*>(workspace) + padded((size_t)groups * (E + 1) * 4))};
  by_width<LaunchBalance>(E, b, groups, s);
  if (groups > 1) hipLaunchKernelGGL(balance_join_kernel, dim3(1), dim3(kLossThreads), 0, s, b, groups);
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
  const RouteBackward b{logits, d_topk_w, topk_idx, counts, token_mask, T, E, k, coef_balance, coef_z,
                        (flags & MOE_RENORM_TOPK) != 0, d_logits};
  by_width<LaunchRoute>(E, b, static_cast<hipStream_t>(stream));
  return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

size_t moe_router_backward_workspace_bytes(int32_t T, int32_t H, int32_t E) {
  return moe::router_status(T, H, E) == MOE_OK ? moe::plan_router(T, H, E).bytes : 0;
}

int moe_router_backward(const void* x_bf16, const float* w_router, const float* d_logits, int32_t T, int32_t H, int32_t E,
                        const void* dx_in, void* dx, float* d_w_router, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace moe;
  const int st = router_status(T, H, E);
  if (st != MOE_OK) return st;
  if (T > 0 && (x_bf16 == nullptr || d_logits == nullptr)) return MOE_ERR_INVALID_ARG;
  if (d_w_router == nullptr || (dx == nullptr ? dx_in != nullptr : w_router == nullptr)) return MOE_ERR_INVALID_ARG;
  if (!aligned16(x_bf16) || !aligned16(dx_in) || !aligned16(dx) || !aligned16(d_w_router)) return MOE_ERR_INVALID_ARG;
  if (workspace == nullptr || !aligned16(workspace) || workspace_bytes < moe_router_backward_workspace_bytes(T, H, E))
    return MOE_ERR_WORKSPACE;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const RouterPlan p = plan_router(T, H, E);
  char* const ws = static_cast<char*>(workspace);
  const int R = router_width(E);
  uint16_t* const split = reinterpret_cast<uint16_t*>(ws + p.split);
  u32x4 *const packed = reinterpret_cast<u32x4*>(ws + p.packed), *const outer = reinterpret_cast<u32x4*>(ws + p.outer);
  if (T > 0) {
    const int split_blocks = dx != nullptr ? ceil_div((int64_t)H * R, kSplitValues * kPackThreads) : 0;
    hipLaunchKernelGGL(router_prepare_kernel, dim3(split_blocks + 2 * p.tiles), dim3(kPackThreads), 0, s, w_router, (int64_t)H * R, E, R, split,
                       split_blocks,
                       Pack{nullptr, nullptr, T, 1, d_logits, 1, E, E % 4 == 0 && aligned16(d_logits), nullptr, nullptr,
                            dx != nullptr ? packed : nullptr, outer});
  }
  const Outer o{nullptr, nullptr, nullptr, nullptr, nullptr, T, 1,
                {{static_cast<const uint16_t*>(x_bf16), outer, nullptr, d_w_router, reinterpret_cast<float*>(ws + p.partial), H,
                  ceil_div(H, kOuterCols), true},
                 {}},
                E, p.chunk};
  if (dx != nullptr && T > 0) {
    const ExpandF32 e{T, packed, E, split, H, static_cast<const uint16_t*>(dx_in), static_cast<uint16_t*>(dx)};
    if (E <= 16) launch_both<1, ExpandByF32<4, 1, false>>(o, p.pieces, e, p.tiles, s);
    else if (E <= 32) launch_both<2, ExpandByF32<4, 1, false>>(o, p.pieces, e, p.tiles, s);
    else if (E <= 64) launch_both<4, ExpandByF32<4, 2, false>>(o, p.pieces, e, p.tiles, s);
    else if (p.tiles * ceil_div(H, ExpandByF32<4, 1, true>::kCols) <= kFewF32) launch_both<4, ExpandByF32<2, 4, true>>(o, p.pieces, e, p.tiles, s);
    else launch_both<4, ExpandByF32<4, 1, true>>(o, p.pieces, e, p.tiles, s);
  } else {
    launch_outer(o, p.pieces, s);
  }
  if (p.slots > 0) launch_reduce(o, s);
  return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

int moe_combine_backward(const void* dy_bf16, const void* y_perm, const int32_t* slot_row, int32_t T, int32_t k, int32_t H,
                         const void* y_shared, const void* x_bf16, const float* w_shared_gate, float* d_topk_w,
                         float* d_shared_gate, uint32_t flags, void* stream) {
  using namespace moe;
  if (T < 0 || T >= (1 << 24) || k < 1 || k > MOE_MAX_TOPK || H < 8 || H > MOE_ROUTER_GRAD_MAX_HIDDEN) return MOE_ERR_INVALID_ARG;
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
    launch_combine_backward<uint16_t>(dy, y_perm, slot_row, T, k, H, y_shared, x, w_shared_gate, d_topk_w, d_shared_gate, s);
  else
    launch_combine_backward<float>(dy, y_perm, slot_row, T, k, H, y_shared, x, w_shared_gate, d_topk_w, d_shared_gate, s);
  return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

}  // extern "C"
