// Low-rank adapters of many requests beside one projection: y += scale_a (x A_a^T) B_a^T with the row's own adapter a, and the
// gradients of A, B and x.
//
// Rows are first sorted by adapter (moe_permute's index kernels; not up to 64 rows, where a wavefront sees all ids at once), then
//   forward:  v = shrink(x, A), y = expand(v, B)
//   backward: u = shrink(dy, B^T), dx = expand(u, A^T), grad A = outer(u, x), grad B = outer(v, dy)
// with the kernels of skinny.hpp.  B^T and A^T are written out first: a few MB, where the products read them 16 bytes at a time along the
// side that is summed.
#include "moe_lora.h"
#include "skinny.hpp"

namespace moe {
namespace {

using namespace skinny;

// out[c][r] = in[r][c] for each adapter that has rows; A in the first tiles_a tiles of 64 x 64, B behind them.
struct Transpose {
  const uint16_t* in[2];
  uint16_t* out[2];
  int R[2], C[2], tiles_c[2], tiles_a;
  const int32_t* offsets;
};
__global__ __launch_bounds__(256) void transpose_kernel(Transpose p) {
  __shared__ uint16_t s[64][66];
  const int g = blockIdx.y;
  if (p.offsets[g] == p.offsets[g + 1]) return;
  const int side = blockIdx.x >= (unsigned)p.tiles_a, b = side ? blockIdx.x - p.tiles_a : blockIdx.x;
  const int R = p.R[side], C = p.C[side], r0 = b / p.tiles_c[side] * 64, c0 = b % p.tiles_c[side] * 64;
  const uint16_t* in = p.in[side] + (size_t)g * R * C;
  uint16_t* out = p.out[side] + (size_t)g * R * C;
  const int i = threadIdx.x >> 3, j = (threadIdx.x & 7) * 8;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int r = r0 + i + 32 * h, c = c0 + j;
    if (r < R && c < C) {
      const uint4 v = *reinterpret_cast<const uint4*>(in + (size_t)r * C + c);
#pragma unroll
      for (int k = 0; k < 8; ++k) s[i + 32 * h][j + k] = (uint16_t)(reinterpret_cast<const uint32_t*>(&v)[k / 2] >> (16 * (k & 1)));
    }
  }
  __syncthreads();
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int c = c0 + i + 32 * h, r = r0 + j;
    if (c < C && r < R) {
      uint32_t v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = s[j + 2 * k][i + 32 * h] | (uint32_t)s[j + 2 * k + 1][i + 32 * h] << 16;
      *reinterpret_cast<uint4*>(out + (size_t)c * R + r) = make_uint4(v[0], v[1], v[2], v[3]);
    }
  }
}

constexpr int kUnsorted = 64;  // up to this many rows are not sorted

int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }
size_t padded(size_t bytes) { return (bytes + 255) / 256 * 256; }

// Tiles of M rows that T rows in at most L groups can have.
int max_tiles(int T, int L, int M) { return T / M + (L < T ? L : T); }

// How a call is cut: a function of its sizes.
struct Plan {
  bool sorted;
  int shrink_rows, tiles, slices;  // rows per tile of the shrink, workgroups, pieces of its sum
  // backward
  int chunk, pieces, slots;        // rows per piece of the outer products, pieces, partial results of cut groups
};

Plan plan_shrink(int T, int K, int L, bool sorted) {
  Plan p = {};
  p.sorted = sorted;
  p.shrink_rows = T <= 16 && !sorted ? 16 : (T <= 32 || sorted ? 32 : 64);
  p.tiles = sorted ? max_tiles(T, L, p.shrink_rows) : T;
  // a piece of 64 k for each of the eight wavefronts at least; about two workgroups a compute unit
  const int most = ceil_div(K, 64 * kShrinkWaves), want = ceil_div(512, p.tiles > 0 ? p.tiles : 1);
  p.slices = most < want ? most : want;
  if (p.slices > 16) p.slices = 16;
  if (p.slices < 1) p.slices = 1;
  return p;
}

Plan plan_backward(int T, int K, int N, int rank, int L) {
  Plan p = plan_shrink(T, N, L, true);
  // about 512 workgroups if the rows were one group's; pieces of 256 rows at least
  const int64_t per_row = (int64_t)(ceil_div(K, kOuterCols) + ceil_div(N, kOuterCols)) * ceil_div(rank, 64);
  int64_t chunk = (T * per_row / 256 + 255) / 256 * 256;
  p.chunk = (int)(chunk < 256 ? 256 : (chunk > 8192 ? 8192 : chunk));
  p.pieces = T / p.chunk + L;
  p.slots = T > p.chunk ? 2 * (T / p.chunk) : 0;
  return p;
}

// The workspace, in order.
struct Space {
  size_t offsets, list, slot, sort, part, u, at, bt, outer, bytes;
};
Space layout(int T, int K, int N, int rank, int L, bool backward, const Plan& p) {
  Space s = {};
  size_t at = 0;
  const auto take = [&at](size_t bytes) {
    const size_t here = at;
    at += padded(bytes);
    return here;
  };
  if (p.sorted) {
    s.offsets = take((L + 1) * sizeof(int32_t));
    s.list = take((size_t)T * sizeof(int32_t));
    s.slot = take((size_t)T * sizeof(int32_t));
    s.sort = take(permute_workspace_bytes(T, 1, L));
  }
  s.part = take((size_t)p.slices * T * rank * sizeof(float));
  if (backward) {
    s.u = take((size_t)T * rank * sizeof(float));
    s.at = take((size_t)L * K * rank * 2);
    s.bt = take((size_t)L * N * rank * 2);
    s.outer = take((size_t)p.slots * rank * ((size_t)K + N) * sizeof(float));
  }
  s.bytes = at > 0 ? at : 256;
  return s;
}

Plan plan_forward(int T, int K, int L) { return plan_shrink(T, K, L, T > kUnsorted); }

hipError_t sort_rows(const int32_t* idx, int T, int L, char* ws, const Space& sp, Rows* rows, hipStream_t s) {
  int32_t* offsets = reinterpret_cast<int32_t*>(ws + sp.offsets);
  int32_t* list = reinterpret_cast<int32_t*>(ws + sp.list);
  *rows = Rows{offsets, list, idx, T, L};
  return launch_permute(nullptr, idx, T, 1, 8, L, 0, nullptr, offsets, list, reinterpret_cast<int32_t*>(ws + sp.slot), ws + sp.sort,
                        s);
}

template <int MT, int U>
void launch_shrink_rows(const Rows& rows, const Plan& p, const uint16_t* x, int K, const uint16_t* m, int rank, float* part,
                        hipStream_t s) {
  const dim3 grid(p.tiles, p.slices), block(kShrinkWaves * 64);
  if (rank <= 16) hipLaunchKernelGGL((shrink_kernel<MT, 1, U>), grid, block, 0, s, rows, x, K, m, rank, part);
  else if (rank <= 32) hipLaunchKernelGGL((shrink_kernel<MT, 2, U>), grid, block, 0, s, rows, x, K, m, rank, part);
  else if (rank <= 64) hipLaunchKernelGGL((shrink_kernel<MT, 4, 1>), grid, block, 0, s, rows, x, K, m, rank, part);
  else hipLaunchKernelGGL((shrink_kernel<MT, 8, 1>), grid, block, 0, s, rows, x, K, m, rank, part);
}

void launch_shrink(Rows rows, const Plan& p, const uint16_t* x, int K, const uint16_t* m, int rank, float* part, hipStream_t s) {
  if (p.sorted) rows.idx = nullptr;
  if (p.shrink_rows == 16) launch_shrink_rows<1, 2>(rows, p, x, K, m, rank, part, s);
  else if (p.shrink_rows == 32) launch_shrink_rows<2, 2>(rows, p, x, K, m, rank, part, s);
  else launch_shrink_rows<4, 1>(rows, p, x, K, m, rank, part, s);
}

template <typename YT, int SPLIT, int WCH>
void launch_expand_width(Expand e, hipStream_t s) {
  constexpr int M = SPLIT * 32 * WCH <= 256 ? 128 : 64;  // as in the kernel
  const int T = e.rows.T;
  const bool sorted = e.rows.offsets != nullptr;
  e.n_tiles = sorted ? max_tiles(T, e.rows.L, M) : T;
  const bool bare = sorted && (e.keep != nullptr || (e.y_out != nullptr && e.y_out != e.y_in));
  const dim3 grid(e.y_out != nullptr ? ceil_div(e.N, kExpandWaves * 64) : 1, e.n_tiles + (bare ? ceil_div(T, 64) : 0));
  hipLaunchKernelGGL((expand_kernel<YT, SPLIT, WCH, 4, false>), grid, dim3(kExpandThreads), 0, s, e);
}

template <typename YT, int SPLIT>
void launch_expand(const Expand& e, hipStream_t s) {
  if (e.r <= 32) launch_expand_width<YT, SPLIT, 1>(e, s);
  else if (e.r <= 64) launch_expand_width<YT, SPLIT, 2>(e, s);
  else launch_expand_width<YT, SPLIT, 4>(e, s);
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int size_status(int32_t T, int32_t K, int32_t N, int32_t rank, int32_t L) {
  if (T < 0 || T >= (1 << 24) || K < 8 || N < 8 || rank < 1 || L < 1 || L > MOE_LORA_MAX_ADAPTERS) return MOE_ERR_INVALID_ARG;
  if (K % 8 != 0 || N % 8 != 0 || rank % 8 != 0 || rank > MOE_LORA_MAX_RANK) return MOE_ERR_UNSUPPORTED_SHAPE;
  return MOE_OK;
}

}  // namespace
}  // namespace moe

extern "C" {

size_t moe_lora_workspace_bytes(int32_t T, int32_t K, int32_t N, int32_t rank, int32_t n_adapters, int32_t backward) {
  if (moe::size_status(T, K, N, rank, n_adapters) != MOE_OK) return 0;
  using namespace moe;
  const Plan p = backward ? plan_backward(T, K, N, rank, n_adapters) : plan_forward(T, K, n_adapters);
  return layout(T, K, N, rank, n_adapters, backward != 0, p).bytes;
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
  const Plan p = plan_forward(T, K, n_adapters);
  const Space sp = layout(T, K, N, rank, n_adapters, false, p);
  char* const ws = static_cast<char*>(workspace);
  Rows rows{nullptr, nullptr, adapter_idx, T, n_adapters};
  if (p.sorted && sort_rows(adapter_idx, T, n_adapters, ws, sp, &rows, s) != hipSuccess) return MOE_ERR_HIP;
  float* const part = reinterpret_cast<float*>(ws + sp.part);
  launch_shrink(rows, p, static_cast<const uint16_t*>(x_bf16), K, static_cast<const uint16_t*>(lora_a), rank, part, s);
  const Expand e{rows, part, p.slices, rank, scale, v, false, static_cast<const uint16_t*>(lora_b), rank, N, y_in, y_out, 0, true};
  if (flags & MOE_OUT_F32) launch_expand<float, 3>(e, s);
  else launch_expand<uint16_t, 2>(e, s);
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
  const Plan p = plan_backward(T, K, N, rank, n_adapters);
  const Space sp = layout(T, K, N, rank, n_adapters, true, p);
  char* const ws = static_cast<char*>(workspace);
  Rows rows;
  if (sort_rows(adapter_idx, T, n_adapters, ws, sp, &rows, s) != hipSuccess) return MOE_ERR_HIP;
  float *const part = reinterpret_cast<float*>(ws + sp.part), *const u = reinterpret_cast<float*>(ws + sp.u);
  uint16_t *const at = reinterpret_cast<uint16_t*>(ws + sp.at), *const bt = reinterpret_cast<uint16_t*>(ws + sp.bt);
  if (T > 0) {
    const int ra = ceil_div(rank, 64), ca = ceil_div(K, 64), cb = ceil_div(N, 64);
    const Transpose tr{{static_cast<const uint16_t*>(lora_a), static_cast<const uint16_t*>(lora_b)}, {at, bt}, {rank, N}, {K, rank},
                       {ca, ra}, ra * ca, rows.offsets};
    hipLaunchKernelGGL(transpose_kernel, dim3(ra * (ca + cb), n_adapters), dim3(256), 0, s, tr);
    launch_shrink(rows, p, dy, N, bt, rank, part, s);
    const Expand e{rows, part, p.slices, rank, scale, u, true, at, rank, K, dx_in, dx, 0, true};
    launch_expand<uint16_t, 2>(e, s);
  }
  float* const cut = reinterpret_cast<float*>(ws + sp.outer);
  const Outer o{{rows.offsets, rows.list, nullptr, T, n_adapters},
                {{x, u, nullptr, grad_a, cut, K, ceil_div(K, kOuterCols), false},
                 {dy, v, scale, grad_b, cut + (size_t)p.slots * rank * K, N, ceil_div(N, kOuterCols), true}},
                rank, p.chunk};
  const dim3 block(kOuterWaves * 64);
  const int tiles = o.side[0].tiles + o.side[1].tiles;
  if (rank <= 16) hipLaunchKernelGGL(outer_kernel<1>, dim3(tiles, p.pieces, 1), block, 0, s, o);
  else if (rank <= 32) hipLaunchKernelGGL(outer_kernel<2>, dim3(tiles, p.pieces, 1), block, 0, s, o);
  else hipLaunchKernelGGL(outer_kernel<4>, dim3(tiles, p.pieces, ceil_div(rank, 64)), block, 0, s, o);
  if (p.slots > 0) hipLaunchKernelGGL(reduce_kernel, dim3(ceil_div((int64_t)rank * (K > N ? K : N), 4096), n_adapters), dim3(256), 0, s, o);
  return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

}  // extern "C"
