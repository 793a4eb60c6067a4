// Low-rank adapters of many requests beside one projection: y += scale_a (x A_a^T) B_a^T with the row's own adapter a, and the
// gradients of A, B and x.
//
// A decoding batch of up to 64 rows: fused_few_kernel, or shrink_few_kernel and expand_few_kernel.  More rows are sorted by adapter first
// (skinny.hpp), a launch for each product:
//   forward:  v = shrink(x, A), y = expand(v, B)
//   backward: u = shrink(dy, B^T), then dx = expand(u, A^T), grad A = outer(u, x) and grad B = outer(v, dy) in one launch
// B^T and A^T are written out for that: a few MB, where the products read them 16 bytes at a time along the side that is summed.
#include "moe_lora.h"
#include "skinny.hpp"

namespace moe {
namespace {

using namespace skinny;

// ---- up to 64 rows -------------------------------------------------------------------------------------------------------------
// A short kernel or two, bound by their latency: every workgroup looks at all ids, one a lane.  With two, the adapters' matrices are read
// straight into the MFMA's operands (48 rows of 32 adapters, 4096 x 4096, rank 16: 4.2 and 5.1 us; through LDS, as for many rows, 7.5 and
// 7.2 where they had taken 5.7 and 5.0).
constexpr int kFewRows = 64, kFewTile = 16;

struct Few {
  const int32_t* idx;
  int T, L;
};

// Sixteen rows of one adapter, or fewer, are a tile; its number follows from the first row of its adapter, which stands for them all.
int few_tiles(int T, int L) {
  const int groups = T < L + 1 ? T : L + 1;
  return groups + (T - groups) / kFewTile;
}

// Rows of tile b: fills s_rows, returns how many, 0 past the last one; group -1: without an adapter.
__device__ __forceinline__ int few_rows(const Few& f, int b, int32_t* s_rows, int& group) {
  const int lane = threadIdx.x & (kWave - 1);
  const bool in = lane < f.T;
  int g = in ? f.idx[lane] : -1;
  if ((unsigned)g >= (unsigned)f.L) g = -1;
  const unsigned long long same = match_lanes(g + 1, in, 32 - __clz(f.L));
  const int all = (int)__popcll(same), rank = (int)__popcll(same & ((1ull << lane) - 1ull));
  const int tiles = in && rank == 0 ? (all + kFewTile - 1) / kFewTile : 0;
  int end = tiles;  // tiles up to this lane's
#pragma unroll
  for (int d = 1; d <= kFewRows / kFewTile; ++d) end += (int)__popcll(__ballot(tiles >= d) & ((1ull << lane) - 1ull));
  const unsigned long long owner = __ballot(b >= end - tiles && b < end);
  if (owner == 0) return 0;
  const int src = __ffsll((long long)owner) - 1;
  group = (int)__builtin_amdgcn_readlane(g, src);
  const int first = (b - (int)__builtin_amdgcn_readlane(end - tiles, src)) * kFewTile;
  const int n = min((int)__builtin_amdgcn_readlane(all, src) - first, kFewTile);
  if (threadIdx.x < kWave && in && g == group && rank >= first && rank < first + kFewTile) s_rows[rank - first] = lane;
  return n;
}

constexpr int kFewWaves = 8;

// blockIdx.y: a piece of the sum over k; part [pieces][T][r].  A wavefront multiplies the rows by all of A_a over every
// (8 gridDim.y)-th 64 of k; lane (row, q) loads k = 16 q .. 16 q + 15 of them and so does the lane of A_a, whose halves the two MFMAs take.
template <int NT>
__global__ __launch_bounds__(kFewWaves * 64) void shrink_few_kernel(Few few, const uint16_t* __restrict__ x, int K,
                                                                    const uint16_t* __restrict__ m, int r, float* __restrict__ part) {
  __shared__ int32_t s_rows[kFewTile];
  __shared__ float red[kFewWaves][16][NT * 16 + 1];
  int group;
  const int n = few_rows(few, blockIdx.x, s_rows, group);
  if (n == 0 || group < 0) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, row = lane & 15, q = lane >> 4;
  const uint16_t* mr[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) mr[j] = m + ((size_t)group * r + min(16 * j + row, r - 1)) * K + 16 * q;
  __syncthreads();
  const uint16_t* const xr = x + (size_t)s_rows[min(row, n - 1)] * K + 16 * q;
  f32x4 acc[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int stride = kFewWaves * gridDim.y * 64;
  for (int c = (blockIdx.y * kFewWaves + wave) * 64; c < K; c += stride) {
    u32x4 xv[2], mv[NT][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const bool in = c + 8 * h + 16 * q < K;  // (K is a multiple of 8)
#pragma unroll
      for (int j = 0; j < NT; ++j) mv[j][h] = in ? *reinterpret_cast<const u32x4*>(mr[j] + c + 8 * h) : u32x4{};
      xv[h] = in ? *reinterpret_cast<const u32x4*>(xr + c + 8 * h) : u32x4{};
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int j = 0; j < NT; ++j) acc[j] = mfma(xv[h], mv[j][h], acc[j]);
  }
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) red[wave][4 * q + e][16 * j + row] = acc[j][e];
  __syncthreads();
  part += (size_t)blockIdx.y * few.T * r;
  for (int o = tid; o < 16 * 16 * NT; o += kFewWaves * 64) {
    const int ro = o / (16 * NT), col = o % (16 * NT);
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) sum += red[w][ro][col];
    if (ro < n && col < r) part[(size_t)s_rows[ro] * r + col] = sum;
  }
}

// A wavefront computes 64 columns: lane (c, q) holds four neighbouring ones of row c for each accumulator, dealt so that 16 bytes of a row
// are one lane's.  The pieces of v's sum are added in order, its parts go through LDS (rows 16 bytes longer than a multiple of 32).
struct ExpandFew {
  Few few;
  const float* part;
  int pieces, r;
  const float* scale;
  float* keep;
  const uint16_t* m;
  int N;
  const void* y_in;
  void* y_out;
};

// The wavefront's columns from its fragments of M_a, v's parts in LDS and y.
template <typename YT, int CH>
__device__ __forceinline__ void few_out(const u32x4 (&w)[CH][4], u32x4 (&y)[sizeof(YT)], const char* s_p, int n, int nbase, size_t at,
                                        const ExpandFew& e) {
  constexpr int R = 32 * CH, W = 16 / sizeof(YT), UNITS = 64 / (4 * W), kRowBytes = kParts * R * 2 + 16;
  const int lane = threadIdx.x & 63, ln = lane & 15, q = lane >> 4, c0 = nbase + q * W;
  YT* const out = static_cast<YT*>(e.y_out);
  f32x4 acc[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int s = kParts - 1; s >= 0; --s) {  // the small parts first
      const u32x4 b = *reinterpret_cast<const u32x4*>(s_p + ln * kRowBytes + s * R * 2 + c * 64 + q * 16);
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[j] = mfma(w[c][j], b, acc[j]);
    }
  if (ln >= n) return;
#pragma unroll
  for (int h = 0; h < UNITS; ++h) {
    if (c0 + h * 4 * W >= e.N) break;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t d = y[h][i];
      if constexpr (W == 8) {
        const f32x4 a = acc[2 * h + i / 2];
        y[h][i] = pack_bf16x2(bf16_lo(d) + a[2 * (i & 1)], bf16_hi(d) + a[2 * (i & 1) + 1]);
      } else {
        y[h][i] = __float_as_uint(__uint_as_float(d) + acc[h][i]);
      }
    }
    *reinterpret_cast<u32x4*>(out + at + h * 4 * W) = y[h];
  }
}

template <typename YT, int CH>
__global__ __launch_bounds__(kExpandThreads) void expand_few_kernel(ExpandFew e) {
  constexpr int R = 32 * CH, W = 16 / sizeof(YT), UNITS = 64 / (4 * W), kRowBytes = kParts * R * 2 + 16, ITEMS = kFewTile * (R / 8);
  __shared__ int32_t s_rows[kFewTile];
  __shared__ __align__(16) char s_p[kFewTile * kRowBytes];
  static_assert(ITEMS <= kExpandThreads, "a thread has eight values of v at most");
  int group;
  const int n = few_rows(e.few, blockIdx.y, s_rows, group);
  if (n == 0) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, ln = lane & 15, q = lane >> 4, r = e.r;
  const int nbase = (blockIdx.x * kExpandWaves + wave) * 64;
  u32x4 w[CH][4];
  if (group >= 0 && nbase < e.N)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int col = W == 8 ? (j >> 1) * 32 + (ln >> 2) * 8 + (j & 1) * 4 + (ln & 3) : 16 * j + ln;
      const uint16_t* const mr = e.m + ((size_t)group * e.N + min(nbase + col, e.N - 1)) * r + 8 * q;
#pragma unroll
      for (int c = 0; c < CH; ++c)
        w[c][j] = 32 * c + 8 * q < r ? *reinterpret_cast<const u32x4*>(mr + 32 * c) : u32x4{};
    }
  __syncthreads();
  if (group < 0) {
    copy_rows<YT>(e.y_in, e.y_out, e.N, s_rows, n, blockIdx.x * kExpandWaves * 64, kExpandWaves * 64);
    if (e.keep != nullptr && blockIdx.x == 0)
      for (int i = tid; i < n * r; i += kExpandThreads) e.keep[(size_t)s_rows[i / r] * r + i % r] = 0.f;
    return;
  }
  const YT* in = static_cast<const YT*>(e.y_in);
  const int c0 = nbase + q * W;
  const size_t at = (size_t)s_rows[min(ln, n - 1)] * e.N + c0;
  u32x4 y[UNITS];
#pragma unroll
  for (int h = 0; h < UNITS; ++h)
    y[h] = in != nullptr && c0 + h * 4 * W < e.N ? *reinterpret_cast<const u32x4*>(in + at + h * 4 * W) : u32x4{};
  if (tid < ITEMS) {
    const int i = tid / (R / 8), j0 = tid % (R / 8) * 8;
    float v[8] = {};
    if (i < n && j0 < r) {
      const size_t row = (size_t)s_rows[i] * r + j0, piece = (size_t)e.few.T * r;
      for (int s0 = 0; s0 < e.pieces; s0 += 4) {
        float more[4][8];
#pragma unroll
        for (int s = 0; s < 4; ++s)
          if (s0 + s < e.pieces) load8(e.part + (s0 + s) * piece + row, more[s]);
#pragma unroll
        for (int s = 0; s < 4; ++s)
          if (s0 + s < e.pieces)
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] += more[s][k];
      }
      const float scale = e.scale[group];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        if (e.keep != nullptr && blockIdx.x == 0) e.keep[row + k] = v[k];
        v[k] *= scale;
      }
    }
#pragma unroll
    for (int s = 0; s < kParts; ++s) *reinterpret_cast<u32x4*>(s_p + i * kRowBytes + s * R * 2 + j0 * 2) = take_bf16(v);
  }
  __syncthreads();
  few_out<YT, CH>(w, y, s_p, n, nbase, at, e);
}

// Both products in one launch: each workgroup computes v for its 512 columns (or 1024) anew.  The wavefronts take an eighth of k each, all
// of it on its way at once, 128 bytes of a row by eight neighbouring lanes and through LDS into the MFMA's operands: read as operands, 16 bytes
// from each of 16 rows, an instruction would take 64 clocks.  Two launches / one, us, in a graph and one by one from the host: 8 rows of 8
// adapters, 4096 x 4096, rank 16 7.6 / 7.3, 11.4 / 8.3; 2048 x 2048, rank 32, 40 adapters 8.0 / 7.0, 10.9 / 8.3.
constexpr int kFusedWaves = 8, kFusedThreads = kFusedWaves * 64;

template <typename YT, int NT, int FLIGHT, int WIDE>
__global__ __launch_bounds__(kFusedThreads, 2) void fused_few_kernel(ExpandFew e, const uint16_t* __restrict__ x, int K,
                                                                     const uint16_t* __restrict__ m) {
  constexpr int R = 32, W = 16 / sizeof(YT), UNITS = 64 / (4 * W), kRowBytes = kParts * R * 2 + 16, ITEMS = kFewTile * (R / 8);
  constexpr int kStage = (16 + 16 * NT) * 128, kCols = WIDE * kFusedWaves * 64;
  __shared__ int32_t s_rows[kFewTile];
  __shared__ __align__(16) char s_p[kFewTile * kRowBytes];
  __shared__ __align__(16) char s_stage[kFusedWaves * kStage];
  __shared__ float red[kFusedWaves][16][NT * 16 + 1];
  int group;
  const int n = few_rows(e.few, blockIdx.y, s_rows, group);
  if (n == 0) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, ln = lane & 15, q = lane >> 4, sub = lane >> 3, ch = lane & 7;
  const int r = e.r;
  __syncthreads();
  if (group < 0) {
    copy_rows<YT, kFusedThreads>(e.y_in, e.y_out, e.N, s_rows, n, blockIdx.x * kCols, kCols);
    if (e.keep != nullptr && blockIdx.x == 0)
      for (int i = tid; i < n * r; i += kFusedThreads) e.keep[(size_t)s_rows[i / r] * r + i % r] = 0.f;
    return;
  }
  // (loads without conditions: past the end the last piece again, past K the first columns, both taken as zeros)
  const int pieces = (K + 63) / 64, first = pieces * wave / kFusedWaves, count = pieces * (wave + 1) / kFusedWaves - first;
  const uint16_t *xr[2], *mr[2 * NT];
#pragma unroll
  for (int i = 0; i < 2; ++i) xr[i] = x + (size_t)s_rows[min(8 * i + sub, n - 1)] * K + 8 * ch;
#pragma unroll
  for (int i = 0; i < 2 * NT; ++i) mr[i] = m + ((size_t)group * r + min(8 * i + sub, r - 1)) * K + 8 * ch;
  u32x4 xv[FLIGHT][2], mv[FLIGHT][2 * NT];
#pragma unroll
  for (int f = 0; f < FLIGHT; ++f) {
    int c = (first + max(min(f, count - 1), 0)) * 64;
    c = c + 8 * ch < K ? c : -8 * ch;
#pragma unroll
    for (int i = 0; i < 2; ++i) xv[f][i] = *reinterpret_cast<const u32x4*>(xr[i] + c);
#pragma unroll
    for (int i = 0; i < 2 * NT; ++i) mv[f][i] = *reinterpret_cast<const u32x4*>(mr[i] + c);
  }
  // what the second product needs, on its way meanwhile
  const int nbase = blockIdx.x * kCols + wave * 64, c0 = nbase + q * W;  // the next 64 columns of a wavefront: kFusedThreads further
  u32x4 w[WIDE][1][4], y[WIDE][UNITS];
  const size_t at = (size_t)s_rows[min(ln, n - 1)] * e.N + c0;
  {
    const bool some = e.y_in != nullptr;
    const YT* const in = some ? static_cast<const YT*>(e.y_in) + (size_t)s_rows[min(ln, n - 1)] * e.N : reinterpret_cast<const YT*>(e.m);
    const int last = some ? e.N - W : 0;
#pragma unroll
    for (int i = 0; i < WIDE; ++i) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int col = nbase + i * kFusedThreads + (W == 8 ? (j >> 1) * 32 + (ln >> 2) * 8 + (j & 1) * 4 + (ln & 3) : 16 * j + ln);
        w[i][0][j] = *reinterpret_cast<const u32x4*>(e.m + ((size_t)group * e.N + min(col, e.N - 1)) * r + min(8 * q, r - 8));
      }
#pragma unroll
      for (int h = 0; h < UNITS; ++h)
        y[i][h] = *reinterpret_cast<const u32x4*>(in + min(c0 + i * kFusedThreads + h * 4 * W, last));
    }
  }
  const float scale = e.scale[group];
  f32x4 acc[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  char* const s_x = s_stage + wave * kStage;
  char* const s_m = s_x + 2048;
  const int put = sub * 128 + (ch ^ sub) * 16;  // + 1024 for each eight rows
#pragma unroll
  for (int f = 0; f < FLIGHT; ++f) {
    const bool in = f < count && (first + f) * 64 + 8 * ch < K;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const u32x4 v = xv[f][i];
      *reinterpret_cast<u32x4*>(s_x + put + 1024 * i) = u32x4{in ? v.x : 0u, in ? v.y : 0u, in ? v.z : 0u, in ? v.w : 0u};
    }
#pragma unroll
    for (int i = 0; i < 2 * NT; ++i) *reinterpret_cast<u32x4*>(s_m + put + 1024 * i) = mv[f][i];
    wave_fence();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int from = ln * 128 + (((4 * h + q) ^ (ln & 7)) * 16);
      const u32x4 a = *reinterpret_cast<const u32x4*>(s_x + from);
#pragma unroll
      for (int j = 0; j < NT; ++j) acc[j] = mfma(a, *reinterpret_cast<const u32x4*>(s_m + 2048 * j + from), acc[j]);
    }
    wave_fence();
  }
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int k = 0; k < 4; ++k) red[wave][4 * q + k][16 * j + ln] = acc[j][k];
  __syncthreads();
  if (tid < ITEMS) {
    const int i = tid / (R / 8), j0 = tid % (R / 8) * 8;
    float v[8] = {};
    if (i < n && j0 < r) {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
#pragma unroll
        for (int p = 0; p < kFusedWaves; ++p) v[k] += red[p][i][j0 + k];
        if (e.keep != nullptr && blockIdx.x == 0) e.keep[(size_t)s_rows[i] * r + j0 + k] = v[k];
        v[k] *= scale;
      }
    }
#pragma unroll
    for (int p = 0; p < kParts; ++p) *reinterpret_cast<u32x4*>(s_p + i * kRowBytes + p * R * 2 + j0 * 2) = take_bf16(v);
  }
#pragma unroll
  for (int i = 0; i < WIDE; ++i) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (8 * q >= r) w[i][0][j] = u32x4{};
    if (e.y_in == nullptr)
#pragma unroll
      for (int h = 0; h < UNITS; ++h) y[i][h] = u32x4{};
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < WIDE; ++i) few_out<YT, 1>(w[i], y[i], s_p, n, nbase + i * kFusedThreads, at + i * kFusedThreads, e);
}

// Where k comes in one go (else its halves wait for each other: 2 x 256 KB, rank 32, 7.8 / 8.9 us; 2 x 88 KB of K = 5632 7.5 / 8.4), the
// workgroups run side by side and what they read again is little.  Two launches / one, us in a graph, by the bytes of A that one reads:
// 8 MB 7.6 / 7.3, 21 MB (40 rows of 40, 2048 x 4096, rank 32) 8.4 / 7.9, 33 MB and 256 workgroups (64 of 64) 9.3 / 9.8.
constexpr int64_t kFusedBytes = 28 << 20;
// 512 columns a workgroup, or 1024 where that alone keeps to it: narrow is faster where both do (24 rows of 24, 4096 x 4096, rank 8 7.2 / 8.0,
// one row of rank 16 7.1 / 7.7).  48 rows of 32, rank 16 take 8.4 in two launches, 9.9 narrow and 8.6 wide in a graph, 10.7, 9.7 and 8.4
// from the host.  0: two launches.
int fused_wide(int T, int K, int N, int rank, int L) {
  if (rank > 32 || K * ceil_div(rank, 16) > 4096) return 0;
  for (int wide = 1; wide <= 2; ++wide) {
    const int64_t groups = (int64_t)few_tiles(T, L) * ceil_div(N, wide * kFusedThreads);
    if (groups <= 256 && groups * K * rank * 2 <= kFusedBytes) return wide;
  }
  return 0;
}

template <typename YT, int NT, int FLIGHT>
void launch_fused(const ExpandFew& e, const uint16_t* x, int K, const uint16_t* m, int wide, hipStream_t s) {
  const auto kernel = wide == 2 ? fused_few_kernel<YT, NT, FLIGHT, 2> : fused_few_kernel<YT, NT, FLIGHT, 1>;
  hipLaunchKernelGGL(kernel, dim3(ceil_div(e.N, wide * kFusedThreads), few_tiles(e.few.T, e.few.L)), dim3(kFusedThreads), 0, s, e, x, K, m);
}
template <typename YT>
void launch_fused_few(const ExpandFew& e, const uint16_t* x, int K, const uint16_t* m, int wide, hipStream_t s) {
  if (e.r > 16) launch_fused<YT, 2, 4>(e, x, K, m, wide, s);
  else if (K <= 64 * kFusedWaves * 4) launch_fused<YT, 1, 4>(e, x, K, m, wide, s);
  else launch_fused<YT, 1, 8>(e, x, K, m, wide, s);
}

// Pieces of the sum over k: 64 of k for each of the eight wavefronts, 16 at most.
int few_pieces(int K) {
  const int n = ceil_div(K, 64 * kFewWaves);
  return n > 16 ? 16 : n;
}

void launch_shrink_few(const Few& few, const uint16_t* x, int K, const uint16_t* m, int r, float* part, hipStream_t s) {
  const dim3 grid(few_tiles(few.T, few.L), few_pieces(K)), block(kFewWaves * 64);
  if (r <= 16) hipLaunchKernelGGL(shrink_few_kernel<1>, grid, block, 0, s, few, x, K, m, r, part);
  else if (r <= 32) hipLaunchKernelGGL(shrink_few_kernel<2>, grid, block, 0, s, few, x, K, m, r, part);
  else if (r <= 64) hipLaunchKernelGGL(shrink_few_kernel<4>, grid, block, 0, s, few, x, K, m, r, part);
  else hipLaunchKernelGGL(shrink_few_kernel<8>, grid, block, 0, s, few, x, K, m, r, part);
}

template <typename YT>
void launch_expand_few(const ExpandFew& e, hipStream_t s) {
  const dim3 grid(ceil_div(e.N, kExpandWaves * 64), few_tiles(e.few.T, e.few.L)), block(kExpandThreads);
  if (e.r <= 32) hipLaunchKernelGGL((expand_few_kernel<YT, 1>), grid, block, 0, s, e);
  else if (e.r <= 64) hipLaunchKernelGGL((expand_few_kernel<YT, 2>), grid, block, 0, s, e);
  else hipLaunchKernelGGL((expand_few_kernel<YT, 4>), grid, block, 0, s, e);
}

// ---- sorted rows ---------------------------------------------------------------------------------------------------------------
// Whether each workgroup that needs v adds its slices itself, which saves a launch, or pack_kernel does it once.  Once / each, us, 4096 x
// 4096: rank 16, 300 rows 16.4 / 13.1, 8192 65.3 / 60.5; rank 64, 300 rows 20.2 / 19.2, 4096 (8 slices) 45.3 / 49.3, 8192 (4) 77.6 / 79.8.
bool from_sums(int T, int rank, int slices) { return rank <= 32 || (rank <= 64 && T * slices <= 24576); }

template <typename YT>
void launch_expand(const Expand& e, int n_tiles, hipStream_t s) {
  if (e.packed == nullptr) {
    if (e.r <= 32) launch_expand_kernel<YT, 1, 8, true>(e, n_tiles, s);
    else launch_expand_kernel<YT, 2, 8, true>(e, n_tiles, s);
  } else {
    if (e.r <= 64) launch_expand_kernel<YT, 2, 8, false>(e, n_tiles, s);
    else launch_expand_kernel<YT, 4, 4, false>(e, n_tiles, s);  // (fewer columns, for the registers)
  }
}

// Before the products of a backward pass: out[c][r] = in[r][c] for A and B of each adapter that has rows, 64 x 64 values by half a workgroup,
// four times that a workgroup.  Up to kSortOnce rows each workgroup looks for its adapter among the ids itself, and so does not wait
// for the sort, which the launch's first workgroup does meanwhile (the whole pass, 4096 x 4096, us: 777 rows of 4 adapters, rank 64 35.0 / 31.6,
// 8192 of 8 119 / 115, 300 of 256, rank 16 144 / 158).
struct Transpose {
  const uint16_t* in[2];
  uint16_t* out[2];
  int R[2], C[2], tiles_c[2], tiles_a, tiles, L;  // A's tiles come first
  const int32_t* offsets;
};
constexpr int kTurnTiles = 4;

__device__ __forceinline__ void transpose_block(const Transpose& p, int block, const int32_t* idx, int T) {
  __shared__ uint16_t s_turn[2][64][66];
  static_assert(kSortThreads == 2 * 64 * 8, "two halves, eight lanes a row");
  const int per = (p.tiles + kTurnTiles - 1) / kTurnTiles, g = block / per, first = block % per * kTurnTiles;
  if (idx == nullptr) {
    if (p.offsets[g] == p.offsets[g + 1]) return;
  } else {
    int id[kSortSteps];
#pragma unroll
    for (int u = 0; u < kSortSteps; ++u) id[u] = idx[min((int)threadIdx.x + u * kSortThreads, T - 1)];
    bool some = false;
#pragma unroll
    for (int u = 0; u < kSortSteps; ++u) some |= id[u] == g;
    if (!__syncthreads_or(some)) return;
  }
  const int half = threadIdx.x >> 9, i = (threadIdx.x & 511) >> 3, j = (threadIdx.x & 7) * 8;
  uint16_t(*const s)[66] = s_turn[half];
#pragma unroll
  for (int n = 0; n < kTurnTiles; n += 2) {
    const int tile = first + n + half;
    const bool in_range = tile < p.tiles, second = tile >= p.tiles_a;
    const int b = second ? tile - p.tiles_a : tile, R = second ? p.R[1] : p.R[0], C = second ? p.C[1] : p.C[0];
    const int tc = second ? p.tiles_c[1] : p.tiles_c[0], r0 = b / tc * 64, c0 = b % tc * 64;
    const uint16_t* in = (second ? p.in[1] : p.in[0]) + (size_t)g * R * C;
    uint16_t* out = (second ? p.out[1] : p.out[0]) + (size_t)g * R * C;
    if (in_range && r0 + i < R && c0 + j < C) {
      const u32x4 v = *reinterpret_cast<const u32x4*>(in + (size_t)(r0 + i) * C + c0 + j);
#pragma unroll
      for (int k = 0; k < 8; ++k) s[i][j + k] = (uint16_t)(v[k / 2] >> (16 * (k & 1)));
    }
    __syncthreads();
    if (in_range && c0 + i < C && r0 + j < R) {
      uint32_t v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = s[j + 2 * k][i] | (uint32_t)s[j + 2 * k + 1][i] << 16;
      *reinterpret_cast<u32x4*>(out + (size_t)(c0 + i) * R + r0 + j) = u32x4{v[0], v[1], v[2], v[3]};
    }
    __syncthreads();
  }
}

__global__ __launch_bounds__(kSortThreads) void sort_and_transpose_kernel(Sort s, Transpose p) {
  if (blockIdx.x == 0) sort_block<true>(s);
  else transpose_block(p, blockIdx.x - 1, s.idx, s.T);
}
__global__ __launch_bounds__(kSortThreads) void transpose_kernel(Transpose p) { transpose_block(p, blockIdx.x, nullptr, 0); }

// The fragments of u and of v, 32 rows a workgroup.
__global__ __launch_bounds__(kPackThreads) void pack_both_kernel(Pack u, Pack v, int blocks) {
  __shared__ __align__(16) PackBuffer s_sum;
  const bool second = blockIdx.x >= (unsigned)blocks;
  pack_block(second ? v : u, blockIdx.x - (second ? blocks : 0), &s_sum[0][0], kPackStride);
}

// How a call is cut, and its workspace in order: a function of its sizes.
struct Plan {
  bool few;
  int n_tiles, slices;
  int chunk, n_pieces, slots;  // backward: rows per piece of the outer products, pieces, partial results of cut groups
  size_t offsets, list, tiles, pieces, piece_slots, slot0, part, packed, at, bt, outer_u, outer_v, partial, bytes;
};

Plan make_plan(int T, int K, int N, int rank, int L, bool backward) {
  Plan p = {};
  size_t at = 0;
  const auto take = [&at](size_t bytes) {
    const size_t here = at;
    at += padded(bytes);
    return here;
  };
  p.few = !backward && T <= kFewRows;
  p.slices = p.few ? few_pieces(K) : (T > 0 ? shrink_slices(T, backward ? N : K) : 1);
  p.part = take((size_t)p.slices * T * rank * sizeof(float));
  if (p.few) {
    p.bytes = at > 0 ? at : 256;
    return p;
  }
  p.n_tiles = max_tiles(T, L + 1);
  p.offsets = take((L + 2) * sizeof(int32_t));
  p.list = take((size_t)T * sizeof(int32_t));
  p.tiles = take(p.n_tiles * sizeof(Tile));
  p.packed = take(backward || !from_sums(T, rank, p.slices) ? packed_bytes(p.n_tiles, rank) : 0);
  if (backward) {
    p.chunk = outer_chunk(T, L, ceil_div(K, kOuterCols) + ceil_div(N, kOuterCols), rank, 512);
    p.n_pieces = T / p.chunk + L;
    p.slots = T > p.chunk ? 2 * (T / p.chunk) : 0;
    p.pieces = take(p.n_pieces * sizeof(Tile));
    p.piece_slots = take(p.n_pieces * sizeof(int32_t));
    p.slot0 = take(L * sizeof(int32_t));
    p.at = take((size_t)L * K * rank * 2);
    p.bt = take((size_t)L * N * rank * 2);
    p.outer_u = take(outer_bytes(p.n_tiles, rank));
    p.outer_v = take(outer_bytes(p.n_tiles, rank));
    p.partial = take((size_t)p.slots * rank * ((size_t)K + N) * sizeof(float));
  }
  p.bytes = at;
  return p;
}

template <typename T>
T* at(char* ws, size_t offset) {
  return reinterpret_cast<T*>(ws + offset);
}

Sort sort_of(const Plan& p, const int32_t* idx, int T, int L, char* ws) {
  return Sort{idx, T, L, p.chunk, p.n_tiles, p.n_pieces, at<int32_t>(ws, p.offsets), at<int32_t>(ws, p.list), at<Tile>(ws, p.tiles),
              at<Tile>(ws, p.pieces), at<int32_t>(ws, p.piece_slots), at<int32_t>(ws, p.slot0)};
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int size_status(int32_t T, int32_t K, int32_t N, int32_t rank, int32_t L) {
  if (T < 0 || T >= (1 << 24) || K < 8 || N < 8 || K > MOE_LORA_MAX_COLUMNS || N > MOE_LORA_MAX_COLUMNS ||
      rank < 1 || L < 1 || L > MOE_LORA_MAX_ADAPTERS)
    return MOE_ERR_INVALID_ARG;
  if (K % 8 != 0 || N % 8 != 0 || rank % 8 != 0 || rank > MOE_LORA_MAX_RANK) return MOE_ERR_UNSUPPORTED_SHAPE;
  return MOE_OK;
}

}  // namespace
}  // namespace moe

extern "C" {

size_t moe_lora_workspace_bytes(int32_t T, int32_t K, int32_t N, int32_t rank, int32_t n_adapters, int32_t backward) {
  if (moe::size_status(T, K, N, rank, n_adapters) != MOE_OK) return 0;
  return moe::make_plan(T, K, N, rank, n_adapters, backward != 0).bytes;
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
  const Plan p = make_plan(T, K, N, rank, n_adapters, false);
  char* const ws = static_cast<char*>(workspace);
  const uint16_t *x = static_cast<const uint16_t*>(x_bf16), *a = static_cast<const uint16_t*>(lora_a);
  const uint16_t* b = static_cast<const uint16_t*>(lora_b);
  const bool f32 = (flags & MOE_OUT_F32) != 0;
  if (p.few) {
    const Few few{adapter_idx, T, n_adapters};
    float* const part = at<float>(ws, p.part);
    const ExpandFew e{few, part, p.slices, rank, scale, v, b, N, y_in, y_out};
    const int wide = fused_wide(T, K, N, rank, n_adapters);
    if (wide > 0) {
      if (f32) launch_fused_few<float>(e, x, K, a, wide, s);
      else launch_fused_few<uint16_t>(e, x, K, a, wide, s);
    } else {
      launch_shrink_few(few, x, K, a, rank, part, s);
      if (f32) launch_expand_few<float>(e, s);
      else launch_expand_few<uint16_t>(e, s);
    }
  } else {
    launch_sort(sort_of(p, adapter_idx, T, n_adapters, ws), s);
    const int32_t* list = at<int32_t>(ws, p.list);
    const Tile* tiles = at<Tile>(ws, p.tiles);
    float* const part = at<float>(ws, p.part);
    u32x4* const packed = at<u32x4>(ws, p.packed);
    launch_shrink(Shrink{tiles, list, T, n_adapters, x, a, K, rank, part}, p.n_tiles, p.slices, s);
    const bool sums = from_sums(T, rank, p.slices);
    if (!sums)
      hipLaunchKernelGGL(pack_kernel, dim3(2 * p.n_tiles), dim3(kPackThreads), 0, s,
                         Pack{tiles, list, T, n_adapters, part, p.slices, rank, true, scale, v, packed, nullptr});
    const Expand e{tiles, list, T, n_adapters, sums ? nullptr : packed, rank, b, N, y_in, y_out, part, p.slices, scale, v};
    if (f32) launch_expand<float>(e, p.n_tiles, s);
    else launch_expand<uint16_t>(e, p.n_tiles, s);
  }
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
  const Plan p = make_plan(T, K, N, rank, n_adapters, true);
  char* const ws = static_cast<char*>(workspace);
  const Sort sort = sort_of(p, adapter_idx, T, n_adapters, ws);
  const int32_t *list = sort.list, *offsets = sort.offsets;
  const Tile* tiles = sort.tiles;
  u32x4 *const outer_u = at<u32x4>(ws, p.outer_u), *const outer_v = at<u32x4>(ws, p.outer_v);
  if (T > 0) {
    const int ra = ceil_div(rank, 64), ca = ceil_div(K, 64), cb = ceil_div(N, 64);
    uint16_t *const a_t = at<uint16_t>(ws, p.at), *const b_t = at<uint16_t>(ws, p.bt);
    const Transpose turn{{static_cast<const uint16_t*>(lora_a), static_cast<const uint16_t*>(lora_b)}, {a_t, b_t}, {rank, N}, {K, rank},
                         {ca, ra}, ra * ca, ra * (ca + cb), n_adapters, offsets};
    const int blocks = ceil_div(turn.tiles, kTurnTiles) * n_adapters;
    if (T <= kSortOnce) {
      hipLaunchKernelGGL(sort_and_transpose_kernel, dim3(1 + blocks), dim3(kSortThreads), 0, s, sort, turn);
    } else {
      launch_sort(sort, s);
      hipLaunchKernelGGL(transpose_kernel, dim3(blocks), dim3(kSortThreads), 0, s, turn);
    }
    float* const part = at<float>(ws, p.part);
    u32x4* const packed = at<u32x4>(ws, p.packed);
    launch_shrink(Shrink{tiles, list, T, n_adapters, dy, b_t, N, rank, part}, p.n_tiles, p.slices, s);
    hipLaunchKernelGGL(pack_both_kernel, dim3(4 * p.n_tiles), dim3(kPackThreads), 0, s,
                       Pack{tiles, list, T, n_adapters, part, p.slices, rank, true, scale, nullptr, dx != nullptr ? packed : nullptr, outer_u},
                       Pack{tiles, list, T, n_adapters, v, 1, rank, true, nullptr, nullptr, nullptr, outer_v}, 2 * p.n_tiles);
  } else {
    launch_sort(sort, s);
  }
  float* const partial = at<float>(ws, p.partial);
  const Outer o{at<Tile>(ws, p.pieces), at<int32_t>(ws, p.piece_slots), at<int32_t>(ws, p.slot0), offsets, list, T, n_adapters,
                {{x, outer_u, nullptr, grad_a, partial, K, ceil_div(K, kOuterCols), false},
                 {dy, outer_v, scale, grad_b, partial + (size_t)p.slots * rank * K, N, ceil_div(N, kOuterCols), true}},
                rank, p.chunk};
  if (dx != nullptr && T > 0) {
    const Expand e{tiles, list, T, n_adapters, at<u32x4>(ws, p.packed), rank, at<uint16_t>(ws, p.at), K, dx_in, dx};
    if (rank <= 16) launch_both<1, ExpandByGroup<1, 8>>(o, p.n_pieces, e, p.n_tiles, s);
    else if (rank <= 32) launch_both<2, ExpandByGroup<1, 8>>(o, p.n_pieces, e, p.n_tiles, s);
    else if (rank <= 64) launch_both<4, ExpandByGroup<2, 8>>(o, p.n_pieces, e, p.n_tiles, s);
    else launch_both<4, ExpandByGroup<4, 4>>(o, p.n_pieces, e, p.n_tiles, s);
  } else {
    launch_outer(o, p.n_pieces, s);
  }
  if (p.slots > 0) launch_reduce(o, s);
  return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP;
}

}  // extern "C"
