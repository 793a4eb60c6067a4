// Products of a long bf16 matrix with a narrow one (an adapter's rank, the router's experts: 8 to 256 wide), for rows that are
// grouped by the narrow matrix they use.  Three shapes make up the adapters' and the router's forward and backward passes:
//   shrink  P[t,j] = sum_k X[t,k] M_a[j,k]              a sum over the long side
//   expand  Y[t,n] = Y_in[t,n] + sum_j P[t,j] M_a[n,j]  a sum over the narrow side
//   outer   G_a[j,c] = sum over the rows t of group a of P[t,j] Z[t,c]
// All of them are bound by the one pass over X, Y or Z; the matrix cores do the sums (16x16x32 bf16, fp32 accumulators) with room to
// spare, so that the narrow fp32 operand P may go in as a sum of bf16 parts: two keep 16 bits of it (enough under a bf16 result's
// 8), three all 24 (for fp32 results).  The long operand is bf16 as it is, so nothing of it is lost.
#pragma once
#include "moe_internal.hpp"
#include "unit_list_wave.hpp"

namespace moe {
namespace skinny {

__device__ __forceinline__ f32x4 mfma(const uint4& a, const uint4& b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(*reinterpret_cast<const bf16x8*>(&a), *reinterpret_cast<const bf16x8*>(&b), c, 0,
                                                 0, 0);
}

// The highest 8 bits of eight floats as bf16; `v` keeps the rest, which is exact.
__device__ __forceinline__ uint4 take_bf16(float (&v)[8]) {
  uint32_t p[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    p[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
    v[2 * i] -= bf16_lo(p[i]);
    v[2 * i + 1] -= bf16_hi(p[i]);
  }
  return make_uint4(p[0], p[1], p[2], p[3]);
}

// ---- which rows a workgroup works on -----------------------------------------------------------------------------------------
// A tile: up to M rows of one group.  Rows are given by ids grouped in one of three ways.
struct Rows {
  const int32_t* offsets;  // [L+1] first position of each group in `list`; nullptr: not sorted (idx) or all one group (neither)
  const int32_t* list;     // positions -> rows; nullptr: position = row
  const int32_t* idx;      // [T] group of each row, for at most 64 rows that nobody has sorted
  int T, L;
};
struct Tile {
  int group, first, rows;  // group -1: rows without one; rows 0: nothing to do
};

// The b-th tile of M rows of the sorted groups; with `at_least_one` a group without rows has an empty tile.
// Four neighbouring groups a lane: their tiles are counted, a scan over the lanes finds the lane, the lane the group.
__device__ __forceinline__ Tile find_tile(const int32_t* __restrict__ offsets, int L, int M, int b, bool at_least_one) {
  const int lane = threadIdx.x & (kWave - 1);
  int o[5], c[4], sum = 0;
#pragma unroll
  for (int i = 0; i < 5; ++i) o[i] = offsets[min(4 * lane + i, L)];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    c[i] = (o[i + 1] - o[i] + M - 1) / M;
    if (at_least_one && 4 * lane + i < L) c[i] = max(c[i], 1);
    sum += c[i];
  }
  const int incl = gg::wave_incl_scan(sum);
  int rem = b - (incl - sum);
  const unsigned long long hit = __ballot(rem >= 0 && rem < sum);
  if (hit == 0) return Tile{-1, 0, 0};
  int g = 0, first = o[0], end = o[1];
#pragma unroll
  for (int i = 0; i < 3; ++i)
    if (g == i && rem >= c[i]) {
      rem -= c[i];
      g = i + 1;
      first = o[i + 1];
      end = o[i + 2];
    }
  first += rem * M;
  const int src = __ffsll((long long)hit) - 1;
  return Tile{(int)__builtin_amdgcn_readlane(4 * lane + g, src), (int)__builtin_amdgcn_readlane(first, src),
              (int)__builtin_amdgcn_readlane(min(M, end - first), src)};
}

// Fills s_rows[0 .. rows) and returns the tile.  Every wavefront computes the same; the caller synchronises before it reads s_rows.
template <int M>
__device__ __forceinline__ Tile take_tile(const Rows& r, int b, int32_t* s_rows) {
  const int tid = threadIdx.x, lane = tid & (kWave - 1);
  if (r.idx != nullptr) {
    // at most 64 rows (M of them or fewer), a lane each: the first row of a group works for all of them
    int g = lane < r.T ? r.idx[lane] : -2;
    if (lane < r.T && (unsigned)g >= (unsigned)r.L) g = -1;
    const int mine = (int)__builtin_amdgcn_readlane(g, b);
    const unsigned long long same = __ballot(g == mine);
    if (__ffsll((long long)same) - 1 != b) return Tile{-1, 0, 0};
    if (tid < kWave && g == mine) s_rows[__popcll(same & ((1ull << lane) - 1ull))] = lane;
    return Tile{mine, 0, (int)__popcll(same)};
  }
  Tile t{0, b * M, 0};
  if (r.offsets != nullptr) t = find_tile(r.offsets, r.L, M, b, false);
  else t.rows = max(0, min(M, r.T - t.first));
  for (int i = tid; i < t.rows; i += blockDim.x) s_rows[i] = r.list != nullptr ? r.list[t.first + i] : t.first + i;
  return t;
}

// ---- shrink ------------------------------------------------------------------------------------------------------------------
// A wavefront multiplies 16 MT rows by all of M_a over every (8 gridDim.y)-th 64-wide piece of k.  In each piece lane (row, q) loads k =
// 16 q .. 16 q + 15 of its row, so a row's four lanes read one whole 128-byte line, and so does the lane of M_a: the two MFMAs of a
// piece take the first and the second half of both, whose sum over k is the same in any order.  The eight wavefronts' results
// are added in order through LDS; gridDim.y pieces of the sum go to `part` [slice][T][r] (the reader adds them in order).
// U pieces are in flight before the first product: a prompt batch is a stream of x, a decoding batch a couple of memory round trips.
constexpr int kShrinkWaves = 8;

template <int MT, int NT, int U>
__global__ __launch_bounds__(kShrinkWaves * 64) void shrink_kernel(Rows rows, const uint16_t* __restrict__ x, int K,
                                                                   const uint16_t* __restrict__ m, int r,
                                                                   float* __restrict__ part) {
  constexpr int M = 16 * MT;
  __shared__ int32_t s_rows[M];
  __shared__ float red[kShrinkWaves][16][NT * 16 + 1];
  const Tile tile = take_tile<M>(rows, blockIdx.x, s_rows);
  if (tile.rows == 0 || tile.group < 0) return;
  __syncthreads();
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, row = lane & 15, q = lane >> 4;
  const uint16_t *xr[MT], *mr[NT];
#pragma unroll
  for (int i = 0; i < MT; ++i) xr[i] = x + (size_t)s_rows[min(16 * i + row, tile.rows - 1)] * K + 16 * q;
#pragma unroll
  for (int j = 0; j < NT; ++j) mr[j] = m + ((size_t)tile.group * r + min(16 * j + row, r - 1)) * K + 16 * q;
  f32x4 acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int stride = kShrinkWaves * gridDim.y;
  for (int c0 = (blockIdx.y * kShrinkWaves + wave) * 64; c0 < K; c0 += stride * 64 * U) {
    uint4 xv[U][MT][2], mv[U][NT][2];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int k = c0 + u * stride * 64 + 8 * h;
        const bool in = k + 16 * q < K;  // (K is a multiple of 8)
#pragma unroll
        for (int i = 0; i < MT; ++i) xv[u][i][h] = in ? *reinterpret_cast<const uint4*>(xr[i] + k) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int j = 0; j < NT; ++j) mv[u][j][h] = in ? *reinterpret_cast<const uint4*>(mr[j] + k) : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int j = 0; j < NT; ++j) acc[i][j] = mfma(xv[u][i][h], mv[u][j][h], acc[i][j]);
  }
  part += (size_t)blockIdx.y * rows.T * r;
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    if (16 * i >= tile.rows) break;
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) red[wave][4 * q + e][16 * j + row] = acc[i][j][e];
    __syncthreads();
    for (int o = tid; o < 16 * 16 * NT; o += kShrinkWaves * 64) {
      const int ro = o / (16 * NT), col = o % (16 * NT);
      float sum = 0.f;
#pragma unroll
      for (int w = 0; w < kShrinkWaves; ++w) sum += red[w][ro][col];
      if (16 * i + ro < tile.rows && col < r) part[(size_t)s_rows[16 * i + ro] * r + col] = sum;
    }
    __syncthreads();
  }
}

// ---- expand ------------------------------------------------------------------------------------------------------------------
// A wavefront keeps its 16 NJ rows of M_a (output columns) in registers and walks the tile's rows, 16 at a time.  The MFMA's first operand is
// M_a, its second P: an accumulator's four values are then four neighbouring columns of one row, and with the columns dealt out
// as below a lane holds 4 NJ neighbouring ones, so rows of Y are read and written in whole 128-byte lines.  P's parts lie in LDS, a
// row of them 16 bytes longer than a multiple of 32 so that the lanes' 16-byte reads spread over the banks; narrow sides that are no
// multiple of 32 end in zeros.  HILO: M_a itself is fp32, given as rows of two bf16 parts; the product of the two low parts (2^-17 of the whole) is
// left out.
struct Expand {
  Rows rows;
  const float* part;     // [slices][T][r]
  int slices, r;
  const float* scale;    // per group, or nullptr
  float* keep;           // [T][r] the sum over the slices (times scale if keep_scaled), 0 for rows without a group; or nullptr
  bool keep_scaled;
  const uint16_t* m;     // [L][N][m_stride]
  int m_stride, N;
  const void* y_in;      // [T][N] or nullptr
  void* y_out;           // nullptr: only `keep`
  int n_tiles;           // gridDim.y from here on: workgroups for the rows without a group
  bool vec;              // rows of `part` are made of whole 16-byte pieces
};

constexpr int kExpandThreads = 256;
constexpr int kExpandWaves = kExpandThreads / kWave;

__device__ __forceinline__ void load8(const uint16_t* p, float (&v)[8]) {
  const uint4 a = *reinterpret_cast<const uint4*>(p);
  v[0] = bf16_lo(a.x); v[1] = bf16_hi(a.x); v[2] = bf16_lo(a.y); v[3] = bf16_hi(a.y);
  v[4] = bf16_lo(a.z); v[5] = bf16_hi(a.z); v[6] = bf16_lo(a.w); v[7] = bf16_hi(a.w);
}
__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void store8(uint16_t* p, const float (&v)[8]) {
  *reinterpret_cast<uint4*>(p) =
      make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}

// The rows s_rows[0 .. n) have no group: the output is the input, `keep` is 0.
template <typename YT>
__device__ __forceinline__ void copy_rows(const Expand& e, const int32_t* s_rows, int n, int c0, int cols) {
  const YT* in = static_cast<const YT*>(e.y_in);
  YT* out = static_cast<YT*>(e.y_out);
  cols = min(cols, e.N - c0);
  if (out != nullptr && in != out)
    for (int i = threadIdx.x; i < n * (cols / 8); i += kExpandThreads) {
      const size_t at = (size_t)s_rows[i / (cols / 8)] * e.N + c0 + i % (cols / 8) * 8;
      float v[8] = {};
      if (in != nullptr) load8(in + at, v);
      store8(out + at, v);
    }
  if (e.keep != nullptr && c0 == 0)
    for (int i = threadIdx.x; i < n * e.r; i += kExpandThreads) e.keep[(size_t)s_rows[i / e.r] * e.r + i % e.r] = 0.f;
}

template <typename YT, int SPLIT, int WCH, int NJ, bool HILO>
__global__ __launch_bounds__(kExpandThreads) void expand_kernel(Expand e) {
  constexpr int R = 32 * WCH, M = SPLIT * R <= 256 ? 128 : 64, COLS = kExpandWaves * 16 * NJ;
  constexpr int kRowBytes = SPLIT * R * 2 + 16, PARTS = HILO ? 2 : 1, kGroups = NJ / 2;
  __shared__ int32_t s_rows[M];
  __shared__ __align__(16) char s_p[M * kRowBytes];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, ln = lane & 15, q = lane >> 4;
  const int T = e.rows.T, r = e.r;
  if (blockIdx.y >= (unsigned)e.n_tiles) {  // sorted rows: those that are in no group
    const int t = (blockIdx.y - e.n_tiles) * 64 + lane;
    const bool bare = t < T && (unsigned)e.rows.idx[t] >= (unsigned)e.rows.L;
    const unsigned long long all = __ballot(bare);
    if (all == 0) return;
    if (bare && wave == 0) s_rows[__popcll(all & ((1ull << lane) - 1ull))] = t;
    __syncthreads();
    copy_rows<YT>(e, s_rows, __popcll(all), blockIdx.x * COLS, COLS);
    return;
  }
  Rows sorted = e.rows;
  if (sorted.offsets != nullptr) sorted.idx = nullptr;
  const Tile tile = take_tile<M>(sorted, blockIdx.y, s_rows);
  if (tile.rows == 0) return;
  __syncthreads();
  if (tile.group < 0) {
    copy_rows<YT>(e, s_rows, tile.rows, blockIdx.x * COLS, COLS);
    return;
  }
  const int nbase = (blockIdx.x * kExpandWaves + wave) * 16 * NJ;
  uint4 w[PARTS][WCH][NJ];
  if (e.y_out != nullptr) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int n = nbase + (ln >> 2) * (4 * NJ) + 4 * j + (ln & 3);
      const uint16_t* mr = e.m + ((size_t)tile.group * e.N + min(n, e.N - 1)) * e.m_stride + 8 * q;
#pragma unroll
      for (int p = 0; p < PARTS; ++p)
#pragma unroll
        for (int c = 0; c < WCH; ++c)
          w[p][c][j] = (HILO || 32 * c + 8 * q < r) ? *reinterpret_cast<const uint4*>(mr + p * R + 32 * c) : make_uint4(0, 0, 0, 0);
    }
  }
  const float scale = e.scale != nullptr ? e.scale[tile.group] : 1.f;
  const int row_tiles = (tile.rows + 15) / 16;
  const size_t slice = (size_t)T * r;
  for (int o = tid; o < row_tiles * 16 * (R / 8); o += kExpandThreads) {
    const int i = o / (R / 8), j0 = o % (R / 8) * 8;
    float v[8] = {};
    if (i < tile.rows && j0 < r) {
      const size_t at = (size_t)s_rows[i] * r + j0;
      if (e.vec) {
        const bool second = j0 + 4 < r;
        for (int s = 0; s < e.slices; ++s) {
          const float4 a = *reinterpret_cast<const float4*>(e.part + s * slice + at);
          const float4 b = second ? *reinterpret_cast<const float4*>(e.part + s * slice + at + 4) : make_float4(0.f, 0.f, 0.f, 0.f);
          v[0] += a.x; v[1] += a.y; v[2] += a.z; v[3] += a.w; v[4] += b.x; v[5] += b.y; v[6] += b.z; v[7] += b.w;
        }
      } else {
        for (int s = 0; s < e.slices; ++s)
#pragma unroll
          for (int k = 0; k < 8; ++k)
            if (j0 + k < r) v[k] += e.part[s * slice + at + k];
      }
      if (e.keep != nullptr && blockIdx.x == 0)
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (j0 + k < r) e.keep[at + k] = e.keep_scaled ? scale * v[k] : v[k];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] *= scale;
    }
#pragma unroll
    for (int p = 0; p < SPLIT; ++p) *reinterpret_cast<uint4*>(s_p + i * kRowBytes + p * R * 2 + j0 * 2) = take_bf16(v);
  }
  __syncthreads();
  if (e.y_out == nullptr || nbase >= e.N) return;
  const YT* in = static_cast<const YT*>(e.y_in);
  YT* out = static_cast<YT*>(e.y_out);
  const int c0 = nbase + q * (4 * NJ);
  constexpr int U = 4;
  for (int tt0 = 0; tt0 < row_tiles; tt0 += U) {
    float y[U][kGroups][8];
    size_t at[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      at[u] = (size_t)s_rows[min((tt0 + u) * 16 + ln, tile.rows - 1)] * e.N + c0;
#pragma unroll
      for (int h = 0; h < kGroups; ++h) {
#pragma unroll
        for (int k = 0; k < 8; ++k) y[u][h][k] = 0.f;
        if (in != nullptr && c0 + 8 * h < e.N && (tt0 + u) * 16 + ln < tile.rows) load8(in + at[u] + 8 * h, y[u][h]);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (tt0 + u >= row_tiles) break;
      f32x4 acc[NJ];
#pragma unroll
      for (int j = 0; j < NJ; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
      const char* p = s_p + ((tt0 + u) * 16 + ln) * kRowBytes + q * 16;
#pragma unroll
      for (int c = 0; c < WCH; ++c)
#pragma unroll
        for (int s = SPLIT - 1; s >= 0; --s) {  // the small parts first
          const uint4 b = *reinterpret_cast<const uint4*>(p + s * R * 2 + c * 64);
#pragma unroll
          for (int j = 0; j < NJ; ++j) acc[j] = mfma(w[0][c][j], b, acc[j]);
          if (HILO && s == 0)
#pragma unroll
            for (int j = 0; j < NJ; ++j) acc[j] = mfma(w[PARTS - 1][c][j], b, acc[j]);
        }
      if ((tt0 + u) * 16 + ln < tile.rows)
#pragma unroll
        for (int h = 0; h < kGroups; ++h)
          if (c0 + 8 * h < e.N) {
#pragma unroll
            for (int k = 0; k < 8; ++k) y[u][h][k] += acc[2 * h + k / 4][k % 4];
            store8(out + at[u] + 8 * h, y[u][h]);
          }
    }
  }
}

// ---- outer -------------------------------------------------------------------------------------------------------------------
// A wavefront takes 32 rows at a time: lane (c, q) loads 8 neighbouring columns of rows 8 q .. 8 q + 7, a row's 16 lanes 256 bytes in a
// row, and byte permutations turn the eight 16-byte rows into eight column fragments (rows are the sum's index): no trip through
// LDS.  P's fragments are read as they lie and split in three parts.  The eight wavefronts take every eighth 32 rows; their sums are
// added in order through LDS, 16 of P's columns at a time.  A group of more than `chunk` rows is cut, its pieces' sums go to `part`
// and join in reduce_kernel: which pieces there are follows from the rows alone, so the order of the additions is fixed.
struct OuterSide {
  const uint16_t* z;   // [T][cols]
  const float* p;      // [T][r]
  const float* scale;  // per group, or nullptr
  float* out;          // [L][r][cols], or [L][cols][r] if by_column
  float* part;         // the same for each piece of a cut group
  int cols, tiles;     // tiles of 128 columns
  bool by_column;
};
struct Outer {
  Rows rows;
  OuterSide side[2];
  int r, chunk;
};

constexpr int kOuterWaves = 8, kOuterCols = 128;

// The place of the b-th piece in `part`: the pieces of cut groups before it; -1: its group is not cut.
__device__ __forceinline__ int piece_slot(const Rows& rows, int chunk, const Tile& t) {
  const int lane = threadIdx.x & (kWave - 1);
  if (rows.offsets == nullptr) return rows.T > chunk ? t.first / chunk : -1;
  int before = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int g = 4 * lane + i;
    const int n = g < t.group ? rows.offsets[min(g + 1, rows.L)] - rows.offsets[min(g, rows.L)] : 0;
    if (n > chunk) before += (n + chunk - 1) / chunk;
  }
  before = (int)__builtin_amdgcn_readlane(gg::wave_incl_scan(before), kWave - 1);
  const int first = rows.offsets[t.group], n = rows.offsets[t.group + 1] - first;
  return n > chunk ? before + (t.first - first) / chunk : -1;
}

template <int MT>
__global__ __launch_bounds__(kOuterWaves * 64) void outer_kernel(Outer o) {
  __shared__ float red[kOuterWaves][16][kOuterCols + 4];
  const OuterSide& sd = o.side[blockIdx.x >= (unsigned)o.side[0].tiles];
  const int col_tile = blockIdx.x >= (unsigned)o.side[0].tiles ? blockIdx.x - o.side[0].tiles : blockIdx.x;
  Tile tile{0, (int)blockIdx.y * o.chunk, 0};
  if (o.rows.offsets != nullptr) tile = find_tile(o.rows.offsets, o.rows.L, o.chunk, blockIdx.y, true);
  else tile.rows = min(o.chunk, o.rows.T - tile.first);
  if (tile.group < 0) return;
  const int slot = piece_slot(o.rows, o.chunk, tile);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, c = lane & 15, q = lane >> 4;
  const int r = o.r, r0 = blockIdx.z * 16 * MT, c0 = col_tile * kOuterCols;
  f32x4 acc[MT][8];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int zc = min(c0 + 8 * c, sd.cols - 8);  // columns past the end are computed and not stored
  for (int s0 = wave * 32; s0 < tile.rows; s0 += kOuterWaves * 32) {
    int row[8];
    uint4 z[8];
    float p[MT][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int at = min(s0 + 8 * q + i, tile.rows - 1);  // (past the end: a row of the same group, times 0)
      row[i] = o.rows.list != nullptr ? o.rows.list[tile.first + at] : tile.first + at;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = *reinterpret_cast<const uint4*>(sd.z + (size_t)row[i] * sd.cols + zc);
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int j = r0 + 16 * m + c;
        p[m][i] = (j < r && s0 + 8 * q + i < tile.rows) ? sd.p[(size_t)row[i] * r + j] : 0.f;
      }
    uint4 f[8];
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      uint32_t lo[4], hi[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t a = reinterpret_cast<const uint32_t*>(&z[2 * i])[d], b = reinterpret_cast<const uint32_t*>(&z[2 * i + 1])[d];
        lo[i] = __builtin_amdgcn_perm(b, a, 0x05040100u);
        hi[i] = __builtin_amdgcn_perm(b, a, 0x07060302u);
      }
      f[2 * d] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
      f[2 * d + 1] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
    }
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int s = 0; s < 3; ++s) {
        const uint4 a = take_bf16(p[m]);
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[m][j] = mfma(a, f[j], acc[m][j]);
      }
  }
  const float scale = sd.scale != nullptr ? sd.scale[tile.group] : 1.f;
  float* out = slot >= 0 ? sd.part + (size_t)slot * r * sd.cols : sd.out + (size_t)tile.group * r * sd.cols;
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    if (r0 + 16 * m >= r) break;
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        *reinterpret_cast<float4*>(&red[wave][4 * q + e][8 * c + 4 * h]) =
            make_float4(acc[m][4 * h][e], acc[m][4 * h + 1][e], acc[m][4 * h + 2][e], acc[m][4 * h + 3][e]);
    __syncthreads();
    if (!sd.by_column) {
      const int j = tid >> 5, n = (tid & 31) * 4;
      float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kOuterWaves; ++w) {
        const float4 a = *reinterpret_cast<const float4*>(&red[w][j][n]);
        sum.x += a.x; sum.y += a.y; sum.z += a.z; sum.w += a.w;
      }
      if (r0 + 16 * m + j < r && c0 + n < sd.cols)
        *reinterpret_cast<float4*>(out + (size_t)(r0 + 16 * m + j) * sd.cols + c0 + n) =
            make_float4(sum.x * scale, sum.y * scale, sum.z * scale, sum.w * scale);
    } else {
      const int j = tid & 15;
#pragma unroll
      for (int h = 0; h < kOuterCols / 32; ++h) {
        const int n = (tid >> 4) + 32 * h;
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < kOuterWaves; ++w) sum += red[w][j][n];
        if (r0 + 16 * m + j < r && c0 + n < sd.cols) out[(size_t)(c0 + n) * r + r0 + 16 * m + j] = sum * scale;
      }
    }
    __syncthreads();
  }
}

// Adds the pieces of cut groups in order.  blockIdx.y: the group.
static __global__ __launch_bounds__(256) void reduce_kernel(Outer o) {
  const int g = blockIdx.y;
  const int first = o.rows.offsets != nullptr ? o.rows.offsets[g] : 0;
  const int n = o.rows.offsets != nullptr ? o.rows.offsets[g + 1] - first : o.rows.T;
  if (n <= o.chunk) return;
  const int slot = piece_slot(o.rows, o.chunk, Tile{g, first, n}), pieces = (n + o.chunk - 1) / o.chunk;
  for (int s = 0; s < 2; ++s) {
    const OuterSide& sd = o.side[s];
    const size_t size = (size_t)o.r * sd.cols;  // (a multiple of 8)
    for (size_t i = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4; i < size; i += (size_t)gridDim.x * 1024) {
      float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int p = 0; p < pieces; ++p) {
        const float4 a = *reinterpret_cast<const float4*>(sd.part + (size_t)(slot + p) * size + i);
        sum.x += a.x; sum.y += a.y; sum.z += a.z; sum.w += a.w;
      }
      *reinterpret_cast<float4*>(sd.out + (size_t)g * size + i) = sum;
    }
  }
}

}  // namespace skinny
}  // namespace moe
