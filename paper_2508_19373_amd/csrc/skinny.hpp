// Products of a long bf16 matrix with a narrow one (an adapter's rank, the router's experts: 8 to 256 wide), for rows that are
// grouped by the narrow matrix they use.  Three shapes make up the adapters' and the router's forward and backward passes:
//   shrink  P[t,j] = sum_k X[t,k] M_a[j,k]              a sum over the long side
//   expand  Y[t,n] = Y_in[t,n] + sum_j P[t,j] M_a[n,j]  a sum over the narrow side
//   outer   G_a[j,c] = sum over the rows t of group a of P[t,j] Z[t,c]
// All of them are bound by the one pass over X, Y or Z; the matrix cores do the sums (16x16x32 bf16, fp32 accumulators) with room to
// spare, so that the narrow fp32 operand P goes in as a sum of three bf16 parts, all 24 bits of it.  The long operand is bf16 as it is, so
// nothing of it is lost either.
//
// How the long side is read decides the speed: an MFMA's lanes l, l + 1, ... hold different rows, and a load in that order takes the address
// unit 64 clocks an instruction (a lane at a time) instead of 16.  So neighbouring lanes read neighbouring 16 bytes of a row, and either
// LDS (shrink, M_a) or the choice of which columns an accumulator stands for (expand's Y, outer's Z) brings them to the lanes that need
// them.  P, small and read by every column block, is laid out once in the order of the lanes ("packed").
#pragma once
#include "moe_internal.hpp"
#include "unit_list_wave.hpp"

namespace moe {
namespace skinny {

// 16 bytes as the compiler's own vector (arrays of them stay in registers)
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x4 mfma(const u32x4& a, const u32x4& b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(*reinterpret_cast<const bf16x8*>(&a), *reinterpret_cast<const bf16x8*>(&b), c, 0,
                                                 0, 0);
}

// Between LDS accesses by which lanes of one wavefront hand values to each other: the hardware keeps them in order, the compiler has to.
__device__ __forceinline__ void wave_fence() {
#ifdef __HIP_DEVICE_COMPILE__
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#endif
}

// The highest 8 bits of eight floats as bf16; `v` keeps the rest, which is exact.
__device__ __forceinline__ u32x4 take_bf16(float (&v)[8]) {
  uint32_t p[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    p[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
    v[2 * i] -= bf16_lo(p[i]);
    v[2 * i + 1] -= bf16_hi(p[i]);
  }
  return u32x4{p[0], p[1], p[2], p[3]};
}

__device__ __forceinline__ void load8(const uint16_t* p, float (&v)[8]) {
  const u32x4 a = *reinterpret_cast<const u32x4*>(p);
  v[0] = bf16_lo(a.x); v[1] = bf16_hi(a.x); v[2] = bf16_lo(a.y); v[3] = bf16_hi(a.y);
  v[4] = bf16_lo(a.z); v[5] = bf16_hi(a.z); v[6] = bf16_lo(a.w); v[7] = bf16_hi(a.w);
}
__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}

constexpr int kParts = 3;  // bf16 parts of an fp32 operand

inline int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }
inline size_t padded(size_t bytes) { return (bytes + 255) / 256 * 256; }

// ---- rows sorted by group ----------------------------------------------------------------------------------------------------
// Rows in order of their group (of equal groups in their own order), and lists of the work that follows from it: tiles of rows of one
// group each.  Rows without a group (ids outside [0, L)) come last, as group L.
struct Tile {
  int32_t group, first, rows, at;  // first: position in the list; rows 0: nothing to do
};
constexpr int kTileRows = 64;

// Tiles of kTileRows rows that T rows in at most L groups can have.
inline int max_tiles(int T, int L) { return T / kTileRows + (L < T ? L : T); }

constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / kWave, kMaxGroups = 256;

struct Sort {
  const int32_t* idx;
  int T, L, chunk;           // chunk: rows of a piece, 0: none are listed
  int n_tiles, n_pieces;     // entries of the lists
  int32_t* offsets;          // [L+2] first position of each group in `list`
  int32_t* list;             // [T] positions -> rows
  Tile* tiles;               // of kTileRows rows; at: their number
  Tile* pieces;              // of up to `chunk` rows, one at least for each group < L; at: the number of their first 32 rows
  int32_t* slots;            // the place of a piece's partial result, -1: its group is not cut
  int32_t* slot0;            // [L] that of a group's first piece
};

// The lanes of the wavefront with this lane's group: a ballot for each bit of the id.  Prompts lie in runs, so often it is all of them.
__device__ __forceinline__ unsigned long long match_lanes(int g, bool in, int bits) {
  const unsigned long long all = __ballot(in);
  if (__ballot(in && g == (int)__builtin_amdgcn_readfirstlane(g)) == ~0ull) return all;
  unsigned long long same = all;
  for (int b = 0; b < bits; ++b) {
    const unsigned long long set = __ballot((g >> b) & 1);
    same &= ((g >> b) & 1) ? set : ~set;
  }
  return same;
}

// The last entry of pre[0 .. n] (non-decreasing) that is not above v.
__device__ __forceinline__ int find_group(const int32_t* pre, int n, int v) {
  int lo = 0, hi = n;  // pre[lo] <= v < pre[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (pre[mid] <= v) lo = mid;
    else hi = mid;
  }
  return lo;
}

// One workgroup: each wavefront counts the groups of its share of the rows, a scan over the groups places them, and the rows go to their
// places.  ONE: up to kSortOnce rows, whose places within the share stay in registers; else the wavefronts count again.  (Several workgroups
// would need launches between the steps, which cost more until there are some ten thousand rows; beyond, the products take longer by
// far.)  4096 rows take 4.6 us, 8192 7.2, bound by latency.
constexpr int kSortSteps = 8, kSortOnce = kSortWaves * kSortSteps * kWave;

template <bool ONE>
__device__ __forceinline__ void sort_block(const Sort& s) {
  __shared__ int32_t cnt[kSortWaves][kMaxGroups + 1];
  __shared__ int32_t pre[5][kMaxGroups + 2];  // prefixes over the groups of rows, tiles, whole pieces, other pieces, slots
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, groups = s.L + 1, bits = 32 - __clz(s.L);
  const int share = ((s.T + kSortWaves - 1) / kSortWaves + kWave - 1) / kWave * kWave;
  const int t0 = min(wave * share, s.T), t1 = min(t0 + share, s.T);
  int g[kSortSteps], place[kSortSteps];
  const auto load_groups = [&](int t) {
#pragma unroll
    for (int u = 0; u < kSortSteps; ++u) {
      const int at = t + u * kWave + lane;
      const int id = s.idx[min(at, s.T - 1)];
      g[u] = (unsigned)id < (unsigned)s.L ? id : s.L;
    }
  };
  // Places of 64 rows behind each other among their group's rows that `cnt` has counted, which counts them.
  const auto count = [&](int t) {
#pragma unroll
    for (int u = 0; u < kSortSteps; ++u) {
      if (t + u * kWave >= t1) break;
      const bool in = t + u * kWave + lane < t1;
      const unsigned long long same = match_lanes(g[u], in, bits);
      const int leader = __ffsll((long long)same) - 1;
      int before = 0;
      if (in && lane == leader) before = atomicAdd(&cnt[wave][g[u]], (int)__popcll(same));
      place[u] = __shfl(before, leader) + (int)__popcll(same & ((1ull << lane) - 1ull));
    }
  };
  if (ONE && s.T > 0) load_groups(t0);
  for (int e = lane; e < groups; e += kWave) cnt[wave][e] = 0;
  wave_fence();
  if (ONE) {
    count(t0);
  } else {
    for (int t = t0; t < t1; t += kSortSteps * kWave) {
      load_groups(t);
      count(t);
    }
  }
  __syncthreads();
  for (int e = tid; e < groups; e += kSortThreads) {  // rows of the group in the wavefronts before each; all of them
    int run = 0;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
      const int c = cnt[w][e];
      cnt[w][e] = run;
      run += c;
    }
    pre[0][e] = run;
  }
  __syncthreads();
  if (wave == 0) {
    int carry[5] = {};
    for (int e0 = 0; e0 < groups; e0 += kWave) {
      const int e = e0 + lane;
      const int c = e < groups ? pre[0][e] : 0;
      int v[5] = {c, (c + kTileRows - 1) / kTileRows, 0, 0, 0};
      if (s.chunk > 0 && e < s.L) {
        v[2] = c / s.chunk;
        v[3] = c % s.chunk != 0 || c == 0;
        v[4] = c > s.chunk ? v[2] + v[3] : 0;
      }
#pragma unroll
      for (int k = 0; k < 5; ++k) {
        const int incl = gg::wave_incl_scan(v[k]);
        if (e < groups) pre[k][e] = carry[k] + incl - v[k];
        carry[k] += (int)__builtin_amdgcn_readlane(incl, kWave - 1);
      }
    }
    if (lane == 0)
#pragma unroll
      for (int k = 0; k < 5; ++k) pre[k][groups] = carry[k];
  }
  __syncthreads();
  for (int e = tid; e <= groups; e += kSortThreads) s.offsets[e] = pre[0][e];
  for (int t = t0; t < t1; t += kSortSteps * kWave) {
    if (!ONE) {
      load_groups(t);
      count(t);  // (`cnt` goes on from the rows before)
    }
#pragma unroll
    for (int u = 0; u < kSortSteps; ++u) {
      const int row = t + u * kWave + lane;
      if (row < t1) s.list[pre[0][g[u]] + place[u] + (ONE ? cnt[wave][g[u]] : 0)] = row;
    }
  }
  for (int i = tid; i < s.n_tiles; i += kSortThreads) {
    Tile t{-1, 0, 0, 0};
    if (i < pre[1][groups]) {
      const int e = find_group(pre[1], groups, i), k = (i - pre[1][e]) * kTileRows, n = pre[0][e + 1] - pre[0][e];
      t = Tile{e, pre[0][e] + k, min(kTileRows, n - k), i};
    }
    s.tiles[i] = t;
  }
  const int whole = pre[2][groups];
  for (int i = tid; i < s.n_pieces; i += kSortThreads) {  // the whole pieces first: workgroups that end last are short ones
    Tile t{-1, 0, 0, 0};
    int slot = -1;
    if (i < whole + pre[3][groups]) {
      const int e = i < whole ? find_group(pre[2], groups, i) : find_group(pre[3], groups, i - whole);
      const int n = pre[0][e + 1] - pre[0][e], p = i < whole ? i - pre[2][e] : n / s.chunk, k = p * s.chunk;
      t = Tile{e, pre[0][e] + k, min(s.chunk, n - k), pre[1][e] * (kTileRows / 32) + k / 32};
      if (n > s.chunk) slot = pre[4][e] + p;
      if (p == 0) s.slot0[e] = slot;
    }
    s.pieces[i] = t;
    s.slots[i] = slot;
  }
}

template <bool ONE>
__global__ __launch_bounds__(kSortThreads) void sort_kernel(Sort s) {
  sort_block<ONE>(s);
}

inline void launch_sort(const Sort& a, hipStream_t s) {
  if (a.T <= kSortOnce) hipLaunchKernelGGL(sort_kernel<true>, dim3(1), dim3(kSortThreads), 0, s, a);
  else hipLaunchKernelGGL(sort_kernel<false>, dim3(1), dim3(kSortThreads), 0, s, a);
}

// ---- shrink ------------------------------------------------------------------------------------------------------------------
// A workgroup of 4 wavefronts computes one slice (blockIdx.y) of the sum for 64 rows, a wavefront a quarter of the slice in pieces of 64:
// 128 bytes of each row, read by eight neighbouring lanes, put into the wavefront's own piece of LDS with the 16-byte parts of a row
// rearranged by the row's number, and read back as fragments without bank conflicts.  The next piece of x is on its way from HBM
// meanwhile, and the next 32 rows of M_a from L2.  The wavefronts' sums are added in order through LDS, the slices' by pack_kernel.
// Why slices: what counts is how many bytes the busiest compute unit reads, about 45 KB a microsecond at best.  With 16 rows of all of k a
// workgroup, M_a would be twice x's bytes at rank 32, and 260 workgroups on 256 units took half as long again as 256 (19 and 12.6 us; 33 MB
// of x).  Now 14.1 us for 4096 rows of 4096 at rank 32 (2.4 TB/s of x), 29.7 for 8192 at rank 64.  The busiest unit's bytes (288 and 768 KB)
// take 6.4 and 17 of these; what the rest goes into is not known: a slice leaves a wavefront two to four pieces and the next one's loads
// cover little of their own latency.
constexpr int kShrinkWaves = 4, kShrinkThreads = kShrinkWaves * 64;

struct Shrink {
  const Tile* tiles;
  const int32_t* list;
  int T, L;
  const uint16_t* x;  // [T][K]
  const uint16_t* m;  // [L][r][K]
  int K, r;
  float* part;        // [slices][T][r]
};

template <int NT>
__global__ __launch_bounds__(kShrinkThreads, 2) void shrink_kernel(Shrink a) {
  constexpr int M = kTileRows, MT = M / 16, NG = NT < 2 ? NT : 2, GROUPS = NT / NG;
  constexpr int kWaveBytes = (M + 16 * NG) * 128, kRedStride = NT * 16 + 4, kRound = NT <= 2 ? 64 : 128 / NT;  // rows joined at a time
  constexpr int kRedBytes = kShrinkWaves * kRound * kRedStride * 4, kBytes = kShrinkWaves * kWaveBytes;
  __shared__ int32_t s_rows[M];
  __shared__ __align__(16) char s_buf[kBytes > kRedBytes ? kBytes : kRedBytes];
  const Tile tile = a.tiles[blockIdx.x];
  if (tile.rows == 0 || tile.group == a.L) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, ln = lane & 15, q = lane >> 4, sub = lane >> 3, ch = lane & 7;
  const int K = a.K, r = a.r;
  if (tid < M) s_rows[tid] = a.list[tile.first + min(tid, tile.rows - 1)];
  const uint16_t* xr[2 * MT];
#pragma unroll
  for (int i = 0; i < 2 * MT; ++i) xr[i] = a.x + (size_t)a.list[tile.first + min(8 * i + sub, tile.rows - 1)] * K + 8 * ch;
  const uint16_t* const mg = a.m + (size_t)tile.group * r * K + 8 * ch;
  char* const s_x = s_buf + wave * kWaveBytes;
  char* const s_m = s_x + M * 128;
  const int put = sub * 128 + (ch ^ sub) * 16;  // + 1024 for each eight rows
  f32x4 acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int pieces = (K + 63) / 64, parts = kShrinkWaves * gridDim.y, w = blockIdx.y * kShrinkWaves + wave;
  const int first = pieces * w / parts, n = pieces * (w + 1) / parts - first;
  // Straight-line code: a load under a condition makes the compiler wait for all loads.  Past the end the last piece is loaded again,
  // past K the first columns, and x's part set to zero.  Loads return in the order they are issued in, so M_a's go first.
  u32x4 xv[2 * MT], mv[2 * NG];
  const auto load_x = [&](int i) {
    int c = (first + min(i, n - 1)) * 64;
    c = c + 8 * ch < K ? c : -8 * ch;  // (K is a multiple of 8)
#pragma unroll
    for (int k = 0; k < 2 * MT; ++k) xv[k] = *reinterpret_cast<const u32x4*>(xr[k] + c);
  };
  const auto load_m = [&](int i, int g) {
    int c = (first + min(i, n - 1)) * 64;
    c = c + 8 * ch < K ? c : -8 * ch;
#pragma unroll
    for (int k = 0; k < 2 * NG; ++k) mv[k] = *reinterpret_cast<const u32x4*>(mg + (size_t)min(32 * g + 8 * k + sub, r - 1) * K + c);
  };
  if (n > 0) {
    load_m(0, 0);
    load_x(0);
  }
  for (int i = 0; i < n; ++i) {
    const bool in = (first + i) * 64 + 8 * ch < K;
#pragma unroll
    for (int k = 0; k < 2 * MT; ++k) {
      const u32x4 v = xv[k];
      *reinterpret_cast<u32x4*>(s_x + put + 1024 * k) = u32x4{in ? v.x : 0u, in ? v.y : 0u, in ? v.z : 0u, in ? v.w : 0u};
    }
    wave_fence();
    u32x4 f[MT][2];
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        f[t][h] = *reinterpret_cast<const u32x4*>(s_x + (16 * t + ln) * 128 + (((4 * h + q) ^ (ln & 7)) * 16));
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
#pragma unroll
      for (int k = 0; k < 2 * NG; ++k) *reinterpret_cast<u32x4*>(s_m + put + 1024 * k) = mv[k];
      wave_fence();
      if (g + 1 < GROUPS) load_m(i, g + 1);
      else {
        load_m(i + 1, 0);
        __builtin_amdgcn_sched_barrier(0);
        load_x(i + 1);
      }
#pragma unroll
      for (int j = 0; j < NG; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const u32x4 b = *reinterpret_cast<const u32x4*>(s_m + (16 * j + ln) * 128 + (((4 * h + q) ^ (ln & 7)) * 16));
#pragma unroll
          for (int t = 0; t < MT; ++t) acc[t][g * NG + j] = mfma(f[t][h], b, acc[t][g * NG + j]);
        }
      wave_fence();
    }
  }
  float* const red = reinterpret_cast<float*>(s_buf);  // [wave][kRound][kRedStride]
  float* const part = a.part + (size_t)blockIdx.y * a.T * r;
#pragma unroll
  for (int t0 = 0; t0 < M; t0 += kRound) {
    if (t0 >= tile.rows) break;
    __syncthreads();
#pragma unroll
    for (int t = 0; t < kRound / 16; ++t)
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          red[(wave * kRound + 16 * t + 4 * q + e) * kRedStride + 16 * j + ln] = acc[t0 / 16 + t][j][e];
    __syncthreads();
#pragma unroll
    for (int o = tid; o < kRound * 4 * NT; o += kShrinkThreads) {
      const int ro = o / (4 * NT), col = o % (4 * NT) * 4;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kShrinkWaves; ++w) {
        const float4 p = *reinterpret_cast<const float4*>(red + (w * kRound + ro) * kRedStride + col);
        v.x += p.x, v.y += p.y, v.z += p.z, v.w += p.w;
      }
      if (t0 + ro < tile.rows && col < r) *reinterpret_cast<float4*>(part + (size_t)s_rows[t0 + ro] * r + col) = v;
    }
  }
}

// Slices of the sum: about 512 workgroups, two pieces of 64 for each wavefront at least, 8 slices (which pack_kernel reads at once) at most.
inline int shrink_slices(int T, int K) {
  int n = ceil_div(512, ceil_div(T, kTileRows));
  const int most = ceil_div(K, 64 * 2 * kShrinkWaves);
  if (n > most) n = most;
  return n < 8 ? n : 8;
}

inline void launch_shrink(const Shrink& a, int n_tiles, int slices, hipStream_t s) {
  const dim3 grid(n_tiles, slices), block(kShrinkThreads);
  if (a.r <= 16) hipLaunchKernelGGL(shrink_kernel<1>, grid, block, 0, s, a);
  else if (a.r <= 32) hipLaunchKernelGGL(shrink_kernel<2>, grid, block, 0, s, a);
  else if (a.r <= 64) hipLaunchKernelGGL(shrink_kernel<4>, grid, block, 0, s, a);
  else hipLaunchKernelGGL(shrink_kernel<8>, grid, block, 0, s, a);
}

// ---- pack --------------------------------------------------------------------------------------------------------------------
// P from its slices, added in order, in the forms that the products read: a wavefront's 64 lanes one after the other, 16 bytes each.
// 32 rows a workgroup: half a tile.
struct Pack {
  const Tile* tiles;    // nullptr: all rows one group
  const int32_t* list;
  int T, L;
  const float* part;    // [slices][T][r]
  int slices, r;
  bool vec;             // rows of `part` are made of whole 16-byte pieces
  const float* scale;   // per group, for `packed` and `outer`; or nullptr
  float* keep;          // [T][r] the sums as they are, zeros for rows without a group; or nullptr
  u32x4* packed;        // for expand: [tiles][4][chunks of 32 columns][kParts][64]; or nullptr
  u32x4* outer;         // for outer: [tiles][2][tiles of 16 columns][kParts][64]; or nullptr
};
constexpr int kPackThreads = 512, kPackStride = 132;
typedef float PackBuffer[32][kPackStride];

__device__ __forceinline__ void pack_block(const Pack& a, int b, float* s_sum, int stride) {
  const int tid = threadIdx.x, half = b & 1;
  Tile t{0, (b >> 1) * kTileRows, 0, b >> 1};
  if (a.tiles != nullptr) t = a.tiles[b >> 1];
  else t.rows = min(kTileRows, a.T - t.first);
  const int rows = min(32, t.rows - 32 * half), first = t.first + 32 * half, r = a.r;
  if (rows <= 0) return;
  const auto row_of = [&](int i) { return a.list != nullptr ? a.list[first + i] : first + i; };
  if (t.group == a.L) {
    if (a.keep != nullptr)
      for (int o = tid; o < rows * r; o += kPackThreads) a.keep[(size_t)row_of(o / r) * r + o % r] = 0.f;
    return;
  }
  const int chunks = (r + 31) / 32, cols = 32 * chunks;
  const size_t slice = (size_t)a.T * r;
  for (int o = tid; o < 32 * cols / 4; o += kPackThreads) {  // four values
    const int i = o / (cols / 4), j = o % (cols / 4) * 4;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (i < rows && j < r) {
      const size_t at = (size_t)row_of(i) * r + j;
      if (a.vec) {
        for (int s0 = 0; s0 < a.slices; s0 += 8) {
          float4 p[8];
#pragma unroll
          for (int s = 0; s < 8; ++s) p[s] = *reinterpret_cast<const float4*>(a.part + min(s0 + s, a.slices - 1) * slice + at);
#pragma unroll
          for (int s = 0; s < 8; ++s)
            if (s0 + s < a.slices) v.x += p[s].x, v.y += p[s].y, v.z += p[s].z, v.w += p[s].w;
        }
        if (a.keep != nullptr) *reinterpret_cast<float4*>(a.keep + at) = v;
      } else {  // (one slice)
        v.x = a.part[at];
        if (j + 1 < r) v.y = a.part[at + 1];
        if (j + 2 < r) v.z = a.part[at + 2];
        if (j + 3 < r) v.w = a.part[at + 3];
      }
    }
    *reinterpret_cast<float4*>(s_sum + i * stride + j) = v;
  }
  __syncthreads();
  const float scale = a.scale != nullptr ? a.scale[t.group] : 1.f;
  if (a.packed != nullptr)
    for (int o = tid; o < 2 * chunks * 64; o += kPackThreads) {  // lane (row, 8 columns)
      const int l = o & 63, c = (o >> 6) % chunks, h = (o >> 6) / chunks;
      float v[8];
      load8(s_sum + (16 * h + (l & 15)) * stride + 32 * c + 8 * (l >> 4), v);
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] *= scale;
      u32x4* const to = a.packed + ((((size_t)t.at * 4 + 2 * half + h) * chunks + c) * kParts) * 64 + l;
#pragma unroll
      for (int s = 0; s < kParts; ++s) to[s * 64] = take_bf16(v);
    }
  if (a.outer != nullptr) {
    const int tiles = (r + 15) / 16;
    for (int o = tid; o < tiles * 64; o += kPackThreads) {  // lane (column, 8 rows)
      const int l = o & 63, m = o >> 6;
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = scale * s_sum[(8 * (l >> 4) + k) * stride + 16 * m + (l & 15)];
      u32x4* const to = a.outer + ((size_t)t.at * 2 + half) * tiles * kParts * 64 + m * kParts * 64 + l;
#pragma unroll
      for (int s = 0; s < kParts; ++s) to[s * 64] = take_bf16(v);
    }
  }
}

static __global__ __launch_bounds__(kPackThreads) void pack_kernel(Pack a) {
  __shared__ __align__(16) PackBuffer s_sum;
  pack_block(a, blockIdx.x, &s_sum[0][0], kPackStride);
}

// Bytes of both forms for n tiles.
inline size_t packed_bytes(int n, int r) { return (size_t)n * 4 * ceil_div(r, 32) * kParts * 1024; }
inline size_t outer_bytes(int n, int r) { return (size_t)n * 2 * ceil_div(r, 16) * kParts * 1024; }

// ---- expand ------------------------------------------------------------------------------------------------------------------
// A wavefront computes up to 64 rows of 16 NJ columns, 16 rows at a time.  The MFMA's first operand is P, its second M_a; accumulator j of
// lane c stands for column NJ c + j (of fp32 results 4 c + j % 4 of every 64), so that a lane's values of one row are neighbours and the 16
// lanes of a row read and write up to 256 bytes in a row.  M_a's fragments stay in registers; they come through the wavefront's own LDS,
// where they are put as they lie in memory.  The next 16 rows' P and Y are on their way during a step's products.  4096 rows of 4096 columns, bf16 in and out, rank 32: 20.2 us from packed P (3.3 TB/s), 22.4 from sums, where pack_kernel's 4 us are saved.  (All 64 rows of Y on
// their way from the start instead of 16 ahead took more registers and 5 % longer.)
constexpr int kExpandThreads = 256, kExpandWaves = kExpandThreads / kWave;

struct Expand {
  const Tile* tiles;    // nullptr: all rows one group
  const int32_t* list;
  int T, L;
  const u32x4* packed;
  int r;
  const uint16_t* m;    // [L][N][r]
  int N;
  const void* y_in;     // [T][N] or nullptr
  void* y_out;          // [T][N]
  // FROM_SUMS: instead of `packed`, the slices of v's sum, the groups' scales and where v is kept (or nullptr)
  const float* part;
  int slices;
  const float* scale;
  float* keep;
};

// `n` rows without a group: the output is the input.
template <typename YT, int THREADS = kExpandThreads>
__device__ __forceinline__ void copy_rows(const void* y_in, void* y_out, int N, const int32_t* s_rows, int n, int c0, int cols) {
  constexpr int W = 16 / sizeof(YT);
  const YT* in = static_cast<const YT*>(y_in);
  YT* out = static_cast<YT*>(y_out);
  cols = min(cols, N - c0);
  if (in == out) return;
  {
    const int per_row = cols / W, total = n * per_row;
    for (int i0 = threadIdx.x; i0 < total; i0 += 8 * THREADS) {
      u32x4 v[8];
      size_t at[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int i = min(i0 + u * THREADS, total - 1);
        at[u] = (size_t)s_rows[i / per_row] * N + c0 + i % per_row * W;
        v[u] = in != nullptr ? *reinterpret_cast<const u32x4*>(in + at[u]) : u32x4{};
      }
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (i0 + u * THREADS < total) *reinterpret_cast<u32x4*>(out + at[u]) = v[u];
    }
  }
}

constexpr int kExpandCols = kExpandWaves * 16;  // of a workgroup, times NJ

// FROM_SUMS: the workgroup adds v's slices and splits it itself, into s_p (as launch_shrink left them, [slices][T][r]).
template <typename YT, int CH, int NJ, bool FROM_SUMS = false>
__device__ __forceinline__ void expand_tile(const Expand& e, int col_block, int which, int32_t* s_rows, char* s_buf, u32x4* s_p = nullptr) {
  constexpr int BYTES = NJ * (int)sizeof(YT) < 16 ? NJ * (int)sizeof(YT) : 16, W = BYTES / (int)sizeof(YT), UNITS = NJ / W;
  constexpr int COLS = 16 * NJ, U = kTileRows / 16;
  typedef uint32_t unit __attribute__((ext_vector_type(BYTES / 4)));
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, ln = lane & 15, q = lane >> 4;
  Tile tile{0, which * kTileRows, 0, which};
  if (e.tiles != nullptr) tile = e.tiles[which];
  else tile.rows = min(kTileRows, e.T - tile.first);
  if (tile.rows == 0) return;
  if (tid < kTileRows) {
    const int at = tile.first + min(tid, tile.rows - 1);
    s_rows[tid] = e.list != nullptr ? e.list[at] : at;
  }
  __syncthreads();
  if (tile.group == e.L) {
    copy_rows<YT>(e.y_in, e.y_out, e.N, s_rows, tile.rows, col_block * kExpandWaves * COLS, kExpandWaves * COLS);
    if (FROM_SUMS && e.keep != nullptr && col_block == 0)
      for (int i = tid; i < tile.rows * e.r; i += kExpandThreads) e.keep[(size_t)s_rows[i / e.r] * e.r + i % e.r] = 0.f;
    return;
  }
  const int nbase = (col_block * kExpandWaves + wave) * COLS;
  if (!FROM_SUMS && nbase >= e.N) return;
  const int chunks = (e.r + 31) / 32;
  const YT* in = static_cast<const YT*>(e.y_in);
  YT* out = static_cast<YT*>(e.y_out);
  const int c0 = nbase + ln * W;
  unit y[2][4][UNITS];
  u32x4 p[2][CH][kParts];
  // (no load under a condition: the compiler would wait for all loads behind it)
  const unit* const base = in != nullptr ? reinterpret_cast<const unit*>(in) : reinterpret_cast<const unit*>(e.m);
  const int in_last = in != nullptr ? e.N - W : 0;
  const size_t in_stride = in != nullptr ? e.N : 0;
  const auto load = [&](unit(&yy)[4][UNITS], u32x4(&pp)[CH][kParts], int u) {
    if constexpr (!FROM_SUMS) {
      const u32x4* const from = e.packed + ((size_t)tile.at * U + u) * chunks * kParts * 64 + lane;
#pragma unroll
      for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int s = 0; s < kParts; ++s) pp[c][s] = from[(min(c, chunks - 1) * kParts + s) * 64];
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int h = 0; h < UNITS; ++h)
        yy[k][h] = *reinterpret_cast<const unit*>(reinterpret_cast<const YT*>(base) + s_rows[16 * u + 4 * q + k] * in_stride +
                                                  min(c0 + 64 * h, in_last));
  };
  // v's sums first: they are needed first, and loads return in order
  constexpr int PER_ROW = 4 * CH, ITEMS = FROM_SUMS ? kTileRows * PER_ROW / kExpandThreads : 1, SLICES = FROM_SUMS ? 8 : 1;
  float4 sums[ITEMS][SLICES][2];
  if constexpr (FROM_SUMS) {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int item = tid + i * kExpandThreads, j0 = min(item % PER_ROW * 8, e.r - 8);
      const float* const from = e.part + (size_t)s_rows[item / PER_ROW] * e.r + j0;
#pragma unroll
      for (int p = 0; p < SLICES; ++p)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          sums[i][p][h] = *reinterpret_cast<const float4*>(from + (size_t)min(p, e.slices - 1) * e.T * e.r + 4 * h);
    }
  }
  // M_a: 32 columns at a time into LDS, a row's four 16-byte parts rearranged so that both sides meet few bank conflicts
  u32x4 w[CH][NJ];
  char* const s_m = s_buf + wave * COLS * 64;
  const uint16_t* const mr = e.m + (size_t)tile.group * e.N * e.r;
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int i = 0; i < NJ; ++i) {
      const int n = min(nbase + 16 * i + (lane >> 2), e.N - 1), col = 32 * c + 8 * (lane & 3);
      w[c][i] = *reinterpret_cast<const u32x4*>(mr + (size_t)n * e.r + (col < e.r ? col : 0));
    }
  const int last = (tile.rows - 1) / 16;
  load(y[0], p[0], 0);
  __builtin_amdgcn_sched_barrier(0);
  if constexpr (FROM_SUMS) {
    const float scale = e.scale[tile.group];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int item = tid + i * kExpandThreads, row = item / PER_ROW, j0 = item % PER_ROW * 8;
      float v[8] = {};
      if (j0 < e.r) {
#pragma unroll
        for (int p = 0; p < SLICES; ++p) {
          const bool in = p < e.slices;
          const float4 a = sums[i][p][0], b = sums[i][p][1];
          const float more[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
          for (int k = 0; k < 8; ++k) v[k] += in ? more[k] : 0.f;
        }
        if (e.keep != nullptr && col_block == 0 && row < tile.rows) {
          float4* const at = reinterpret_cast<float4*>(e.keep + (size_t)s_rows[row] * e.r + j0);
          at[0] = make_float4(v[0], v[1], v[2], v[3]);
          at[1] = make_float4(v[4], v[5], v[6], v[7]);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] *= scale;
      }
#pragma unroll
      for (int s = 0; s < kParts; ++s)
        s_p[((row / 16 * CH + j0 / 32) * kParts + s) * 64 + j0 % 32 / 8 * 16 + row % 16] = take_bf16(v);
    }
    __syncthreads();
    if (nbase >= e.N) return;
  }
#pragma unroll
  for (int c = 0; c < CH; ++c) {
#pragma unroll
    for (int i = 0; i < NJ; ++i) {  // column n: accumulator and lane
      const int n = 16 * i + (lane >> 2);
      const int j = sizeof(YT) == 2 ? n % NJ : (n >> 6) * 4 + (n & 3), l = sizeof(YT) == 2 ? n / NJ : (n >> 2) & 15;
      const bool zero = 32 * c + 8 * (lane & 3) >= e.r;
      const u32x4 v = w[c][i];
      *reinterpret_cast<u32x4*>(s_m + (j * 16 + l) * 64 + (((lane & 3) ^ (l >> 1 & 3)) * 16)) =
          u32x4{zero ? 0u : v.x, zero ? 0u : v.y, zero ? 0u : v.z, zero ? 0u : v.w};
    }
    wave_fence();
#pragma unroll
    for (int j = 0; j < NJ; ++j) w[c][j] = *reinterpret_cast<const u32x4*>(s_m + (j * 16 + ln) * 64 + ((q ^ (ln >> 1 & 3)) * 16));
    wave_fence();
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (16 * u >= tile.rows) break;
    if (u + 1 < U) load(y[(u + 1) & 1], p[(u + 1) & 1], min(u + 1, last));
    f32x4 acc[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int s = kParts - 1; s >= 0; --s) {  // the small parts first
        const u32x4 a = FROM_SUMS ? s_p[((u * CH + c) * kParts + s) * 64 + lane] : p[u & 1][c][s];
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[j] = mfma(a, w[c][j], acc[j]);
      }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (16 * u + 4 * q + k >= tile.rows) continue;
#pragma unroll
      for (int h = 0; h < UNITS; ++h) {
        if (c0 + 64 * h >= e.N) continue;
        unit o;
#pragma unroll
        for (int i = 0; i < BYTES / 4; ++i) {
          const uint32_t d = in != nullptr ? y[u & 1][k][h][i] : 0u;
          if constexpr (sizeof(YT) == 2) o[i] = pack_bf16x2(bf16_lo(d) + acc[2 * i][k], bf16_hi(d) + acc[2 * i + 1][k]);
          else o[i] = __float_as_uint(__uint_as_float(d) + acc[4 * h + i][k]);
        }
        *reinterpret_cast<unit*>(out + (size_t)s_rows[16 * u + 4 * q + k] * e.N + c0 + 64 * h) = o;
      }
    }
  }
}

template <typename YT, int CH, int NJ, bool FROM_SUMS>
__global__ __launch_bounds__(kExpandThreads, 2) void expand_kernel(Expand e, int n_tiles) {
  __shared__ int32_t s_rows[kTileRows];
  __shared__ u32x4 s_p[FROM_SUMS ? kTileRows / 16 * CH * kParts * 64 : 1];
  __shared__ __align__(16) char s_buf[kExpandCols * NJ * 64];
  const int which = blockIdx.z * gridDim.y + blockIdx.y;
  if (which < n_tiles) expand_tile<YT, CH, NJ, FROM_SUMS>(e, blockIdx.x, which, s_rows, s_buf, s_p);
}

template <typename YT, int CH, int NJ, bool FROM_SUMS>
void launch_expand_kernel(const Expand& e, int n_tiles, hipStream_t s) {
  constexpr int kMaxY = 32768;  // (a grid's y is 16 bits)
  hipLaunchKernelGGL((expand_kernel<YT, CH, NJ, FROM_SUMS>),
                     dim3(ceil_div(e.N, kExpandCols * NJ), n_tiles < kMaxY ? n_tiles : kMaxY, ceil_div(n_tiles, kMaxY)),
                     dim3(kExpandThreads), 0, s, e, n_tiles);
}

// ---- expand by an fp32 matrix --------------------------------------------------------------------------------------------------
// The same where M is fp32 too (the router's weights) and all rows are one group.  P and M are three bf16 parts each, all 24 bits of
// either; of the nine products of parts the three below 2^-23 of the whole are left out, so that the sums are as exact as fp32 products'.
// A wavefront has 16 NJ columns of all 64 rows in its accumulators and takes 32 of M's columns after the other, AHEAD of them on their way at
// once (LOOP: there are more than AHEAD).  P's parts lie in LDS, where the workgroup's four wavefronts share them.  Up to 64 columns come in one
// go, which leaves registers for a third workgroup on a compute unit where it is 32 (2048 columns, one wide, 3000 rows 19.1 us instead of
// 21.1 with the loop's code, one row 7.3 instead of 7.8).
struct ExpandF32 {
  int T;
  const u32x4* packed;   // [tiles][4][chunks of 32 columns][kParts][64]
  int r;
  const uint16_t* m;     // [N][kParts][32 chunks]
  int N;
  const uint16_t* y_in;  // [T][N] or nullptr
  uint16_t* y_out;       // [T][N]
};
constexpr int kF32Fragments = kTileRows / 16 * kParts;  // of P, for 32 columns

template <int NJ, int AHEAD, bool LOOP>
__device__ __forceinline__ void expand_f32_tile(const ExpandF32& e, int col_block, int which, char* s_buf) {
  constexpr int U = kTileRows / 16, ITEMS = kF32Fragments / kExpandWaves;
  static_assert(kF32Fragments % kExpandWaves == 0, "the wavefronts bring as many fragments each");
  typedef uint32_t unit __attribute__((ext_vector_type(NJ / 2)));
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, ln = lane & 15, q = lane >> 4;
  const int first = which * kTileRows, rows = min(kTileRows, e.T - first), chunks = (e.r + 31) / 32;
  const int nbase = (col_block * kExpandWaves + wave) * 16 * NJ, c0 = nbase + NJ * ln;
  u32x4* const s_p = reinterpret_cast<u32x4*>(s_buf);  // two of them in turns
  char* const s_m = s_buf + 2 * kF32Fragments * 1024 + wave * NJ * 1024;
  u32x4 m[AHEAD][kParts][NJ], p[AHEAD][ITEMS];
  const auto load = [&](int at, int c) {
#pragma unroll
    for (int pt = 0; pt < kParts; ++pt)
#pragma unroll
      for (int i = 0; i < NJ; ++i)  // (past the last column: that one again, not stored)
        m[at][pt][i] = *reinterpret_cast<const u32x4*>(
            e.m + ((size_t)min(nbase + 16 * i + (lane >> 2), e.N - 1) * kParts + pt) * 32 * chunks + 32 * c + 8 * (lane & 3));
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int f = i * kExpandWaves + wave;
      p[at][i] = e.packed[((((size_t)which * U + f / kParts) * chunks + c) * kParts + f % kParts) * 64 + lane];
    }
  };
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) load(i, min(i, chunks - 1));
  f32x4 acc[U][NJ];  // from y_in on; without it the same bytes of M again, not used (no load under a condition)
  const bool some = e.y_in != nullptr;
  const uint16_t* const in = some ? e.y_in + (size_t)first * e.N + min(c0, e.N - NJ) : e.m;
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const unit d = *reinterpret_cast<const unit*>(in + (some ? (size_t)min(16 * u + 4 * q + k, rows - 1) * e.N : 0));
#pragma unroll
      for (int j = 0; j < NJ; ++j) acc[u][j][k] = some ? (j & 1 ? bf16_hi(d[j / 2]) : bf16_lo(d[j / 2])) : 0.f;
    }
  for (int first_c = 0; first_c < chunks; first_c += AHEAD) {
#pragma unroll
    for (int at = 0; at < AHEAD; ++at) {
      const int c = first_c + at;
      if (AHEAD > 1 && c >= chunks) break;
      u32x4* const parts = s_p + (c & 1) * kF32Fragments * 64;
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) parts[(i * kExpandWaves + wave) * 64 + lane] = p[at][i];
      u32x4 w[kParts][NJ];
#pragma unroll
      for (int pt = 0; pt < kParts; ++pt) {
#pragma unroll
        for (int i = 0; i < NJ; ++i) {  // column n: accumulator n % NJ of lane n / NJ
          const int n = 16 * i + (lane >> 2), l = n / NJ;
          *reinterpret_cast<u32x4*>(s_m + (n % NJ * 16 + l) * 64 + (((lane & 3) ^ (l >> 1 & 3)) * 16)) = m[at][pt][i];
        }
        wave_fence();
#pragma unroll
        for (int j = 0; j < NJ; ++j) w[pt][j] = *reinterpret_cast<const u32x4*>(s_m + (j * 16 + ln) * 64 + ((q ^ (ln >> 1 & 3)) * 16));
        wave_fence();
      }
      __syncthreads();  // (one is enough: `parts` is written again only after the next one)
      if (LOOP && c + AHEAD < chunks) load(at, c + AHEAD);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (16 * u >= rows) break;
        u32x4 a[kParts];
#pragma unroll
        for (int s = 0; s < kParts; ++s) a[s] = parts[(u * kParts + s) * 64 + lane];
#pragma unroll
        for (int sum = kParts - 1; sum >= 0; --sum)  // the small products first
#pragma unroll
          for (int s = sum; s >= 0; --s)
#pragma unroll
            for (int j = 0; j < NJ; ++j) acc[u][j] = mfma(a[s], w[sum - s][j], acc[u][j]);
      }
    }
    if (!LOOP) break;
  }
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int row = 16 * u + 4 * q + k;
      if (row >= rows || c0 >= e.N) continue;
      unit o;
#pragma unroll
      for (int i = 0; i < NJ / 2; ++i) o[i] = pack_bf16x2(acc[u][2 * i][k], acc[u][2 * i + 1][k]);
      *reinterpret_cast<unit*>(e.y_out + (size_t)(first + row) * e.N + c0) = o;
    }
}

// ---- outer -------------------------------------------------------------------------------------------------------------------
// A wavefront takes 32 rows at a time: lane (c, q) loads 8 neighbouring columns of rows 8 q .. 8 q + 7, a row's 16 lanes 256 bytes in a
// row, and byte permutations turn the eight 16-byte rows into eight column fragments (rows are the sum's index): no trip through
// LDS.  P's fragments come packed in parts.  The wavefronts take every fourth 32 rows; their sums are added in order through LDS,
// one tile of P's columns at a time.  A group of more than `chunk` rows is cut, its pieces' sums go to `part` and join in
// reduce_kernel: which pieces there are follows from the rows alone, so the order of the additions is fixed.  8192 rows of 4096 and 4096
// columns at rank 64: 47 us for 134 MB of Z.  Each column tile reads P's fragments anew (200 MB): 27 us without these loads, 43 with as many of
// them that all read the same 12 KB, so that it is their number that costs, not the way to L2.
struct OuterSide {
  const uint16_t* z;    // [T][cols]
  const u32x4* packed;
  const float* scale;   // per group, or nullptr
  float* out;           // [L][r][cols], or [L][cols][r] if by_column
  float* part;          // the same for each piece of a cut group
  int cols, tiles;      // tiles of 128 columns
  bool by_column;
};
struct Outer {
  const Tile* pieces;   // nullptr: all rows one group
  const int32_t *slots, *slot0, *offsets, *list;
  int T, L;
  OuterSide side[2];
  int r, chunk;         // rows of a piece, a multiple of 32
};

constexpr int kOuterWaves = 4, kOuterThreads = kOuterWaves * 64, kOuterCols = 128, kMaxChunk = 4096;

constexpr int kOuterBytes = kOuterWaves * 16 * (kOuterCols + 4) * 4;

template <int MT>
__device__ __forceinline__ void outer_tile(const Outer& o, int tile_of_cols, int piece, int part_of_r, char* s_buf) {
  static_assert(kOuterBytes >= kMaxChunk * 4, "the rows' numbers lie where the sums are joined later");
  int32_t* const s_rows = reinterpret_cast<int32_t*>(s_buf);
  float(*const red)[16][kOuterCols + 4] = reinterpret_cast<float(*)[16][kOuterCols + 4]>(s_buf);
  const bool second = tile_of_cols >= o.side[0].tiles;
  const OuterSide sd = second ? o.side[1] : o.side[0];
  const int col_tile = second ? tile_of_cols - o.side[0].tiles : tile_of_cols;
  Tile tile{0, piece * o.chunk, 0, piece * (o.chunk / 32)};
  if (o.pieces != nullptr) tile = o.pieces[piece];
  else tile.rows = min(o.chunk, o.T - tile.first);
  if (tile.group < 0) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, c = lane & 15, q = lane >> 4;
  if (o.list != nullptr) {
    for (int i = tid; i < tile.rows; i += kOuterThreads) s_rows[i] = o.list[tile.first + i];
    __syncthreads();
  }
  const int r = o.r, tiles = (r + 15) / 16, m0 = part_of_r * MT, c0 = col_tile * kOuterCols;
  f32x4 acc[MT][8];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const uint16_t* const zc = sd.z + min(c0 + 8 * c, sd.cols - 8);  // columns past the end are computed and not stored
  const int blocks = (tile.rows + 31) / 32;
  const u32x4* const packed = sd.packed + ((size_t)tile.at * tiles + m0) * kParts * 64 + lane;
  const int m_last = min(MT, tiles - m0) - 1;  // (tiles past the last: computed from it again and not stored)
  constexpr int FIRST = MT < 2 ? MT : 2;  // tiles of P's columns whose parts are loaded a block ahead
  u32x4 z[8], p[FIRST][kParts];
  const auto load_z = [&](int b) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int at = min(32 * b + 8 * q + i, tile.rows - 1);  // (past the end: a row of the same group, times 0)
      z[i] = *reinterpret_cast<const u32x4*>(zc + (size_t)(o.list != nullptr ? s_rows[at] : tile.first + at) * sd.cols);
    }
  };
  const auto load_p = [&](u32x4(&v)[kParts], int b, int m) {
#pragma unroll
    for (int s = 0; s < kParts; ++s) v[s] = packed[((size_t)b * tiles + min(m, m_last)) * kParts * 64 + s * 64];
  };
  int b = wave;
  if (b < blocks) {
#pragma unroll
    for (int m = 0; m < FIRST; ++m) load_p(p[m], b, m);
    load_z(b);
  }
  for (; b < blocks; b += kOuterWaves) {
    const int next = min(b + kOuterWaves, blocks - 1);
    u32x4 f[8];
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      uint32_t lo[4], hi[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        lo[i] = __builtin_amdgcn_perm(z[2 * i + 1][d], z[2 * i][d], 0x05040100u);
        hi[i] = __builtin_amdgcn_perm(z[2 * i + 1][d], z[2 * i][d], 0x07060302u);
      }
      f[2 * d] = u32x4{lo[0], lo[1], lo[2], lo[3]};
      f[2 * d + 1] = u32x4{hi[0], hi[1], hi[2], hi[3]};
    }
    // P's columns 32 ahead, the next block's after this one's; Z's rows between them, as loads return in the order they are issued in
#pragma unroll
    for (int m = 0; m < MT; ++m) {
#pragma unroll
      for (int s = 0; s < kParts; ++s)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[m][j] = mfma(p[m % FIRST][s], f[j], acc[m][j]);
      if (m > 0 && m + FIRST == MT) load_z(next);
      load_p(p[m % FIRST], m + FIRST < MT ? b : next, (m + FIRST) % MT);
      if (MT == FIRST && m + 1 == MT) load_z(next);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  const int slot = o.pieces != nullptr ? o.slots[piece] : (o.T > o.chunk ? piece : -1);
  const float scale = sd.scale != nullptr && tile.rows > 0 ? sd.scale[tile.group] : 1.f;  // (without rows: zeros, whatever the scale is)
  float* out = slot >= 0 ? sd.part + (size_t)slot * r * sd.cols : sd.out + (size_t)tile.group * r * sd.cols;
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    if (m0 + m >= tiles) break;
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        *reinterpret_cast<float4*>(&red[wave][4 * q + e][8 * c + 4 * h]) =
            make_float4(acc[m][4 * h][e], acc[m][4 * h + 1][e], acc[m][4 * h + 2][e], acc[m][4 * h + 3][e]);
    __syncthreads();
    if (!sd.by_column) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int jj = 8 * k + (tid >> 5), j = 16 * (m0 + m) + jj, n = (tid & 31) * 4;
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kOuterWaves; ++w) {
          const float4 a = *reinterpret_cast<const float4*>(&red[w][jj][n]);
          sum.x += a.x; sum.y += a.y; sum.z += a.z; sum.w += a.w;
        }
        if (j < r && c0 + n < sd.cols)
          *reinterpret_cast<float4*>(out + (size_t)j * sd.cols + c0 + n) =
              make_float4(sum.x * scale, sum.y * scale, sum.z * scale, sum.w * scale);
      }
    } else {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int n = 64 * k + (tid >> 2), jj = (tid & 3) * 4, j = 16 * (m0 + m) + jj;
        float sum[4] = {};
#pragma unroll
        for (int w = 0; w < kOuterWaves; ++w)
#pragma unroll
          for (int i = 0; i < 4; ++i) sum[i] += red[w][jj + i][n];
        float* at = out + (size_t)(c0 + n) * r + j;
        if (c0 + n < sd.cols) {
          if ((r & 3) == 0) {
            if (j < r) *reinterpret_cast<float4*>(at) = make_float4(sum[0] * scale, sum[1] * scale, sum[2] * scale, sum[3] * scale);
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (j + i < r) at[i] = sum[i] * scale;
          }
        }
      }
    }
  }
}

template <int MT>
__global__ __launch_bounds__(kOuterThreads, 2) void outer_kernel(Outer o) {
  __shared__ __align__(16) char s_buf[kOuterBytes];
  outer_tile<MT>(o, blockIdx.x, blockIdx.y, blockIdx.z, s_buf);
}

// The products of a backward pass in one launch: neither needs the other, so the end of the one is the other's beginning.
// Workgroups are numbered through: outer's (x fastest), then expand's; the two taking turns was slower (the whole pass 115 / 129 us).
// 8192 rows, rank 64, 4096 and 4096 columns: 64.0 us for 201 MB (3.1 TB/s; the sums over rows alone 47); 8192 tokens of 3584, 64 experts
// 51 for 117 MB (23), of which the six products of W_r's and d_logits' parts are 23 GFLOP.
template <int CH, int NJ>
struct ExpandByGroup {
  typedef Expand Args;
  static constexpr int kCols = kExpandCols * NJ, kBytes = kExpandCols * NJ * 64;
  static __device__ __forceinline__ void run(const Args& e, int col_block, int which, int32_t* s_rows, char* s_buf) {
    expand_tile<uint16_t, CH, NJ>(e, col_block, which, s_rows, s_buf);
  }
};
template <int NJ, int AHEAD, bool LOOP>
struct ExpandByF32 {
  typedef ExpandF32 Args;
  static constexpr int kCols = kExpandCols * NJ, kBytes = (2 * kF32Fragments + kExpandWaves * NJ) * 1024;
  static __device__ __forceinline__ void run(const Args& e, int col_block, int which, int32_t*, char* s_buf) {
    expand_f32_tile<NJ, AHEAD, LOOP>(e, col_block, which, s_buf);
  }
};
template <typename EXPAND>
struct Both {
  Outer o;
  typename EXPAND::Args e;
  int outer_x, pieces, outers, expand_x;
};
template <int MT, typename EXPAND>
__global__ __launch_bounds__(kOuterThreads, 2) void both_kernel(Both<EXPAND> a) {
  static_assert(kOuterThreads == kExpandThreads, "one block size");
  __shared__ int32_t s_rows[kTileRows];
  __shared__ __align__(16) char s_buf[EXPAND::kBytes > kOuterBytes ? EXPAND::kBytes : kOuterBytes];
  const int b = blockIdx.x;
  if (b < a.outers) {
    outer_tile<MT>(a.o, b % a.outer_x, b / a.outer_x % a.pieces, b / a.outer_x / a.pieces, s_buf);
  } else {
    EXPAND::run(a.e, (b - a.outers) % a.expand_x, (b - a.outers) / a.expand_x, s_rows, s_buf);
  }
}

// Adds the pieces of cut groups in order.  blockIdx.y: the group; four pieces in flight.
static __global__ __launch_bounds__(256) void reduce_kernel(Outer o) {
  const int g = blockIdx.y;
  const int n = o.pieces != nullptr ? o.offsets[g + 1] - o.offsets[g] : o.T;
  if (n <= o.chunk) return;
  const int slot = o.pieces != nullptr ? o.slot0[g] : 0, pieces = (n + o.chunk - 1) / o.chunk;
  const size_t sizes[2] = {(size_t)o.r * o.side[0].cols, (size_t)o.r * o.side[1].cols};  // (multiples of 8)
  for (size_t i = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4; i < sizes[0] + sizes[1]; i += (size_t)gridDim.x * 1024) {
    const bool second = i >= sizes[0];
    const size_t size = second ? sizes[1] : sizes[0], at = second ? i - sizes[0] : i;
    const float* part = (second ? o.side[1].part : o.side[0].part) + (size_t)slot * size + at;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int p = 0; p < pieces; p += 4) {
      float4 a[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) a[k] = *reinterpret_cast<const float4*>(part + (size_t)min(p + k, pieces - 1) * size);
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (p + k < pieces) sum.x += a[k].x, sum.y += a[k].y, sum.z += a[k].z, sum.w += a[k].w;
    }
    *reinterpret_cast<float4*>((second ? o.side[1].out : o.side[0].out) + (size_t)g * size + at) = sum;
  }
}

// MT columns' tiles of P a workgroup, one at a time where the launch is thin all the same: shorter steps, and what Z's rows are read again for
// comes from L2 (2048 columns, 60 wide, 333 rows 13.2 / 11.5 us, 700 17.5 / 12.5, 3000 (768 workgroups) 27.7 / 30.5).
constexpr int kThin = 256;
// (More workgroups than a grid's x has room for would need more rows than the memory holds.)
template <int MT, typename EXPAND>
void launch_both_tiles(Both<EXPAND> a, int n_tiles, hipStream_t s) {
  a.outers = a.outer_x * a.pieces * ceil_div(a.o.r, 16 * MT);
  hipLaunchKernelGGL((both_kernel<MT, EXPAND>), dim3(a.outers + a.expand_x * n_tiles), dim3(kOuterThreads), 0, s, a);
}
template <int MT, typename EXPAND>
void launch_both(const Outer& o, int pieces, const typename EXPAND::Args& e, int n_tiles, hipStream_t s) {
  const Both<EXPAND> a{o, e, o.side[0].tiles + o.side[1].tiles, pieces, 0, ceil_div(e.N, EXPAND::kCols)};
  if (MT > 1 && a.outer_x * pieces * ceil_div(o.r, 16) <= kThin) launch_both_tiles<1, EXPAND>(a, n_tiles, s);
  else launch_both_tiles<MT, EXPAND>(a, n_tiles, s);
}

template <int MT>
void launch_outer_tiles(const Outer& o, int pieces, hipStream_t s) {
  hipLaunchKernelGGL(outer_kernel<MT>, dim3(o.side[0].tiles + o.side[1].tiles, pieces, ceil_div(o.r, 16 * MT)), dim3(kOuterThreads),
                     0, s, o);
}

inline void launch_outer(const Outer& o, int pieces, hipStream_t s) {
  if (o.r <= 16) launch_outer_tiles<1>(o, pieces, s);
  else if (o.r <= 32) launch_outer_tiles<2>(o, pieces, s);
  else launch_outer_tiles<4>(o, pieces, s);
}

inline void launch_reduce(const Outer& o, hipStream_t s) {
  const int64_t values = (int64_t)o.r * (o.side[0].cols + o.side[1].cols);
  hipLaunchKernelGGL(reduce_kernel, dim3(ceil_div(values, 1024), o.L), dim3(256), 0, s, o);
}

// Rows of a piece: about `want` workgroups for the column tiles there are, 256 rows at least.  The router wants 256: with dx, whose
// workgroups fill the units as well, fewer and longer pieces are a little better, without it worse (512 / 256 / 128, us: with dx 4096 tokens
// of 2048, 60 experts 32.8 / 32.6 / 26.7, 16384 79.4 / 76.3 / 71.5; 8192 of 3584, 64 experts 68.3 / 65.6 / 64.6, of 4096, 8 experts 56.5 /
// 55.3 / 51.2; 256 / 128 without dx 33.0 / 37.6, 28.9 / 34.0 and 20.9 / 23.6 for the last three; the sums are the same with dx and without,
// so one number serves both).  The adapters have two sides and groups of different lengths, which few pieces divide unevenly, and want
// 512 (512 / 256, us, 4096 x 4096: 8192 rows of 4, rank 16 76.5 / 81.9, of 8, rank 64 118 / 114, 4096 of 4, rank 64 74.5 / 67.2).  Few rows
// are not cut, which saves the launch that adds the pieces: up to 512 of one group for a P of up to 32 columns, 1024 of a wider one (2048
// columns, cut / not, us: 30 wide, 600 rows 11.7 / 11.3, 800 12.5 / 12.8; 60 wide, 600 15.5 / 11.9, 1024 17.3 / 14.9, 2000 20.3 / 22.7); twice
// as many of several groups, among which they are seldom all one's (4 groups, 64 wide, 2000 rows 36.0 / 31.7, 4096 columns 49.9 / 39.5; all
// of one group 35.5 / 46.7, 4096 columns 48.1 / 50.4).
inline int outer_chunk(int T, int L, int tiles, int r, int want) {
  const int uncut = (r <= 32 ? 512 : 1024) * (L > 1 ? 2 : 1);
  if (T <= uncut) return uncut;
  const int64_t chunk = ((int64_t)T * tiles * ceil_div(r, 64) / want + 255) / 256 * 256;
  return chunk < 256 ? 256 : (chunk > kMaxChunk ? kMaxChunk : (int)chunk);
}

}  // namespace skinny
}  // namespace moe
