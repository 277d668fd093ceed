// tg_project: a shared projection and the low-rank adapters of many cameras, y = x w^T + the
// adapter's scale_g (x a_g^T) b_g^T (low-rank adaptation, Hu et al. 2021, one adapter a token).
//
// Two launches. With many tokens:
//  1. shrink: h[t] = scale_g x[t] a_g^T for the tokens that have an adapter, in binary32, and as
//     two values of the type whose sum is h (the first rounded, the second what that rounding
//     left): 22 bits of binary16, 16 of bfloat16. In binary16 a row of smaller or larger numbers
//     is first brought near 2^13 by a power of two: below 2^-14 bits would be lost, and above 2^16
//     all.
//  2. the product: tiles of x and w go through LDS to the matrix instructions. An adapter of the
//     tile's tokens is some more steps of the same loop, with the two values of h in the place of
//     x, 0 for tokens of other adapters, and b_g in the place of w: the joint takes no further
//     registers and no work of its own, but that in binary16 a token's sums take on the power of
//     two of its row of h before, and lose it after.
// With few tokens, where launches and loads are what takes the time:
//  1. tiles of x and w with k cut over workgroups, so that every CU has a share of w to read,
//     and beside them one workgroup a token for its row of h;
//  2. finish: the cuts are added up, and each token's adapter to them.
// 0 times an infinite b_g, or a row of h past what its power of two can bring back, would leave NaN
// at tokens it does not belong to, or in the place of a number. Sums that are not finite at the
// end of a tile with adapters are therefore formed again one by one, from binary32 h and the
// token's own adapter.
// Results lie transposed in the registers (a lane holds 4 outputs of one token), so that stores
// are contiguous and a token's adapter belongs to the lane.
// The product is bound by how fast tiles reach LDS (about 20 bytes a cycle and CU in every shape,
// matrix units at work 65 % of the time with the largest tile) and, with few tokens, by reading w
// and the two launches. bfloat16, adapters in runs: 25,600 x 4,096, k 4,096, rank 32: 0.79 ms,
// 1.1 PFLOP/s, of which 0.06 for h; without adapters 0.70 (a library's product 0.61). 6,400 x
// 1,536, k 1,024, rank 16: 39 us, 7 of them for h, without adapters 26 (31). 8 x 1,536, k 1,024,
// rank 8: 8 us.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <cstdint>

#include "tg.h"
#include "token_math.h"

namespace {

using namespace tok;

constexpr int kMaxStride = 1 << 22;

struct ProjectParams {
  const void *x, *w, *a, *b;
  const int32_t *adapter;
  const float *scale;
  void *y;
  int64_t x_stride, w_stride, y_stride;
  int32_t n_tokens, k, n, n_adapters, rank;
  int32_t pad_rank;  // 16, 32 or 64
  int32_t b_apart;   // rows of b lie on 4-byte boundaries, which loads to LDS ask for: 0, else 1
  int32_t b_rank;    // values of a row of b: rank, or pad_rank when it has been laid out anew
  void *h;           // [n_tokens][2][pad_rank] of the type
  float *h32;        // [n_tokens][pad_rank]
  float *h_up;       // [n_tokens]: the power of two that h has been multiplied by, in binary16
  int32_t gather;    // adapters are added by add_gathered
  int32_t b_whole;   // all of b is within the reach of one buffer
  float *part;       // [splits][n_tokens][part_stride]: sums over a cut of k
  int32_t part_stride, splits, low_blocks;
  int32_t tiles_t, tiles_n;
};

__device__ __forceinline__ int adapter_of(const ProjectParams &P, int t) {
  if (!P.adapter || t >= P.n_tokens) return -1;
  const int g = P.adapter[t];
  return g >= 0 && g < P.n_adapters ? g : -1;
}

// ------------------------------------------------------------------------------- shrink

constexpr int kShrinkThreads = 512;
constexpr int kShrinkWaves = kShrinkThreads / 64;

// One token's row of h as the product wants it. `v[f]`: h of rank 16 f + r0, of the 16 threads
// (r0 = 0 .. 15) of the token; ranks past the last are 0.
template <int kType, int kFrags>
__device__ __forceinline__ void keep_h(const ProjectParams &P, int t, float (&v)[kFrags], int r0) {
  typedef typename Num<kType>::E E;
  E *h = static_cast<E *>(P.h) + int64_t(t) * 2 * P.pad_rank;
  float *h32 = P.h32 + int64_t(t) * P.pad_rank;
  float up = 1.0f;
  if constexpr (kType == TG_F16) {
    float most = 0.0f;
#pragma unroll
    for (int f = 0; f < kFrags; ++f) most = fmaxf(most, fabsf(v[f]));
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor(most, o));
    // Rows with a largest from 2^-3 to 2^15 have their 22 bits as they are. Up to 2^60 either way:
    // sums of binary16 products stay far from binary32's ends, and h below 2^-47 adds less than
    // half of binary16's smallest number to any result.
    const int e = static_cast<int>(__builtin_bit_cast(uint32_t, most) >> 23) - 127;
    if (e < -3 || e >= 15)
      up = __builtin_bit_cast(float, (min(max(13 - e, -60), 60) + 127) << 23);
    if (r0 == 0) P.h_up[t] = up;
  }
#pragma unroll
  for (int f = 0; f < kFrags; ++f) {
    const float w = v[f] * up;
    const E hi = static_cast<E>(w);
    h32[f * 16 + r0] = v[f];
    h[f * 16 + r0] = hi;
    h[P.pad_rank + f * 16 + r0] = static_cast<E>(w - static_cast<float>(hi));
  }
}

// 16 kTok tokens a workgroup, kFrags x 16 ranks, k cut over the waves. The distinct adapters of
// the tokens are dealt out over gridDim.y workgroups.
template <int kType, int kFrags, int kTok>
__global__ __launch_bounds__(kShrinkThreads) void shrink_kernel(const ProjectParams P) {
  typedef Num<kType> N;
  typedef typename N::E E;
  typedef typename N::V8 V8;
  constexpr int kAhead = kTok * (kFrags + 1) <= 4 ? 4 : 2;  // steps whose loads are under way
  __shared__ float part[kShrinkWaves][kFrags * 16][17];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, quad = lane >> 4;
  const int t0 = blockIdx.x * 16 * kTok;
  const E *x[kTok];
  int mine[kTok];
#pragma unroll
  for (int i = 0; i < kTok; ++i) {
    const int t = t0 + 16 * i + col;
    mine[i] = adapter_of(P, t);
    x[i] = static_cast<const E *>(P.x) + int64_t(min(t, P.n_tokens - 1)) * P.x_stride;
  }
  f32x4 sum[kTok][kFrags] = {};
  uint64_t done[kTok] = {}, own[kTok] = {};  // tokens whose adapter has had its turn, and here
  int turn = -1;
  for (;;) {
    // the first token that waits names the adapter; the same in every wave
    int g = -1;
#pragma unroll
    for (int i = kTok - 1; i >= 0; --i) {
      const uint64_t left = __ballot(mine[i] >= 0) & 0xFFFF & ~done[i];
      if (left) g = __builtin_amdgcn_readlane(mine[i], __builtin_ctzll(left));
    }
    if (g < 0) break;
    uint64_t has[kTok];
#pragma unroll
    for (int i = 0; i < kTok; ++i) {
      has[i] = __ballot(mine[i] == g) & 0xFFFF;
      done[i] |= has[i];
    }
    if (++turn % gridDim.y != blockIdx.y) continue;
#pragma unroll
    for (int i = 0; i < kTok; ++i) own[i] |= has[i];
    f32x4 acc[kTok][kFrags] = {};
    const E *a = static_cast<const E *>(P.a) + int64_t(g) * P.rank * P.k;
    const E *row[kFrags];
#pragma unroll
    for (int f = 0; f < kFrags; ++f) row[f] = a + int64_t(min(f * 16 + col, P.rank - 1)) * P.k;
    for (int k0 = wave * 32; k0 < P.k; k0 += kAhead * kShrinkWaves * 32) {
      V8 av[kAhead][kFrags], xv[kAhead][kTok];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int k = k0 + u * kShrinkWaves * 32 + quad * 8;
        const bool in = k < P.k;
#pragma unroll
        for (int f = 0; f < kFrags; ++f) {
          av[u][f] = V8{};
          if (in) av[u][f] = *reinterpret_cast<const V8 *>(row[f] + k);
        }
#pragma unroll
        for (int i = 0; i < kTok; ++i) {
          xv[u][i] = V8{};
          if (in && has[i]) xv[u][i] = *reinterpret_cast<const V8 *>(x[i] + k);
        }
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
#pragma unroll
        for (int i = 0; i < kTok; ++i)
#pragma unroll
          for (int f = 0; f < kFrags; ++f) acc[i][f] = N::mfma16(av[u][f], xv[u][i], acc[i][f]);
    }
#pragma unroll
    for (int i = 0; i < kTok; ++i)
      if (mine[i] == g) {
#pragma unroll
        for (int f = 0; f < kFrags; ++f) sum[i][f] = acc[i][f];
      }
  }
  if (turn < static_cast<int>(blockIdx.y)) return;  // no adapter fell to this workgroup
  const int tok = threadIdx.x >> 4, r0 = threadIdx.x & 15;  // 16 threads a token
#pragma unroll
  for (int i = 0; i < kTok; ++i) {
    if (!own[i]) continue;
    __syncthreads();
#pragma unroll
    for (int f = 0; f < kFrags; ++f)
#pragma unroll
      for (int r = 0; r < 4; ++r) part[wave][f * 16 + quad * 4 + r][col] = sum[i][f][r];
    __syncthreads();
    if (tok >= 16 || !(own[i] >> tok & 1)) continue;
    const int t = t0 + 16 * i + tok;
    const float scale = P.scale[adapter_of(P, t)];
    float v[kFrags];
#pragma unroll
    for (int f = 0; f < kFrags; ++f) {
      v[f] = 0.0f;
#pragma unroll
      for (int w = 0; w < kShrinkWaves; ++w) v[f] += part[w][f * 16 + r0][tok];
      v[f] = f * 16 + r0 < P.rank ? v[f] * scale : 0.0f;
    }
    keep_h<kType, kFrags>(P, t, v, r0);
  }
}

// 4 ranks a wave of one token's row of h, from rank r0 on, by a workgroup of 4 waves: rows of x
// and a are read as they lie.
constexpr int kTokenRanks = 16;
template <int kType, int kWaves>
__device__ __forceinline__ void shrink_token(const ProjectParams &P, int t, int r0) {
  typedef typename Num<kType>::E E;
  typedef typename Num<kType>::V8 V8;
  static_assert(kWaves * 4 == kTokenRanks, "4 ranks a wave");
  constexpr int kAhead = 4;  // loads of a row under way
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = adapter_of(P, t);
  if (g < 0) return;  // nothing reads h of a token without an adapter
  const E *x = static_cast<const E *>(P.x) + t * P.x_stride;
  const E *a = static_cast<const E *>(P.a) + int64_t(g) * P.rank * P.k;
  const float scale = P.scale[g];
  r0 += wave * 4;
  float sum[4] = {};
  for (int k = lane * 8; k < P.k; k += kAhead * 512) {
    V8 xv[kAhead] = {}, av[kAhead][4] = {};
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (k + u * 512 < P.k) {
        xv[u] = *reinterpret_cast<const V8 *>(x + k + u * 512);
#pragma unroll
        for (int r = 0; r < 4; ++r)
          av[u][r] = *reinterpret_cast<const V8 *>(a + int64_t(min(r0 + r, P.rank - 1)) * P.k + k +
                                                   u * 512);
      }
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int i = 0; i < 8; ++i)
          sum[r] = __builtin_fmaf(static_cast<float>(av[u][r][i]), static_cast<float>(xv[u][i]),
                                  sum[r]);
  }
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    sum[r] = wave_sum(sum[r]);
    if (lane == 0)
      P.h32[int64_t(t) * P.pad_rank + r0 + r] = r0 + r < P.rank ? sum[r] * scale : 0.0f;
  }
}

template <int kType, int kFrags>
void launch_shrink_rank(const ProjectParams &P, hipStream_t s) {
  const int most = P.n_adapters < 16 ? P.n_adapters : 16;
  if (P.n_tokens < 8192)
    hipLaunchKernelGGL((shrink_kernel<kType, kFrags, 1>),
                       dim3((P.n_tokens + 15) / 16, P.n_tokens < 1024 ? most : (most + 3) / 4),
                       dim3(kShrinkThreads), 0, s, P);
  else
    hipLaunchKernelGGL((shrink_kernel<kType, kFrags, 4>),
                       dim3((P.n_tokens + 63) / 64, (most + 3) / 4), dim3(kShrinkThreads), 0, s,
                       P);
}

template <int kType>
void launch_shrink(const ProjectParams &P, hipStream_t s) {
  switch (P.pad_rank / 16) {
    case 1: return launch_shrink_rank<kType, 1>(P, s);
    case 2: return launch_shrink_rank<kType, 2>(P, s);
    default: return launch_shrink_rank<kType, 4>(P, s);
  }
}

// ---------------------------------------------------------------------------- the product

// 8 values of b_g's row j from rank r on, zero past the rank and past the last output. Rows may
// start anywhere: the 16 bytes are loaded as they lie, into the next row where the rank ends
// inside, and one by one where that would be past the last row.
template <int kType>
__device__ __forceinline__ typename Num<kType>::V8 b_chunk(const ProjectParams &P, int g, int j,
                                                            int r) {
  typedef typename Num<kType>::E E;
  typedef typename Num<kType>::V8 V8;
  V8 v = {};
  if (j >= P.n || r >= P.b_rank) return v;
  const int64_t at = (int64_t(g) * P.n + j) * P.b_rank + r;
  const E *b = static_cast<const E *>(P.b) + at;
  if (at + 8 <= int64_t(P.n_adapters) * P.n * P.b_rank) {
    __builtin_memcpy(&v, b, sizeof(v));
#pragma unroll
    for (int i = 1; i < 8; ++i)
      if (r + i >= P.b_rank) v[i] = static_cast<E>(0.0f);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (r + i < P.b_rank) v[i] = b[i];
  }
  return v;
}

// Adds b_g h[t] to a wave's results: acc[j][i] holds outputs n0 + 16 j + 4 (lane / 16) .. of
// token t0 + 16 i + lane % 16. Each lane takes its own token's adapter: the time does not hang on
// how many there are, and all loads are independent.
template <int kType, int kFn, int kFt>
__device__ __forceinline__ void add_gathered(const ProjectParams &P, int t0, int n0,
                                             f32x4 (&acc)[kFn][kFt]) {
  typedef typename Num<kType>::V8 V8;
  const int lane = threadIdx.x & 63, col = lane & 15, quad = lane >> 4;
#pragma unroll
  for (int i = 0; i < kFt; ++i) {
    const int t = t0 + 16 * i + col;
    const int g = adapter_of(P, t);
    if (g < 0) continue;
    const f32x4 *h = reinterpret_cast<const f32x4 *>(P.h32 + int64_t(t) * P.pad_rank);
    for (int r0 = 0; r0 < P.rank; r0 += 16) {
#pragma unroll
      for (int r = r0; r < r0 + 16; r += 8) {
        const f32x4 h0 = h[r / 4], h1 = h[r / 4 + 1];
#pragma unroll
        for (int j = 0; j < kFn; ++j)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const V8 b = b_chunk<kType>(P, g, n0 + 16 * j + 4 * quad + q, r);
#pragma unroll
            for (int e = 0; e < 8; ++e)
              acc[j][i][q] = __builtin_fmaf(static_cast<float>(b[e]), e < 4 ? h0[e & 3] : h1[e & 3],
                                            acc[j][i][q]);
          }
      }
    }
  }
}

// One result from the formula. A sum that is NaN stays so, whatever follows: 25,600 x 4,096, k
// 4,096, all results NaN by the first value of x 1.4 ms for 0.8; all infinite 128 ms.
template <int kType>
__device__ __forceinline__ float strict_value(const void *x, const void *w, int k,
                                                        const float *h, const void *b, int rank) {
  typedef typename Num<kType>::E E;
  typedef typename Num<kType>::V8 V8;
  float sum = 0.0f;
  for (int i = 0; i < k && sum == sum; i += 8) {
    const V8 xv = *reinterpret_cast<const V8 *>(static_cast<const E *>(x) + i);
    const V8 wv = *reinterpret_cast<const V8 *>(static_cast<const E *>(w) + i);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      sum = __builtin_fmaf(static_cast<float>(xv[e]), static_cast<float>(wv[e]), sum);
  }
  for (int r = 0; r < rank && sum == sum; ++r)
    sum = __builtin_fmaf(h[r], static_cast<float>(static_cast<const E *>(b)[r]), sum);
  return sum;
}

// Forms those of a wave's results again that are not finite (they have been stored).
template <int kType, int kFn, int kFt>
__device__ __forceinline__ void mend(const ProjectParams &P, int t0, int n0,
                                     const f32x4 (&acc)[kFn][kFt]) {
  typedef typename Num<kType>::E E;
  const int lane = threadIdx.x & 63, col = lane & 15, quad = lane >> 4;
  bool fine = true;
  uint32_t bad[(kFn * kFt * 4 + 31) / 32] = {};
#pragma unroll
  for (int j = 0; j < kFn; ++j)
#pragma unroll
    for (int i = 0; i < kFt; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) fine = fine && fabsf(acc[j][i][q]) < INFINITY;
  if (__ballot(!fine) == 0) return;
#pragma unroll
  for (int j = 0; j < kFn; ++j)
#pragma unroll
    for (int i = 0; i < kFt; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int at = (j * kFt + i) * 4 + q;
        bad[at / 32] |= fabsf(acc[j][i][q]) < INFINITY ? 0u : 1u << (at % 32);
      }
#pragma unroll
  for (int word = 0; word < (kFn * kFt * 4 + 31) / 32; ++word)
    for (uint32_t left = bad[word]; left; left &= left - 1) {
      const int at = word * 32 + __builtin_ctz(left);
      const int t = t0 + 16 * (at / 4 % kFt) + col;
      const int n = n0 + 16 * (at / 4 / kFt) + 4 * quad + at % 4;
      if (t >= P.n_tokens || n >= P.n) continue;
      const int g = adapter_of(P, t);
      const float v = strict_value<kType>(
          static_cast<const E *>(P.x) + t * P.x_stride, static_cast<const E *>(P.w) + n * P.w_stride,
          P.k, P.h32 + int64_t(t) * P.pad_rank,
          static_cast<const E *>(P.b) + (int64_t(max(g, 0)) * P.n + n) * P.b_rank,
          g < 0 ? 0 : P.rank);
      static_cast<E *>(P.y)[t * P.y_stride + n] = static_cast<E>(v);
    }
}

// The distinct adapters among ids[0 .. kT), as list; returns how many. One id a thread, the whole
// workgroup takes part. Neighbours of one adapter are folded first.
template <int kT, int kWaves>
__device__ __forceinline__ int distinct(const int *ids, int *heads, int *list, int *counts) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  auto compact = [&](bool keep, int value, int *to) {
    const uint64_t all = __ballot(keep);
    if (lane == 0) counts[wave] = __popcll(all);
    __syncthreads();
    int before = 0, total = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      if (w < wave) before += counts[w];
      total += counts[w];
    }
    if (keep) to[before + __popcll(all & ((1ull << lane) - 1))] = value;
    __syncthreads();
    return total;
  };
  const int mine = tid < kT ? ids[tid] : -1;
  const int n = compact(mine >= 0 && (tid == 0 || ids[tid - 1] != mine), mine, heads);
  const int head = tid < n ? heads[tid] : -1;
  bool first = tid < n;
  for (int i = 0; i < n - 1; ++i) first = first && (i >= tid || heads[i] != head);
  return __builtin_amdgcn_readfirstlane(compact(first, head, list));
}

template <int kType, int kFn, int kFt>
__device__ __forceinline__ void store(const ProjectParams &P, int t0, int n0,
                                      const f32x4 (&acc)[kFn][kFt]) {
  typedef typename Num<kType>::E E;
  typedef typename Num<kType>::V4 V4;
  const int lane = threadIdx.x & 63, col = lane & 15, quad = lane >> 4;
#pragma unroll
  for (int i = 0; i < kFt; ++i) {
    const int t = t0 + 16 * i + col;
    if (t >= P.n_tokens) continue;
    E *row = static_cast<E *>(P.y) + int64_t(t) * P.y_stride;
#pragma unroll
    for (int j = 0; j < kFn; ++j) {
      const int n = n0 + 16 * j + 4 * quad;
      const V4 v = __builtin_convertvector(acc[j][i], V4);
      if (n + 3 < P.n) {  // as they lie: rows may start anywhere
        __builtin_memcpy(row + n, &v, sizeof(v));
      } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (n + r < P.n) row[n + r] = v[r];
      }
    }
  }
}

// A tile of kT tokens x kN outputs, kWt x kWn waves, 64 values of k a step, kStages steps of
// loads under way. The next 32 values' operands are read from LDS while these are multiplied, so
// that the matrix units have work across the barrier; the buffer of step s is free for step
// s + kStages behind the barrier at the end of it, since its operands are in registers by then.
// Rows of a tile lie in LDS as 8 chunks of 16 bytes, in an order that serves the operands' reads
// (one chunk of 16 rows) best: 156 bytes a cycle and CU measured, where (row / 4) in the place of
// (row / 2) gives 116 and no change of order 123.
constexpr int kBK = 64;
__device__ __forceinline__ int place_of(int row, int c) { return c ^ ((row >> 1) & 7); }

// Which tile a workgroup takes: workgroups go round the 8 XCDs, so each XCD gets a run of tiles
// of its own, in blocks of kGroup token tiles by all output tiles, whose operands its L2 shares.
constexpr int kXcds = 8, kGroup = 4;
__device__ __forceinline__ void tile_of(int id, int tiles_t, int tiles_n, int &tt, int &tn) {
  const int total = tiles_t * tiles_n;
  const int each = total / kXcds, more = total % kXcds, x = id % kXcds;
  const int k = x * each + min(x, more) + id / kXcds;
  const int per = kGroup * tiles_n, g = k / per, in = k - g * per;
  const int rows = min(kGroup, tiles_t - g * kGroup);
  tt = g * kGroup + in % rows;
  tn = in / rows;
}

template <int kType, int kT, int kN, int kWt, int kWn, int kStages, bool kCut>
__global__ __launch_bounds__(kWt *kWn * 64, 2) void project_kernel(const ProjectParams P) {
  typedef Num<kType> N;
  typedef typename N::E E;
  typedef typename N::V8 V8;
  constexpr int kWaves = kWt * kWn, kFt = kT / kWt / 16, kFn = kN / kWn / 16;
  constexpr int kChunks = kBK / 8, kRows = kT + kN, kPer = 64 / kChunks;  // rows of one load
  constexpr int kLoads = kRows / kPer / kWaves;
  static_assert(kLoads * kPer * kWaves == kRows && kT % kPer == 0, "whole loads");
  __shared__ __attribute__((aligned(16))) E tile[kStages][kRows * kBK];
  __shared__ int s_id[kT], s_heads[kT], s_list[kT], s_counts[kWaves];
  __shared__ float s_up[kType == TG_F16 && !kCut ? kT : 1];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, quad = lane >> 4;
  int tt, tn, cut = 0;
  if constexpr (kCut) {
    int id = blockIdx.x;
    if (id < P.low_blocks)
      return shrink_token<kType, kWaves>(P, id % P.n_tokens, id / P.n_tokens * kTokenRanks);
    id -= P.low_blocks;
    cut = id % P.splits;
    id /= P.splits;
    tt = id % P.tiles_t;
    tn = id / P.tiles_t;
  } else {
    tile_of(blockIdx.x, P.tiles_t, P.tiles_n, tt, tn);
  }
  const int t0 = tt * kT, n0 = tn * kN;
  const int xr = min(kT, P.n_tokens - t0), wr = min(kN, P.n - n0);
  const auto xb = buffer(static_cast<const E *>(P.x) + t0 * P.x_stride,
                         static_cast<uint32_t>(((xr - 1) * P.x_stride + P.k) * 2));
  const auto wb = buffer(static_cast<const E *>(P.w) + n0 * P.w_stride,
                         static_cast<uint32_t>(((wr - 1) * P.w_stride + P.k) * 2));
  // load i of a wave covers kPer rows; rows past the tensor are not read. A lane's chunk is the
  // same in all loads, since their rows are 4 kPer apart or more.
  static_assert(kWaves * kPer % 16 == 0, "rows of one lane");
  const int chunk = place_of(wave * kPer + lane / kChunks, lane % kChunks);
  uint32_t at[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int row = (i * kWaves + wave) * kPer + lane / kChunks;
    at[i] = row < kT ? static_cast<uint32_t>((row * P.x_stride + chunk * 8) * 2)
                     : static_cast<uint32_t>(((row - kT) * P.w_stride + chunk * 8) * 2);
    if (row < kT ? row >= xr : row - kT >= wr) at[i] = kNowhere;
  }
  const int all_steps = (P.k + kBK - 1) / kBK;
  int s0 = 0, main_steps = all_steps;
  if constexpr (kCut) {
    const int each = (all_steps + P.splits - 1) / P.splits;
    s0 = cut * each;
    main_steps = min(each, all_steps - s0);  // the host leaves no cut empty
  }
  const int k_end = min(P.k, (s0 + main_steps) * kBK);
  int steps = main_steps;  // and then the adapters' steps
  // every step's loads are issued, past the last one too, so that they can be counted
  auto fetch = [&](int s) {
    const int k0 = (s0 + s) * kBK;
    const bool past = k0 + chunk * 8 >= k_end;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int first = (i * kWaves + wave) * kPer;
      load_lds(first < kT ? xb : wb, &tile[s % kStages][first * kBK], past ? kNowhere : at[i],
               static_cast<uint32_t>(k0) * 2);
    }
  };
  // values of k that an adapter has of the steps: whole steps, or part of one that others share,
  // where one buffer holds all of b
  const int wide = 2 * P.pad_rank;
  const int slot = P.b_whole ? wide : (wide + kBK - 1) / kBK * kBK;
  const int slot_log2 = 31 - __builtin_clz(slot);
  int n_low = 0;  // adapters in this tile
  auto fetch_low = [&](int s) {
    const int at_k = (s - main_steps) * kBK + chunk * 8;
    const int a = at_k >> slot_log2, e = at_k & (slot - 1), r = e & (P.pad_rank - 1);
    const bool in = a < n_low && e < wide;
    const int g = in ? s_list[a] : 0;
    // the adapter whose b the buffer starts at: with whole steps each, all lanes' of the step
    const int a0 = (s - main_steps) * kBK >> slot_log2;
    const int g0 = P.b_whole || a0 >= n_low ? 0 : __builtin_amdgcn_readfirstlane(s_list[a0]);
    const auto hb = buffer(static_cast<const E *>(P.h) + int64_t(t0) * 2 * P.pad_rank,
                           static_cast<uint32_t>(xr) * 4 * P.pad_rank);
    const auto bb =
        buffer(static_cast<const E *>(P.b) + int64_t(g0) * P.n * P.b_rank,
               static_cast<uint32_t>(P.b_whole ? P.n_adapters : 1) * P.n * P.b_rank * 2);
    const uint32_t from = static_cast<uint32_t>(g - g0) * P.n + n0 - kT;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int first = (i * kWaves + wave) * kPer, row = first + lane / kChunks;
      uint32_t off = kNowhere;
      if (first < kT) {
        if (in && s_id[row] == g) off = static_cast<uint32_t>((row * 2 * P.pad_rank + e) * 2);
      } else if (in && r < P.rank && n0 + row - kT < P.n) {
        off = ((from + row) * P.b_rank + r) * 2;
      }
      load_lds(first < kT ? hb : bb, &tile[s % kStages][first * kBK], off, 0);
    }
  };
  f32x4 acc[kFn][kFt] = {};
  const int wt = (wave % kWt) * (kT / kWt), wn = (wave / kWt) * (kN / kWn);
  struct Operands {  // of 32 values of k
    V8 x[kFt], w[kFn];
  };
  auto read = [&](Operands &o, int s, int ks) {
    const E *m = tile[s % kStages];
#pragma unroll
    for (int i = 0; i < kFt; ++i) {
      const int row = wt + 16 * i + col;
      o.x[i] = *reinterpret_cast<const V8 *>(m + row * kBK + place_of(row, ks * 4 + quad) * 8);
    }
#pragma unroll
    for (int j = 0; j < kFn; ++j) {
      const int row = kT + wn + 16 * j + col;
      o.w[j] = *reinterpret_cast<const V8 *>(m + row * kBK + place_of(row, ks * 4 + quad) * 8);
    }
  };
  auto multiply = [&](const Operands &o) {
#pragma unroll
    for (int j = 0; j < kFn; ++j)
#pragma unroll
      for (int i = 0; i < kFt; ++i) acc[j][i] = N::mfma16(o.w[j], o.x[i], acc[j][i]);
  };
  // the scheduler would put the reads at the end, where the products after them wait for them
  auto interleave = [&](bool loads) {
    constexpr int kReads = kFt + kFn, kMul = kFt * kFn;
#pragma unroll
    for (int i = 0; i < kReads; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, kMul / kReads, 0);
      if (loads && i < kLoads) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
    }
  };
  // `now` has the first 32 values of step s, and is left with those of step s + 1
  auto step = [&](int s, Operands &now, Operands &then, bool low) {
    read(then, s, 1);
    multiply(now);
    interleave(false);
    wait_and_meet<(kStages - 2) * kLoads>();  // step s + 1 is here, step s in registers
    if (low && s + kStages >= main_steps) fetch_low(s + kStages);
    else fetch(s + kStages);
    read(now, s + 1, 0);
    multiply(then);
    interleave(true);
  };
  // steps of a small tile are short, so that they wait for their loads: where there are many they
  // are gathered, which takes about as long as pad_rank / 4 of them
  bool gather = P.adapter && P.gather;
  const bool steps_low = !kCut && P.adapter && !P.gather;
  int id = -1;
  float up = 1.0f;
  if (steps_low && threadIdx.x < kT) {
    if (kType == TG_F16 && t0 + threadIdx.x < P.n_tokens) up = P.h_up[t0 + threadIdx.x];
    id = adapter_of(P, t0 + threadIdx.x);
  }
  const int begun = steps_low ? min(main_steps, kStages) : kStages;
  for (int s = 0; s < begun; ++s) fetch(s);
  if (steps_low) {
    if (threadIdx.x < kT) {
      s_id[threadIdx.x] = id;
      if (kType == TG_F16) s_up[threadIdx.x] = id < 0 ? 1.0f : up;
    }
    __syncthreads();
    n_low = distinct<kT, kWaves>(s_id, s_heads, s_list, s_counts);
    const int more = (n_low * slot + kBK - 1) / kBK;
    gather = kFt * kFn <= 4 && more * 4 > P.pad_rank;
    if (!gather) steps += more;
    for (int s = begun; s < kStages; ++s) fetch_low(s);
  }
  wait_and_meet<(kStages - 1) * kLoads>();
  Operands a, b;
  read(a, 0, 0);
  int s = 0;
  for (; s + kStages < main_steps; ++s) step(s, a, b, false);
  // a token's sums times the power of two of its row of h, and back (the exponent negated)
  auto scale = [&](bool back) {
    uint32_t up[kFt];
    bool any = false;
#pragma unroll
    for (int i = 0; i < kFt; ++i) {
      up[i] = __builtin_bit_cast(uint32_t, s_up[wt + 16 * i + col]);
      any = any || up[i] != 0x3F800000u;
    }
    if (!__ballot(any)) return;
#pragma unroll
    for (int i = 0; i < kFt; ++i) {
      const float by = __builtin_bit_cast(float, back ? 0x7F000000u - up[i] : up[i]);
#pragma unroll
      for (int j = 0; j < kFn; ++j) acc[j][i] *= by;
    }
  };
  for (; s < steps; ++s) {
    if constexpr (kType == TG_F16 && !kCut) {
      if (s == main_steps) scale(false);
    }
    step(s, a, b, steps_low);
  }
  if constexpr (kType == TG_F16 && !kCut) {
    if (steps > main_steps) scale(true);
  }
  wait_loads();  // LDS belongs to the next workgroup from here on
  if constexpr (kCut) {
    float *to = P.part + int64_t(cut) * P.n_tokens * P.part_stride;
#pragma unroll
    for (int i = 0; i < kFt; ++i) {
      const int t = t0 + wt + 16 * i + col;
      if (t >= P.n_tokens) continue;
#pragma unroll
      for (int j = 0; j < kFn; ++j) {
        const int n = n0 + wn + 16 * j + 4 * quad;
        if (n < P.part_stride)
          *reinterpret_cast<f32x4 *>(to + int64_t(t) * P.part_stride + n) = acc[j][i];
      }
    }
    return;
  }
  if constexpr (kFt * kFn <= 4) {
    if (gather) add_gathered<kType, kFn, kFt>(P, t0 + wt, n0 + wn, acc);
  }
  store<kType, kFn, kFt>(P, t0 + wt, n0 + wn, acc);
  if (steps > main_steps) mend<kType, kFn, kFt>(P, t0 + wt, n0 + wn, acc);
}

// Rows of b of an odd rank, laid out anew in rows of pad_rank that loads to LDS can take; 8 values
// a thread.
constexpr int kPackThreads = 256;
template <int kType>
__global__ __launch_bounds__(kPackThreads) void pack_kernel(const ProjectParams P, void *to,
                                                            int64_t rows) {
  typedef typename Num<kType>::E E;
  typedef typename Num<kType>::V8 V8;
  const int64_t id = int64_t(blockIdx.x) * kPackThreads + threadIdx.x;
  const int chunks = P.pad_rank / 8;
  const int64_t row = id / chunks;
  if (row >= rows) return;
  const int r = static_cast<int>(id - row * chunks) * 8;
  const E *from = static_cast<const E *>(P.b) + row * P.rank;
  V8 v = {};
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (r + i < P.rank) v[i] = from[r + i];
  *reinterpret_cast<V8 *>(static_cast<E *>(to) + row * P.pad_rank + r) = v;
}

// Adds the cuts of k, and each token's adapter: a thread has 4 outputs of a token.
constexpr int kFinishThreads = 256;

template <int kType>
__global__ __launch_bounds__(kFinishThreads) void finish_kernel(const ProjectParams P) {
  typedef typename Num<kType>::E E;
  typedef typename Num<kType>::V4 V4;
  typedef typename Num<kType>::V8 V8;
  const int t = blockIdx.y, n = (blockIdx.x * kFinishThreads + threadIdx.x) * 4;
  if (n >= P.n) return;
  const float *from = P.part + int64_t(t) * P.part_stride + n;
  const int64_t cut = int64_t(P.n_tokens) * P.part_stride;
  const int g = adapter_of(P, t);
  f32x4 sum = {};
#pragma unroll 8
  for (int s = 0; s < P.splits; ++s) sum += *reinterpret_cast<const f32x4 *>(from + s * cut);
  if (g >= 0) {
    const f32x4 *h = reinterpret_cast<const f32x4 *>(P.h32 + int64_t(t) * P.pad_rank);
    for (int r0 = 0; r0 < P.rank; r0 += 16) {
#pragma unroll
      for (int r = r0; r < r0 + 16; r += 8) {
        const f32x4 h0 = h[r / 4], h1 = h[r / 4 + 1];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const V8 b = b_chunk<kType>(P, g, n + q, r);
#pragma unroll
          for (int e = 0; e < 8; ++e)
            sum[q] = __builtin_fmaf(static_cast<float>(b[e]), e < 4 ? h0[e & 3] : h1[e & 3], sum[q]);
        }
      }
    }
  }
  E *y = static_cast<E *>(P.y) + t * P.y_stride + n;
  const V4 v = __builtin_convertvector(sum, V4);
  if (n + 3 < P.n) {
    __builtin_memcpy(y, &v, sizeof(v));
  } else {
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (n + q < P.n) y[q] = v[q];
  }
}

// `first` enqueues what the tiles wait for, if they can be launched.
template <int kType, int kT, int kN, int kWt, int kWn, int kStages, bool kCut = false, class First>
int launch_tiles(ProjectParams P, hipStream_t s, const First &first) {
  const int64_t tiles_t = (int64_t(P.n_tokens) + kT - 1) / kT;
  const int64_t tiles_n = (int64_t(P.n) + kN - 1) / kN;
  const int64_t blocks = tiles_t * tiles_n * (kCut ? P.splits : 1) + (kCut ? P.low_blocks : 0);
  // threads that a launch takes in one direction
  if (blocks * (kWt * kWn * 64) >= int64_t(1) << 32) return TG_E_INVAL;
  P.tiles_t = static_cast<int32_t>(tiles_t);
  P.tiles_n = static_cast<int32_t>(tiles_n);
  first();
  hipLaunchKernelGGL((project_kernel<kType, kT, kN, kWt, kWn, kStages, kCut>),
                     dim3(static_cast<uint32_t>(blocks)), dim3(kWt * kWn * 64), 0, s, P);
  return TG_OK;
}

// The few-token form: tiles of 32 or 64 tokens x 64 outputs, k in `splits` cuts.
constexpr int kFewTokens = 256;
struct Few {
  bool use, alone;  // for adapters, and without any
  int tile, splits;
};

Few few_of(int n_tokens, int k, int n) {
  Few f = {n_tokens <= kFewTokens, false, n_tokens <= 32 ? 32 : 64, 1};
  if (!f.use) return f;
  const int64_t tiles = int64_t((n_tokens + f.tile - 1) / f.tile) * ((int64_t(n) + 63) / 64);
  const int steps = (k + 63) / 64;
  // two workgroups a CU, and 4 steps at least for a cut
  int64_t want = (512 + tiles - 1) / tiles;
  if (want > steps / 4) want = steps / 4;
  if (want > 16) want = 16;
  if (want < 1) want = 1;
  const int each = (steps + static_cast<int>(want) - 1) / static_cast<int>(want);
  f.splits = (steps + each - 1) / each;
  f.alone = tiles <= 64 && steps >= 32;  // else the second launch costs more than it brings
  return f;
}

int part_stride(int n) { return (n + 3) / 4 * 4; }

template <int kType>
int launch(ProjectParams P, const Few &few, void *packed, hipStream_t s) {
  int rc;
  if (few.use && (P.adapter || few.alone)) {
    P.splits = few.splits;
    P.low_blocks = P.adapter ? P.n_tokens * (P.pad_rank / kTokenRanks) : 0;
    const auto none = [] {};
    rc = few.tile == 32 ? launch_tiles<kType, 32, 64, 1, 4, 4, true>(P, s, none)
                        : launch_tiles<kType, 64, 64, 2, 2, 4, true>(P, s, none);
    if (rc != TG_OK) return rc;
    hipLaunchKernelGGL(finish_kernel<kType>,
                       dim3((P.part_stride / 4 + kFinishThreads - 1) / kFinishThreads, P.n_tokens),
                       dim3(kFinishThreads), 0, s, P);
    return hipGetLastError() == hipSuccess ? TG_OK : TG_E_HIP;
  }
  const ProjectParams given = P;
  const auto first = [&] {
    if (!given.adapter) return;
    launch_shrink<kType>(given, s);
    if (!packed) return;
    const int64_t rows = int64_t(given.n_adapters) * given.n;
    const int64_t threads = rows * (given.pad_rank / 8);
    hipLaunchKernelGGL(pack_kernel<kType>,
                       dim3(static_cast<uint32_t>((threads + kPackThreads - 1) / kPackThreads)),
                       dim3(kPackThreads), 0, s, given, packed, rows);
  };
  if (packed) {
    P.b = packed;
    P.b_rank = P.pad_rank;
    P.b_apart = 0;
  }
  // Large problems take the tile with the least time for its rounds: 512 workgroups at once, two
  // a CU (256 with tiles of 256 values of n), and a round of 160 x 128, 192 x 256 and 256 x 256
  // takes 1.18, 1.37 and 1.64 times one of 128 x 128. Up to half a round of those: one a
  // CU, by 8 waves and with more steps under way; far fewer tiles than CUs: smaller ones, the
  // smallest where each has a CU.
  // Measured (bfloat16, no adapters, us) with tiles of 256 x 256, 192 x 256, 160 x 128, 128 x 128,
  // the latter with 8 waves, 128 x 64, 64 x 64:
  //   25,600 x 4,096, k 4,096: 700, 753, 721, 795, 851, 974, 1238
  //    8,192 x 8,192, k 8,192: 773, 936, 888, 948, 999, 1143, 1473
  //   12,000 x 1,024, k 1,024:  34,  28,  36,  33,  35,   36,   45
  //    6,400 x 1,536, k 1,024:  33,  28,  25,  32,  33,   31,   39
  //    2,048 x 4,096, k 4,096:  88,  71,  69,  63,  65,   75,   97
  //    2,048 x 2,048, k 4,096:                 45,  34,   41,   51
  //    4,000 x 1,000, k 1,000:                 16,  14,   18,   20
  //    1,777 x 2,048, k 1,160:  37,  32,  23,  20,  17,   20,   25
  //   11,019 x   233, k 2,464:  58,  48,  35,  33,  25,   31,   31
  //    2,314 x   721, k 3,632:                 45,  36,   27,   33
  //      512 x 4,096, k 4,096:  86,  68,  45,  43,  30,   25,   28
  //    1,000 x 1,024, k 2,048:  47,  39,  26,  21,  17,   13,   10
  const auto tiles = [&](int t, int n) {
    return ((int64_t(P.n_tokens) + t - 1) / t) * ((int64_t(P.n) + n - 1) / n);
  };
  P.b_whole = int64_t(P.n_adapters) * P.n * P.b_rank * 2 < (int64_t(1) << 31);
  P.gather = P.adapter && P.b_apart;  // rows of b that a load to LDS cannot take
  if (P.gather) rc = launch_tiles<kType, 64, 64, 2, 2, 4>(P, s, first);
  else if (tiles(128, 128) > 256) {
    const auto rounds = [&](int t, int n, int at_once) { return (tiles(t, n) + at_once - 1) / at_once; };
    const int64_t c256 = 164 * rounds(256, 256, 256), c192 = 137 * rounds(192, 256, 256);
    const int64_t c160 = 118 * rounds(160, 128, 512), c128 = 100 * rounds(128, 128, 512);
    const int64_t least = std::min(std::min(c256, c192), std::min(c160, c128));
    if (c256 == least) rc = launch_tiles<kType, 256, 256, 2, 4, 2>(P, s, first);
    else if (c192 == least) rc = launch_tiles<kType, 192, 256, 4, 2, 2>(P, s, first);
    else if (c160 == least) rc = launch_tiles<kType, 160, 128, 2, 2, 2>(P, s, first);
    else rc = launch_tiles<kType, 128, 128, 2, 2, 2>(P, s, first);
  }
  else if (tiles(128, 128) >= 160) rc = launch_tiles<kType, 128, 128, 2, 4, 4>(P, s, first);
  else if (tiles(64, 64) > 256) rc = launch_tiles<kType, 128, 64, 2, 2, 3>(P, s, first);
  else rc = launch_tiles<kType, 64, 64, 2, 2, 4>(P, s, first);
  if (rc != TG_OK) return rc;
  return hipGetLastError() == hipSuccess ? TG_OK : TG_E_HIP;
}

int pad_rank(int rank) { return rank <= 16 ? 16 : rank <= 32 ? 32 : 64; }

// Bytes of h: two values of the type and one of binary32 a rank, and a power of two a token.
size_t h_bytes(size_t n_tokens, int rank) {
  return n_tokens * pad_rank(rank) * (2 * 2 + sizeof(float)) +
         (n_tokens + 3) / 4 * 4 * sizeof(float);
}

// Adapters whose b may be laid out anew: with an odd rank, and not in the few-token form, which
// reads it as it is. What would take more than a few microseconds to lay out is gathered.
size_t pack_row_bytes(int n, int rank) { return size_t(n) * pad_rank(rank) * 2; }
size_t most_packed(int n_tokens, int n, int rank) {
  if (rank % 2 == 0 || n_tokens <= kFewTokens) return 0;
  return (size_t(64) << 20) / pack_row_bytes(n, rank);
}

// Sums over cuts of k, of any number of tokens up to this one: fewer may have more cuts.
size_t part_bytes(int n_tokens, int k, int n, bool low) {
  int64_t rows = 0;
  for (int tokens : {32, 64, 128, 192, 256}) {  // the most of a number of tiles
    const int t = std::min(tokens, n_tokens);
    const Few few = few_of(t, k, n);
    if (low || few.alone) rows = std::max<int64_t>(rows, int64_t(few.splits) * t);
  }
  return static_cast<size_t>(rows) * part_stride(n) * sizeof(float);
}

}  // namespace

extern "C" size_t tg_project_workspace_bytes(int32_t n_tokens, int32_t k, int32_t n,
                                             int32_t n_adapters, int32_t rank) {
  if (n_tokens <= 0 || k <= 0 || n <= 0 || n_adapters < 0 || rank < 0) return 0;
  const bool low = n_adapters > 0 && rank > 0;
  if (n_adapters > 0 && !low) return 0;
  size_t bytes = part_bytes(n_tokens, k, n, low);
  if (low) {
    bytes += h_bytes(n_tokens, rank);
    bytes += std::min<size_t>(n_adapters, most_packed(n_tokens, n, rank)) * pack_row_bytes(n, rank);
  }
  return bytes;
}

extern "C" int tg_project(const tg_project_args *a, void *stream) {
  if (!a || a->n_tokens < 0 || a->k < 1 || a->k % 8 || a->n < 1 || a->n_adapters < 0 ||
      !type_ok(a->type))
    return TG_E_INVAL;
  if (a->x_stride < a->k || a->w_stride < a->k || a->y_stride < a->n || a->x_stride % 8 ||
      a->w_stride % 8 || a->x_stride > kMaxStride || a->w_stride > kMaxStride)
    return TG_E_INVAL;
  const bool low = a->adapter && a->n_adapters > 0;
  if (low && (a->rank < 1 || a->rank > TG_PROJECT_MAX_RANK || a->n > (1 << 23) ||
              a->n_tokens > (1 << 28)))
    return TG_E_INVAL;
  if (a->n_tokens == 0) return TG_OK;
  if (!a->x || !a->w || !a->y || !aligned16(a->x) || !aligned16(a->w)) return TG_E_INVAL;
  if (low && (!a->a || !a->b || !a->scale || !aligned16(a->a))) return TG_E_INVAL;
  ProjectParams P = {};
  P.x = a->x;
  P.w = a->w;
  P.y = a->y;
  P.x_stride = a->x_stride;
  P.w_stride = a->w_stride;
  P.y_stride = a->y_stride;
  P.n_tokens = a->n_tokens;
  P.k = a->k;
  P.n = a->n;
  const Few few = few_of(a->n_tokens, a->k, a->n);
  const size_t need = tg_project_workspace_bytes(a->n_tokens, a->k, a->n,
                                                 low ? a->n_adapters : 0, low ? a->rank : 0);
  if (need > 0 && (!a->workspace || a->workspace_bytes < need || !aligned16(a->workspace)))
    return TG_E_WORKSPACE;
  P.part = static_cast<float *>(a->workspace);
  P.part_stride = part_stride(a->n);
  void *packed = nullptr;
  if (low) {
    P.a = a->a;
    P.b = a->b;
    P.adapter = a->adapter;
    P.scale = a->scale;
    P.n_adapters = a->n_adapters;
    P.rank = a->rank;
    P.pad_rank = pad_rank(a->rank);
    const uintptr_t at = reinterpret_cast<uintptr_t>(a->b);
    P.b_apart = a->rank % 2 != 0 || at % 4 != 0;
    P.h32 = static_cast<float *>(a->workspace);
    P.h = P.h32 + size_t(a->n_tokens) * P.pad_rank;
    P.h_up = P.h32 + size_t(a->n_tokens) * P.pad_rank * 2;
    P.part = P.h32 + h_bytes(a->n_tokens, a->rank) / sizeof(float);
    if (size_t(a->n_adapters) <= most_packed(a->n_tokens, a->n, a->rank)) packed = P.part;
    P.b_rank = a->rank;
  }
  hipStream_t s = static_cast<hipStream_t>(stream);
  return a->type == TG_F16 ? launch<TG_F16>(P, few, packed, s)
                           : launch<TG_BF16>(P, few, packed, s);
}
