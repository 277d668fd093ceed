// tg_project: a shared projection and the low-rank adapters of many cameras, y = x w^T + the
// adapter's scale_g (x a_g^T) b_g^T (low-rank adaptation, Hu et al. 2021, one adapter a token).
//
// Two launches:
//  1. shrink: h[t] = scale_g x[t] a_g^T for the tokens that have an adapter. Kept as two values
//     of the type whose sum is h (the first rounded, the second what that rounding left): 22
//     bits of binary16, 16 of bfloat16. A binary16 row whose largest value is far from 1 is
//     divided by a power of two first, which is kept with it.
//  2. the product: tiles of x and w go through LDS to the matrix instructions; each tile then
//     adds b_g h[t] for its tokens, adapter by adapter, as a few more matrix instructions in
//     which h is 0 for the tokens of other adapters.
// Results lie transposed in the registers (a lane holds 4 outputs of one token), so that a
// token's adapter and power of two belong to the lane, and stores are contiguous.
#include <hip/hip_runtime.h>

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
  void *h;           // [n_tokens][2][pad_rank] of the type
  float *power;      // [n_tokens]
  int32_t tiles_t, tiles_n;
  int32_t vec_y;     // 4 outputs of a token can be stored at once
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
  int e = 0;
  if (kType == TG_F16) {  // bfloat16 has the range of the sums
    float big = 0.0f;
#pragma unroll
    for (int f = 0; f < kFrags; ++f) big = fmaxf(big, fabsf(v[f]));
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) big = fmaxf(big, __shfl_xor(big, o, 16));
    // in between, the second value's last bit is 2^-19 of the largest or less
    if ((big >= 32768.0f || big < 0.015625f) && big > 0.0f && big < INFINITY) frexpf(big, &e);
    e = min(max(e, -126), 127);  // the power itself stays a normal number
  }
  if (r0 == 0) P.power[t] = ldexpf(1.0f, e);
  E *h = static_cast<E *>(P.h) + int64_t(t) * 2 * P.pad_rank;
#pragma unroll
  for (int f = 0; f < kFrags; ++f) {
    const float s = ldexpf(v[f], -e);
    const E hi = static_cast<E>(s);
    const float rest = s - static_cast<float>(hi);
    h[f * 16 + r0] = hi;
    h[P.pad_rank + f * 16 + r0] = static_cast<E>(fabsf(s) < INFINITY ? rest : 0.0f);
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

// Few tokens: a workgroup a token, whose row of x and rows of a are read as they lie.
template <int kType, int kFrags>
__global__ __launch_bounds__(kShrinkThreads) void shrink_few_kernel(const ProjectParams P) {
  typedef typename Num<kType>::E E;
  typedef typename Num<kType>::V8 V8;
  constexpr int kEach = kFrags * 16 / kShrinkWaves;  // ranks of a wave
  __shared__ float part[kFrags * 16];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int t = blockIdx.x;
  const int g = adapter_of(P, t);
  if (g < 0) return;
  const E *x = static_cast<const E *>(P.x) + t * P.x_stride;
  const E *a = static_cast<const E *>(P.a) + int64_t(g) * P.rank * P.k;
  float sum[kEach] = {};
  for (int k = lane * 8; k < P.k; k += 1024) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      if (k + u * 512 >= P.k) continue;
      const V8 xv = *reinterpret_cast<const V8 *>(x + k + u * 512);
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        const int r = min(e * kShrinkWaves + wave, P.rank - 1);
        const V8 av = *reinterpret_cast<const V8 *>(a + int64_t(r) * P.k + k + u * 512);
#pragma unroll
        for (int i = 0; i < 8; ++i)
          sum[e] = __builtin_fmaf(static_cast<float>(av[i]), static_cast<float>(xv[i]), sum[e]);
      }
    }
  }
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    sum[e] = wave_sum(sum[e]);
    if (lane == 0) part[e * kShrinkWaves + wave] = sum[e];
  }
  __syncthreads();
  if (threadIdx.x >= 16) return;
  const float scale = P.scale[g];
  float v[kFrags];
#pragma unroll
  for (int f = 0; f < kFrags; ++f) {
    const int r = f * 16 + threadIdx.x;
    v[f] = r < P.rank ? part[r] * scale : 0.0f;
  }
  keep_h<kType, kFrags>(P, t, v, threadIdx.x);
}

template <int kType, int kFrags>
void launch_shrink_rank(const ProjectParams &P, hipStream_t s) {
  const int most = P.n_adapters < 16 ? P.n_adapters : 16;
  if (P.n_tokens <= 64)
    hipLaunchKernelGGL((shrink_few_kernel<kType, kFrags>), dim3(P.n_tokens), dim3(kShrinkThreads),
                       0, s, P);
  else if (P.n_tokens < 8192)
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

// 8 values of b_g's row j from rank r on, zero past the rank and past the last output.
template <int kType>
__device__ __forceinline__ typename Num<kType>::V8 b_chunk(const ProjectParams &P, int g, int j,
                                                            int r) {
  typedef typename Num<kType>::E E;
  typedef typename Num<kType>::V8 V8;
  V8 v = {};
  if (j >= P.n || r >= P.rank) return v;
  const E *b = static_cast<const E *>(P.b) + (int64_t(g) * P.n + j) * P.rank + r;
  if (P.rank % 8 == 0 && (reinterpret_cast<uintptr_t>(P.b) & 15) == 0) {
    v = *reinterpret_cast<const V8 *>(b);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (r + i < P.rank) v[i] = b[i];
  }
  return v;
}

// Whether one of 8 values is an infinity or NaN.
template <int kType>
__device__ __forceinline__ bool wild(typename Num<kType>::V8 v) {
  const i32x4 d = __builtin_bit_cast(i32x4, v);
  const uint32_t mask = kType == TG_F16 ? 0x7C007C00u : 0x7F807F80u;
  const uint32_t one = kType == TG_F16 ? 0x04000400u : 0x00800080u;  // an exponent's last bit
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) any |= (static_cast<uint32_t>(d[i]) & mask) + one;
  return any & 0x80008000u;
}

// Adds b_g h[t] to a wave's results: acc[j][i] holds outputs n0 + 16 j + 4 (lane / 16) .. of
// token t0 + 16 i + lane % 16. Tokens of other adapters have h = 0 in the product, which adds
// nothing as long as b_g is finite; otherwise, and where h carries a power of two, the product
// is formed by itself and taken by the adapter's own tokens.
template <int kType, int kFn, int kFt>
__device__ __forceinline__ void add_adapters(const ProjectParams &P, int t0, int n0,
                                             f32x4 (&acc)[kFn][kFt]) {
  typedef Num<kType> N;
  typedef typename N::E E;
  typedef typename N::V8 V8;
  const int lane = threadIdx.x & 63, col = lane & 15, quad = lane >> 4;
  int mine[kFt];
  float power[kFt];
  uint64_t left[kFt];
  bool plain = true;
#pragma unroll
  for (int i = 0; i < kFt; ++i) mine[i] = adapter_of(P, t0 + 16 * i + col);
#pragma unroll
  for (int i = 0; i < kFt; ++i) {
    left[i] = __ballot(mine[i] >= 0) & 0xFFFF;
    power[i] = 1.0f;
    if (kType == TG_F16 && mine[i] >= 0) power[i] = P.power[t0 + 16 * i + col];
    plain = plain && power[i] == 1.0f;
  }
  if (kType == TG_F16) plain = __ballot(!plain) == 0;
  const E *h = static_cast<const E *>(P.h) + int64_t(t0 + col) * 2 * P.pad_rank;
  // with 16 ranks one step of 32 holds both values of h, otherwise a step holds one of them
  const int narrow = P.pad_rank == 16;
  for (;;) {
    int g = -1;
#pragma unroll
    for (int i = kFt - 1; i >= 0; --i)
      if (left[i]) g = __builtin_amdgcn_readlane(mine[i], __builtin_ctzll(left[i]));
    if (g < 0) break;
    uint64_t has[kFt];
#pragma unroll
    for (int i = 0; i < kFt; ++i) {
      has[i] = __ballot(mine[i] == g) & 0xFFFF;
      left[i] &= ~has[i];
    }
    for (int r0 = 0; r0 < P.pad_rank; r0 += 32) {
      const int r = r0 + (narrow ? (quad & 1) * 8 : quad * 8);
      V8 bf[kFn];
      bool odd = false;
#pragma unroll
      for (int j = 0; j < kFn; ++j) bf[j] = b_chunk<kType>(P, g, n0 + 16 * j + col, r);
#pragma unroll
      for (int j = 0; j < kFn; ++j) odd = odd || wild<kType>(bf[j]);
      const bool direct = plain && __ballot(odd) == 0;
      constexpr int kAt = kFt < 4 ? kFt : 4;  // token blocks whose h is loaded at once
#pragma unroll
      for (int i0 = 0; i0 < kFt; i0 += kAt) {
        V8 hv[kAt][2];
#pragma unroll
        for (int i = 0; i < kAt; ++i) {
          hv[i][0] = hv[i][1] = V8{};
          if (mine[i0 + i] == g) {
            const E *from = h + int64_t(16 * (i0 + i)) * 2 * P.pad_rank;
            hv[i][0] = *reinterpret_cast<const V8 *>(from + (narrow ? quad * 8 : r));
            if (!narrow) hv[i][1] = *reinterpret_cast<const V8 *>(from + P.pad_rank + r);
          }
        }
#pragma unroll
        for (int i = 0; i < kAt; ++i) {
          if (!has[i0 + i]) continue;
          if (direct) {
#pragma unroll
            for (int j = 0; j < kFn; ++j) {
              acc[j][i0 + i] = N::mfma16(bf[j], hv[i][0], acc[j][i0 + i]);
              if (!narrow) acc[j][i0 + i] = N::mfma16(bf[j], hv[i][1], acc[j][i0 + i]);
            }
          } else {
#pragma unroll
            for (int j = 0; j < kFn; ++j) {
              f32x4 low = {};
              low = N::mfma16(bf[j], hv[i][0], low);
              if (!narrow) low = N::mfma16(bf[j], hv[i][1], low);
              if (mine[i0 + i] == g) {
#pragma unroll
                for (int q = 0; q < 4; ++q) acc[j][i0 + i][q] += power[i0 + i] * low[q];
              }
            }
          }
        }
      }
    }
  }
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
      if (P.vec_y && n + 3 < P.n) {
        *reinterpret_cast<V4 *>(row + n) = v;
      } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (n + r < P.n) row[n + r] = v[r];
      }
    }
  }
}

// A tile of kT tokens x kN outputs, kWt x kWn waves, kBK values of k a step, kStages steps of
// loads under way. Step s + 1's operands are read from LDS while step s's are multiplied, so
// that the matrix units have work across the barrier; the buffer of step s is free for step
// s + kStages behind that barrier, since its operands are in registers by then.
// Rows of a tile lie in LDS as kBK / 8 chunks of 16 bytes, and the 16 rows that an operand takes
// one chunk of fall on 16 different places of the 256 bytes that LDS serves at once.
template <int kBK>
__device__ __forceinline__ int place_of(int row, int c) {
  return kBK == 64 ? c ^ ((row >> 1) & 7) : c ^ ((row >> 2) & 3);
}

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

template <int kType, int kT, int kN, int kWt, int kWn, int kBK, int kStages>
__global__ __launch_bounds__(kWt *kWn * 64, 2) void project_kernel(const ProjectParams P) {
  typedef Num<kType> N;
  typedef typename N::E E;
  typedef typename N::V8 V8;
  constexpr int kWaves = kWt * kWn, kFt = kT / kWt / 16, kFn = kN / kWn / 16;
  constexpr int kChunks = kBK / 8, kRows = kT + kN, kPer = 64 / kChunks;  // rows of one load
  constexpr int kLoads = kRows / kPer / kWaves, kSub = kBK / 32;
  static_assert(kLoads * kPer * kWaves == kRows && kT % kPer == 0, "whole loads");
  __shared__ __attribute__((aligned(16))) E tile[kStages][kRows * kBK];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, quad = lane >> 4;
  int tt, tn;
  tile_of(blockIdx.x, P.tiles_t, P.tiles_n, tt, tn);
  const int t0 = tt * kT, n0 = tn * kN;
  const int xr = min(kT, P.n_tokens - t0), wr = min(kN, P.n - n0);
  const auto xb = buffer(static_cast<const E *>(P.x) + t0 * P.x_stride,
                         static_cast<uint32_t>(((xr - 1) * P.x_stride + P.k) * 2));
  const auto wb = buffer(static_cast<const E *>(P.w) + n0 * P.w_stride,
                         static_cast<uint32_t>(((wr - 1) * P.w_stride + P.k) * 2));
  // load i of a wave covers kPer rows; rows past the tensor repeat its last one. A lane's chunk
  // is the same in all loads, since their rows are 4 kPer apart or more.
  static_assert(kWaves * kPer % 16 == 0, "rows of one lane");
  const int chunk = place_of<kBK>(wave * kPer + lane / kChunks, lane % kChunks);
  uint32_t at[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int row = (i * kWaves + wave) * kPer + lane / kChunks;
    at[i] = row < kT ? static_cast<uint32_t>((min(row, xr - 1) * P.x_stride + chunk * 8) * 2)
                     : static_cast<uint32_t>((min(row - kT, wr - 1) * P.w_stride + chunk * 8) * 2);
  }
  auto fetch = [&](int s) {  // every step's loads are issued, so that they can be counted
    const int k0 = s * kBK;
    const bool past = k0 + chunk * 8 >= P.k;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int first = (i * kWaves + wave) * kPer;
      load_lds(first < kT ? xb : wb, &tile[s % kStages][first * kBK], past ? kNowhere : at[i],
               static_cast<uint32_t>(k0) * 2);
    }
  };
  f32x4 acc[kFn][kFt] = {};
  const int wt = (wave % kWt) * (kT / kWt), wn = (wave / kWt) * (kN / kWn);
  const int steps = (P.k + kBK - 1) / kBK;
  struct Operands {
    V8 x[kSub][kFt], w[kSub][kFn];
  };
  auto read = [&](Operands &o, int s) {
    const E *m = tile[s % kStages];
#pragma unroll
    for (int ks = 0; ks < kSub; ++ks) {
#pragma unroll
      for (int i = 0; i < kFt; ++i) {
        const int row = wt + 16 * i + col;
        o.x[ks][i] =
            *reinterpret_cast<const V8 *>(m + row * kBK + place_of<kBK>(row, ks * 4 + quad) * 8);
      }
#pragma unroll
      for (int j = 0; j < kFn; ++j) {
        const int row = kT + wn + 16 * j + col;
        o.w[ks][j] =
            *reinterpret_cast<const V8 *>(m + row * kBK + place_of<kBK>(row, ks * 4 + quad) * 8);
      }
    }
  };
  auto multiply = [&](const Operands &o) {
#pragma unroll
    for (int ks = 0; ks < kSub; ++ks)
#pragma unroll
      for (int j = 0; j < kFn; ++j)
#pragma unroll
        for (int i = 0; i < kFt; ++i) acc[j][i] = N::mfma16(o.w[ks][j], o.x[ks][i], acc[j][i]);
  };
  auto step = [&](int s, Operands &now, Operands &then) {
    wait_and_meet<(kStages - 2) * kLoads>();  // step s + 1 is here, step s in registers
    fetch(s + kStages);
    read(then, s + 1);
    multiply(now);
    // the scheduler would put the reads at the end, where the next step waits for them
    constexpr int kReads = kSub * (kFt + kFn), kMul = kSub * kFt * kFn;
#pragma unroll
    for (int i = 0; i < kReads; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, kMul / kReads, 0);
      if (i < kLoads) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
    }
  };
#pragma unroll
  for (int s = 0; s < kStages; ++s) fetch(s);
  wait_and_meet<(kStages - 1) * kLoads>();
  Operands a, b;
  read(a, 0);
  for (int s = 0; s < steps; s += 2) {  // a step past the last one multiplies zeros
    step(s, a, b);
    step(s + 1, b, a);
  }
  wait_loads();  // LDS belongs to the next workgroup from here on
  if (P.adapter) add_adapters<kType, kFn, kFt>(P, t0 + wt, n0 + wn, acc);
  store<kType, kFn, kFt>(P, t0 + wt, n0 + wn, acc);
}

// Few tokens (kFt x 16 of them): 16 outputs a workgroup, k cut over its waves, operands straight
// from memory; the waves' sums are joined in LDS. A lane takes 32 bytes of a row at a time, so
// that 4 lanes cover a line; x is read in the same order of k.
constexpr int kFewWaves = 8;

template <int kType, int kFt>
__global__ __launch_bounds__(kFewWaves * 64) void project_few_kernel(const ProjectParams P) {
  typedef Num<kType> N;
  typedef typename N::E E;
  typedef typename N::V8 V8;
  __shared__ f32x4 part[kFewWaves][kFt][64];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, quad = lane >> 4;
  const int n0 = blockIdx.x * 16;
  const E *w = static_cast<const E *>(P.w) + min(n0 + col, P.n - 1) * P.w_stride;
  const E *x[kFt];
#pragma unroll
  for (int i = 0; i < kFt; ++i)
    x[i] = static_cast<const E *>(P.x) + min(16 * i + col, P.n_tokens - 1) * P.x_stride;
  f32x4 acc[kFt] = {};
  // a wave takes 64 values of k at a time, two such at once
  auto take = [&](int k) {
    V8 wf[2][2], xf[2][2][kFt];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int at = k + u * kFewWaves * 64 + 8 * h;
        wf[u][h] = V8{};
        if (at < P.k) wf[u][h] = *reinterpret_cast<const V8 *>(w + at);
#pragma unroll
        for (int i = 0; i < kFt; ++i) {
          xf[u][h][i] = V8{};
          if (at < P.k) xf[u][h][i] = *reinterpret_cast<const V8 *>(x[i] + at);
        }
      }
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < kFt; ++i) acc[i] = N::mfma16(wf[u][h], xf[u][h][i], acc[i]);
  };
  for (int k = wave * 64; k < P.k; k += 2 * kFewWaves * 64) take(k + quad * 16);
#pragma unroll
  for (int i = 0; i < kFt; ++i) part[wave][i][lane] = acc[i];
  __syncthreads();
  if (wave >= kFt) return;
  f32x4 sum[1][1] = {};
#pragma unroll
  for (int v = 0; v < kFewWaves; ++v) sum[0][0] += part[v][wave][lane];
  if (P.adapter) add_adapters<kType, 1, 1>(P, 16 * wave, n0, sum);
  store<kType, 1, 1>(P, 16 * wave, n0, sum);
}

template <int kType, int kT, int kN, int kWt, int kWn, int kBK, int kStages>
int launch_tiles(ProjectParams P, hipStream_t s) {
  const int64_t tiles_t = (int64_t(P.n_tokens) + kT - 1) / kT;
  const int64_t tiles_n = (int64_t(P.n) + kN - 1) / kN;
  if (tiles_t * tiles_n > INT32_MAX / kGroup) return TG_E_INVAL;
  P.tiles_t = static_cast<int32_t>(tiles_t);
  P.tiles_n = static_cast<int32_t>(tiles_n);
  hipLaunchKernelGGL((project_kernel<kType, kT, kN, kWt, kWn, kBK, kStages>),
                     dim3(static_cast<uint32_t>(tiles_t * tiles_n)), dim3(kWt * kWn * 64), 0, s,
                     P);
  return TG_OK;
}

template <int kType, int kFt>
int launch_few(const ProjectParams &P, hipStream_t s) {
  hipLaunchKernelGGL((project_few_kernel<kType, kFt>), dim3((P.n + 15) / 16),
                     dim3(kFewWaves * 64), 0, s, P);
  return TG_OK;
}

template <int kType>
int launch(const ProjectParams &P, hipStream_t s) {
  if (P.adapter) launch_shrink<kType>(P, s);
  int rc;
  const int64_t big = ((int64_t(P.n_tokens) + 255) / 256) * ((P.n + 255) / 256);
  const int64_t mid = ((int64_t(P.n_tokens) + 127) / 128) * ((P.n + 127) / 128);
  if (P.n_tokens <= 16) rc = launch_few<kType, 1>(P, s);
  else if (P.n_tokens <= 32) rc = launch_few<kType, 2>(P, s);
  else if (P.n_tokens <= 64) rc = launch_few<kType, 4>(P, s);
  else if (big >= 256) rc = launch_tiles<kType, 256, 256, 2, 4, 32, 4>(P, s);
  else if (mid >= 256) rc = launch_tiles<kType, 128, 128, 2, 2, 64, 2>(P, s);
  else rc = launch_tiles<kType, 64, 64, 2, 2, 64, 4>(P, s);
  if (rc != TG_OK) return rc;
  return hipGetLastError() == hipSuccess ? TG_OK : TG_E_HIP;
}

int pad_rank(int rank) { return rank <= 16 ? 16 : rank <= 32 ? 32 : 64; }

}  // namespace

extern "C" size_t tg_project_workspace_bytes(int32_t n_tokens, int32_t k, int32_t n,
                                             int32_t n_adapters, int32_t rank) {
  if (n_tokens <= 0 || k <= 0 || n <= 0 || n_adapters <= 0 || rank <= 0) return 0;
  const size_t t = static_cast<size_t>(n_tokens);
  return (t * 4 + 15) / 16 * 16 + t * 2 * pad_rank(rank) * 2;
}

extern "C" int tg_project(const tg_project_args *a, void *stream) {
  if (!a || a->n_tokens < 0 || a->k < 1 || a->k % 8 || a->n < 1 || a->n_adapters < 0 ||
      !type_ok(a->type))
    return TG_E_INVAL;
  if (a->x_stride < a->k || a->w_stride < a->k || a->y_stride < a->n || a->x_stride % 8 ||
      a->w_stride % 8 || a->x_stride > kMaxStride || a->w_stride > kMaxStride)
    return TG_E_INVAL;
  const bool low = a->adapter && a->n_adapters > 0;
  if (low && (a->rank < 1 || a->rank > TG_PROJECT_MAX_RANK)) return TG_E_INVAL;
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
  P.vec_y = reinterpret_cast<uintptr_t>(a->y) % 8 == 0 && a->y_stride % 4 == 0;
  if (low) {
    const size_t need =
        tg_project_workspace_bytes(a->n_tokens, a->k, a->n, a->n_adapters, a->rank);
    if (!a->workspace || a->workspace_bytes < need || !aligned16(a->workspace))
      return TG_E_WORKSPACE;
    P.a = a->a;
    P.b = a->b;
    P.adapter = a->adapter;
    P.scale = a->scale;
    P.n_adapters = a->n_adapters;
    P.rank = a->rank;
    P.pad_rank = pad_rank(a->rank);
    P.power = static_cast<float *>(a->workspace);
    P.h = static_cast<char *>(a->workspace) + (size_t(a->n_tokens) * 4 + 15) / 16 * 16;
  }
  hipStream_t s = static_cast<hipStream_t>(stream);
  return a->type == TG_F16 ? launch<TG_F16>(P, s) : launch<TG_BF16>(P, s);
}
