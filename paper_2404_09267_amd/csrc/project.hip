// tg_project: a shared projection and the low-rank adapters of many cameras, y = x w^T + the
// adapter's scale_g (x a_g^T) b_g^T (low-rank adaptation, Hu et al. 2021, one adapter a token).
//
// Two launches:
//  1. shrink: h[t] = scale_g x[t] a_g^T for the tokens that have an adapter, 16 tokens a
//     workgroup. Kept as two values of the type whose sum is h (the first rounded, the second
//     what that rounding left) and a power of two that brings the row near 1, so that binary16
//     neither overflows nor loses small rows: 22 bits of binary16, 16 of bfloat16.
//  2. the product: tiles of x and w go through LDS to the matrix instructions; each tile then
//     adds b_g h[t] for its tokens, adapter by adapter, as a few more matrix instructions whose
//     result is taken only by the adapter's own tokens.
// Results lie transposed in the registers (a lane holds 4 outputs of one token), so that a
// token's adapter and power of two belong to the lane, and stores are contiguous.
#include <hip/hip_runtime.h>

#include <climits>
#include <cstdint>

#include "tg.h"
#include "token_math.h"

namespace {

using namespace tok;

constexpr int kBK = 64;       // values of k per step: rows of 128 bytes in LDS
constexpr int kMaxStride = 1 << 22;

struct ProjectParams {
  const void *x, *w, *a, *b;
  const int32_t *adapter;
  const float *scale;
  void *y;
  int64_t x_stride, w_stride, y_stride;
  int32_t n_tokens, k, n, n_adapters, rank;
  int32_t pad_rank;  // rank rounded up to 16
  void *h;           // [n_tokens][2][pad_rank] of the type
  float *power;      // [n_tokens]
  int32_t tiles_n;
  int32_t vec_y;     // 4 outputs of a token can be stored at once
};

__device__ __forceinline__ int adapter_of(const ProjectParams &P, int t) {
  if (!P.adapter || t >= P.n_tokens) return -1;
  const int g = P.adapter[t];
  return g >= 0 && g < P.n_adapters ? g : -1;
}

// ------------------------------------------------------------------------------- shrink

constexpr int kShrinkThreads = 256;

template <int kType>
__global__ __launch_bounds__(kShrinkThreads) void shrink_kernel(const ProjectParams P) {
  typedef Num<kType> N;
  typedef typename N::E E;
  typedef typename N::V8 V8;
  constexpr int kWaves = kShrinkThreads / 64, kFrags = TG_PROJECT_MAX_RANK / 16;
  __shared__ float part[kWaves][TG_PROJECT_MAX_RANK][17];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = lane & 15, quad = lane >> 4;
  const int t = blockIdx.x * 16 + col;
  const int mine = adapter_of(P, t);
  const int frags = P.pad_rank / 16;
  f32x4 sum[kFrags] = {};
  // distinct adapters of the 16 tokens, one after the other; the same for every wave
  uint64_t left = __ballot(mine >= 0) & 0xFFFF;
  const E *xrow = static_cast<const E *>(P.x) + int64_t(min(t, P.n_tokens - 1)) * P.x_stride;
  while (left) {
    const int g = __builtin_amdgcn_readlane(mine, __builtin_ctzll(left));
    left &= ~__ballot(mine == g);
    f32x4 acc[kFrags] = {};
    const E *a = static_cast<const E *>(P.a) + int64_t(g) * P.rank * P.k;
    for (int k = wave * 32 + quad * 8; k < P.k + quad * 8; k += kWaves * 32) {
      V8 xv = {};
      if (k < P.k) xv = *reinterpret_cast<const V8 *>(xrow + k);
#pragma unroll
      for (int f = 0; f < kFrags; ++f) {
        if (f >= frags) break;
        V8 av = {};
        const int r = f * 16 + col;
        if (k < P.k && r < P.rank) av = *reinterpret_cast<const V8 *>(a + int64_t(r) * P.k + k);
        acc[f] = N::mfma16(av, xv, acc[f]);
      }
    }
    if (mine == g) {
#pragma unroll
      for (int f = 0; f < kFrags; ++f) sum[f] = acc[f];
    }
  }
#pragma unroll
  for (int f = 0; f < kFrags; ++f) {
    if (f >= frags) break;
#pragma unroll
    for (int i = 0; i < 4; ++i) part[wave][f * 16 + quad * 4 + i][col] = sum[f][i];
  }
  __syncthreads();
  // 16 threads a token
  const int tok = threadIdx.x >> 4, r0 = threadIdx.x & 15;
  const int tt = blockIdx.x * 16 + tok;
  const int g = adapter_of(P, tt);
  if (g < 0) return;  // nothing reads h of a token without an adapter
  const float scale = P.scale[g];
  float v[kFrags], big = 0.0f;
#pragma unroll
  for (int f = 0; f < kFrags; ++f) {
    v[f] = 0.0f;
    if (f >= frags) break;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) v[f] += part[w][f * 16 + r0][tok];
    v[f] *= scale;
    big = fmaxf(big, fabsf(v[f]));
  }
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) big = fmaxf(big, __shfl_xor(big, o, 16));
  int e = 0;
  if (big > 0.0f && big < INFINITY) frexpf(big, &e);
  e = min(max(e, -126), 127);  // the power itself stays a normal number
  if (r0 == 0) P.power[tt] = ldexpf(1.0f, e);
  E *h = static_cast<E *>(P.h) + int64_t(tt) * 2 * P.pad_rank;
#pragma unroll
  for (int f = 0; f < kFrags; ++f) {
    if (f >= frags) break;
    const float s = ldexpf(v[f], -e);
    const E hi = static_cast<E>(s);
    const float rest = s - static_cast<float>(hi);
    h[f * 16 + r0] = hi;
    h[P.pad_rank + f * 16 + r0] = static_cast<E>(fabsf(s) < INFINITY ? rest : 0.0f);
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

// Adds b_g h[t] to a wave's results: acc[j][i] holds outputs n0 + 16 j + 4 (lane / 16) .. of
// token t0 + 16 i + lane % 16.
template <int kType, int kFn, int kFt>
__device__ __forceinline__ void add_adapters(const ProjectParams &P, int t0, int n0,
                                             f32x4 (&acc)[kFn][kFt]) {
  typedef Num<kType> N;
  typedef typename N::E E;
  typedef typename N::V8 V8;
  const int lane = threadIdx.x & 63, col = lane & 15, quad = lane >> 4;
#pragma unroll
  for (int i = 0; i < kFt; ++i) {
    const int t = t0 + 16 * i + col;
    const int mine = adapter_of(P, t);
    uint64_t left = __ballot(mine >= 0) & 0xFFFF;
    if (!left) continue;
    const float power = mine >= 0 ? P.power[t] : 0.0f;
    const E *h = static_cast<const E *>(P.h) + int64_t(t) * 2 * P.pad_rank;
    while (left) {
      const int g = __builtin_amdgcn_readlane(mine, __builtin_ctzll(left));
      left &= ~__ballot(mine == g);
      f32x4 low[kFn] = {};
      for (int s = quad * 8; s < 2 * P.pad_rank; s += 32) {
        V8 hv = {};
        if (mine == g) hv = *reinterpret_cast<const V8 *>(h + s);
        const int r = s < P.pad_rank ? s : s - P.pad_rank;
#pragma unroll
        for (int j = 0; j < kFn; ++j)
          low[j] = N::mfma16(b_chunk<kType>(P, g, n0 + 16 * j + col, r), hv, low[j]);
      }
      if (mine == g) {
#pragma unroll
        for (int j = 0; j < kFn; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[j][i][r] += power * low[j][r];
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

// A tile of kT tokens x kN outputs, kWt x kWn waves. Rows of a tile lie in LDS as 8 chunks of
// 16 bytes, chunk c of row r at place c ^ (r / 2 % 8): the 16 rows that an operand takes from
// one chunk column fall on 16 different places of the 256 bytes that LDS serves at once.
template <int kType, int kT, int kN, int kWt, int kWn>
__global__ __launch_bounds__(kWt *kWn * 64) void project_kernel(const ProjectParams P) {
  typedef Num<kType> N;
  typedef typename N::E E;
  typedef typename N::V8 V8;
  constexpr int kWaves = kWt * kWn, kFt = kT / kWt / 16, kFn = kN / kWn / 16;
  constexpr int kRows = kT + kN, kLoads = kRows * 8 / (kWaves * 64);
  __shared__ __attribute__((aligned(16))) E tile[2][kRows * kBK];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, quad = lane >> 4;
  const int tn = blockIdx.x % P.tiles_n, tt = blockIdx.x / P.tiles_n;
  const int t0 = tt * kT, n0 = tn * kN;
  const int xr = min(kT, P.n_tokens - t0), wr = min(kN, P.n - n0);
  const auto xb = buffer(static_cast<const E *>(P.x) + t0 * P.x_stride,
                         static_cast<uint32_t>(((xr - 1) * P.x_stride + P.k) * 2));
  const auto wb = buffer(static_cast<const E *>(P.w) + n0 * P.w_stride,
                         static_cast<uint32_t>(((wr - 1) * P.w_stride + P.k) * 2));
  // load i of a wave covers 8 rows; rows past the tensor repeat its last one
  uint32_t at[kLoads];
  int kc[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int row = (i * kWaves + wave) * 8 + (lane >> 3);
    const int c = (lane & 7) ^ ((row >> 1) & 7);
    kc[i] = c * 8;
    at[i] = row < kT ? static_cast<uint32_t>((min(row, xr - 1) * P.x_stride + c * 8) * 2)
                     : static_cast<uint32_t>((min(row - kT, wr - 1) * P.w_stride + c * 8) * 2);
  }
  auto fetch = [&](int k0, int to) {
    const bool tail = k0 + kBK > P.k;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int first = (i * kWaves + wave) * 8;
      const uint32_t off = tail && k0 + kc[i] >= P.k ? kNowhere : at[i];
      load_lds(first < kT ? xb : wb, &tile[to][first * kBK], off, static_cast<uint32_t>(k0) * 2);
    }
  };
  f32x4 acc[kFn][kFt] = {};
  const int wt = (wave % kWt) * (kT / kWt), wn = (wave / kWt) * (kN / kWn);
  const int steps = (P.k + kBK - 1) / kBK;
  fetch(0, 0);
  for (int s = 0; s < steps; ++s) {
    wait_loads();
    __syncthreads();  // this step's tile is whole, the other one has no readers left
    if (s + 1 < steps) fetch((s + 1) * kBK, (s + 1) & 1);
    const E *m = tile[s & 1];
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      V8 xf[kFt], wf[kFn];
#pragma unroll
      for (int i = 0; i < kFt; ++i) {
        const int row = wt + 16 * i + col;
        xf[i] = *reinterpret_cast<const V8 *>(m + row * kBK +
                                              ((ks * 4 + quad) ^ ((row >> 1) & 7)) * 8);
      }
#pragma unroll
      for (int j = 0; j < kFn; ++j) {
        const int row = kT + wn + 16 * j + col;
        wf[j] = *reinterpret_cast<const V8 *>(m + row * kBK +
                                              ((ks * 4 + quad) ^ ((row >> 1) & 7)) * 8);
      }
#pragma unroll
      for (int j = 0; j < kFn; ++j)
#pragma unroll
        for (int i = 0; i < kFt; ++i) acc[j][i] = N::mfma16(wf[j], xf[i], acc[j][i]);
    }
  }
  if (P.adapter) add_adapters<kType, kFn, kFt>(P, t0 + wt, n0 + wn, acc);
  store<kType, kFn, kFt>(P, t0 + wt, n0 + wn, acc);
}

template <int kType>
int launch(const tg_project_args *a, ProjectParams P, hipStream_t s) {
  if (P.adapter)
    hipLaunchKernelGGL(shrink_kernel<kType>, dim3((P.n_tokens + 15) / 16), dim3(kShrinkThreads),
                       0, s, P);
  const int64_t tiles_t = (int64_t(P.n_tokens) + 127) / 128;
  P.tiles_n = (P.n + 127) / 128;
  if (tiles_t * P.tiles_n > INT32_MAX) return TG_E_INVAL;
  hipLaunchKernelGGL((project_kernel<kType, 128, 128, 2, 2>),
                     dim3(static_cast<uint32_t>(tiles_t * P.tiles_n)), dim3(256), 0, s, P);
  return hipGetLastError() == hipSuccess ? TG_OK : TG_E_HIP;
}

int pad_rank(int rank) { return (rank + 15) / 16 * 16; }

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
  return a->type == TG_F16 ? launch<TG_F16>(a, P, s) : launch<TG_BF16>(a, P, s);
}
