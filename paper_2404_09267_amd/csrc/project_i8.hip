// tg_project_i8: a projection in 8-bit integers, y = (x_scale w_scale) (x w^T), sums exact in 32
// bits.
//
// Few tokens: reading w bounds it. A workgroup takes 16 outputs and 16 tokens, its waves parts of k
// in turn, straight from memory to the matrix instructions' registers, and the waves' sums are
// joined through LDS: one launch, no workspace.
//
// Many tokens: tiles of x and w go through LDS to the matrix instructions, several steps of 128
// values of k under way; how fast they get there bounds it (the matrix units are at work 64 % of
// the time). bfloat16: 25,600 x 4,096, k 4,096: 346 to 369 us by card, 2.33 to 2.48 POPS (a
// library's product, which gives sums of 32 bits, 420; its best at any size 2.5 POPS); 8,192 x
// 8,192, k 8,192: 414 to 425, 2.6; 8 x 1,536, k 1,024: 3.5 to 3.9, a launch. Between them one round
// of small tiles hardly fills the pipeline: 3,500 x 2,048, k 2,048 20, 1.5; 512 x 4,096, k 4,096
// 14, 1.2. Rows of y that do not start on 16 bytes take stores of 8 that straddle lines: 22,333 x
// 2,565, k 144 58, 40 where they are 2,592 apart.
//
// Results lie transposed in the registers (a lane holds 4 outputs of one token), so that stores are
// contiguous and a token's scale belongs to the lane. Both operands take the same values of k in
// the same places, so that the order within an instruction does not matter.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <cstdint>

#include "tg.h"
#include "token_math.h"

namespace {

using namespace tok;

constexpr int kMaxStride = 1 << 22, kMaxRows = 1 << 30;

struct ProjectParams {
  const int8_t *x, *w;
  const float *x_scale, *w_scale;
  void *y;
  int64_t x_stride, w_stride, y_stride;
  int32_t n_tokens, k, n;
  int32_t tiles_t, tiles_n;
  int32_t y_on16, y_on64;  // rows of y start on 16, or 64 bytes
  int32_t whole;  // tiles of 256 x 256 that are taken whole, and
  int32_t first;  // workgroups that take them, one after the other
};

__device__ __forceinline__ i32x4 mfma(i32x4 a, i32x4 b, i32x4 c) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0);
}

// Scales of the tokens and outputs that a lane has results of; of the nearest inside where it has
// none.
__device__ __forceinline__ float scale_of(const ProjectParams &P, int t) {
  return P.x_scale[min(t, P.n_tokens - 1)];
}
__device__ __forceinline__ f32x4 scales_of(const ProjectParams &P, int n) {
  f32x4 v;
#pragma unroll
  for (int r = 0; r < 4; ++r) v[r] = P.w_scale[min(n + r, P.n - 1)];
  return v;
}

// 4 outputs of one token, from n on.
template <int kType>
__device__ __forceinline__ void put(const ProjectParams &P, int t, int n, i32x4 sum, float xs,
                                    f32x4 ws) {
  typedef typename Num<kType>::E E;
  typedef typename Num<kType>::V4 V4;
  if (t >= P.n_tokens || n >= P.n) return;
  E *to = static_cast<E *>(P.y) + int64_t(t) * P.y_stride + n;
  f32x4 v;
#pragma unroll
  for (int r = 0; r < 4; ++r) v[r] = static_cast<float>(sum[r]) * (xs * ws[r]);
  const V4 out = __builtin_convertvector(v, V4);
  if (n + 3 < P.n) {  // as they lie: rows may start anywhere
    __builtin_memcpy(to, &out, sizeof(out));
  } else {
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (n + r < P.n) to[r] = out[r];
  }
}

// The same of two blocks of 16 outputs where rows of y start on 16 bytes, 8 outputs a lane: lanes
// of odd rows of 16 give the first block's for the second's of the row before, so that a token's 64
// bytes are stored at once (25,600 x 4,096, k 4,096: 368 -> 355 us), and where those are whole
// lines' halves past the caches (6,400 x 1,536, k 1,024: 18.0 -> 14.5, through the caches 16.8; but
// 4,000 x 1,000, whose rows start elsewhere, 9.7 for 8.6). Unaligned stores of 16 bytes are slower
// than those of 8 (1,777 x 2,051, k 1,168: 13.1 for 12.7).
template <int kType>
__device__ __forceinline__ void put_pair(const ProjectParams &P, int t, int n0, i32x4 one,
                                         i32x4 two, float xs, f32x4 ws_one, f32x4 ws_two) {
  typedef typename Num<kType>::E E;
  typedef typename Num<kType>::V4 V4;
  typedef typename Num<kType>::V8 V8;
  const int quad = (threadIdx.x & 63) >> 4;
  f32x4 a, b;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    a[r] = static_cast<float>(one[r]) * (xs * ws_one[r]);
    b[r] = static_cast<float>(two[r]) * (xs * ws_two[r]);
  }
  const i32x2 pa = __builtin_bit_cast(i32x2, __builtin_convertvector(a, V4));
  const i32x2 pb = __builtin_bit_cast(i32x2, __builtin_convertvector(b, V4));
  const auto lo = __builtin_amdgcn_permlane16_swap(pa[0], pb[0], false, false);
  const auto hi = __builtin_amdgcn_permlane16_swap(pa[1], pb[1], false, false);
  const i32x4 bits = {static_cast<int>(lo[0]), static_cast<int>(hi[0]), static_cast<int>(lo[1]),
                      static_cast<int>(hi[1])};
  const V8 out = __builtin_bit_cast(V8, bits);
  const int n = n0 + 16 * (quad & 1) + 8 * (quad >> 1);
  if (t >= P.n_tokens) return;
  E *to = static_cast<E *>(P.y) + int64_t(t) * P.y_stride + n;
  if (n + 7 < P.n) {
    if (P.y_on64) {
      asm volatile("");  // or the compiler makes one store of the two, through the caches
      __builtin_nontemporal_store(out, reinterpret_cast<V8 *>(to));
      asm volatile("");
    } else {
      *reinterpret_cast<V8 *>(to) = out;
    }
  } else {
#pragma unroll
    for (int r = 0; r < 8; ++r)
      if (n + r < P.n) to[r] = out[r];
  }
}

// ------------------------------------------------------------------------------ few tokens

constexpr int kFewWaves = 8;

// 16 tokens x 16 outputs a workgroup; a wave takes every kFewWaves-th 512 values of k, all of whose
// loads are under way at once.
template <int kType>
__global__ __launch_bounds__(kFewWaves * 64) void few_kernel(const ProjectParams P) {
  constexpr int kAhead = 8;  // instructions' values of k that are loaded at once
  __shared__ i32x4 s_sum[kFewWaves][64];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, quad = lane >> 4;
  const int id = workgroup();
  const int n0 = id % P.tiles_n * 16, t0 = id / P.tiles_n * 16;
  const int8_t *w = P.w + int64_t(min(n0 + col, P.n - 1)) * P.w_stride;
  const int8_t *x = P.x + int64_t(min(t0 + col, P.n_tokens - 1)) * P.x_stride;
  i32x4 acc = {};
  const float xs = scale_of(P, t0 + col);
  const f32x4 ws = scales_of(P, n0 + 4 * quad);
  for (int k0 = wave * 64 * kAhead; k0 < P.k; k0 += kFewWaves * 64 * kAhead) {
    i32x4 wv[kAhead], xv[kAhead];
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      const int c = k0 + a * 64 + quad * 16;
      const bool in = c < P.k;
      wv[a] = in ? *reinterpret_cast<const i32x4 *>(w + c) : i32x4{};
      xv[a] = in ? *reinterpret_cast<const i32x4 *>(x + c) : i32x4{};
    }
#pragma unroll
    for (int a = 0; a < kAhead; ++a) acc = mfma(wv[a], xv[a], acc);
  }
  s_sum[wave][lane] = acc;
  __syncthreads();
  if (wave > 0) return;
  i32x4 sum = {};
#pragma unroll
  for (int v = 0; v < kFewWaves; ++v) sum += s_sum[v][lane];
  put<kType>(P, t0 + col, n0 + 4 * quad, sum, xs, ws);
}

// ----------------------------------------------------------------------------- many tokens

// A tile of kT tokens x kN outputs, kWt x kWn waves, 128 values of k a step, kStages steps of loads
// under way. The next 64 values' operands are read from LDS while these are multiplied, so that the
// matrix units have work across the barrier; the buffer of step s is free for step s + kStages
// behind the barrier at the end of it, since its operands are in registers by then. Rows of a
// tile lie in LDS as 8 chunks of 16 bytes, in an order in which one chunk of 16 rows, which is
// what the operands' reads ask for, falls on all banks.
// Steps of 64 values with 4 or 5 of them under way are slower (25,600 x 4,096, k 4,096: 453 and 442
// us for 411), 4 waves of 128 x 128 far slower (589).
constexpr int kBK = 128;
__device__ __forceinline__ int place_of(int row, int c) { return c ^ ((row >> 1) & 7); }

// Which tile a workgroup takes: workgroups go round the 8 XCDs, so each XCD gets a run of tiles of
// its own, in blocks of kGroup token tiles by all output tiles, whose operands its L2 shares.
constexpr int kXcds = 8, kGroup = 4;
__device__ __forceinline__ void tile_at(int k, int tiles_t, int tiles_n, int &tt, int &tn) {
  const int per = kGroup * tiles_n, g = k / per, in = k - g * per;
  const int rows = min(kGroup, tiles_t - g * kGroup);
  tt = g * kGroup + in % rows;
  tn = in / rows;
}
__device__ __forceinline__ int run_of(int id, int total) {
  const int each = total / kXcds, more = total % kXcds, x = id % kXcds;
  return x * each + min(x, more) + id / kXcds;
}

template <int kT, int kN, int kStages>
constexpr int kLds = kStages *(kT + kN) * kBK;

// `next` puts the workgroup's next tile in its arguments, or is false; that tile's first steps are
// then loaded under the last steps of this one, and its first operands read before this one's
// results are stored. There are kStages steps or more then. A tile's first loads so wait neither
// for a workgroup to start nor for results: 25,600 x 4,096, k 1,024: 123 -> 117 us, 22,333 x 2,560,
// k 256: 45 -> 41, of 2,565 with k 144 68 -> 61; k 4,096 the same.
template <int kType, int kT, int kN, int kWt, int kWn, int kStages, class Next>
__device__ __forceinline__ void tiles(const ProjectParams &P, int t0, int n0, int8_t *lds,
                                      const Next &next) {
  constexpr int kWaves = kWt * kWn, kFt = kT / kWt / 16, kFn = kN / kWn / 16;
  constexpr int kChunks = kBK / 16, kRows = kT + kN, kPer = 64 / kChunks;  // rows of one load
  constexpr int kLoads = kRows / kPer / kWaves;
  static_assert(kLoads * kPer * kWaves == kRows && kT % kPer == 0, "whole loads");
  static_assert(kWaves * kPer % 16 == 0, "rows of one lane");
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, quad = lane >> 4;
  // Rows past the tensor lie past the buffer's end, since a row is at most as long as its stride.
  const auto x_rows = [&](int t) {
    const int rows = min(kT, P.n_tokens - t);
    return buffer(P.x + t * P.x_stride, static_cast<uint32_t>((rows - 1) * P.x_stride + P.k));
  };
  const auto w_rows = [&](int n) {
    const int rows = min(kN, P.n - n);
    return buffer(P.w + n * P.w_stride, static_cast<uint32_t>((rows - 1) * P.w_stride + P.k));
  };
  auto xb = x_rows(t0), wb = w_rows(n0);
  // load i of a wave covers kPer rows. A lane's chunk is the same in all loads, since their rows
  // are a multiple of 16 apart.
  const int chunk = place_of(wave * kPer + lane / kChunks, lane % kChunks);
  uint32_t at[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int row = (i * kWaves + wave) * kPer + lane / kChunks;
    at[i] = row < kT ? static_cast<uint32_t>(row * P.x_stride + chunk * 16)
                     : static_cast<uint32_t>((row - kT) * P.w_stride + chunk * 16);
  }
  const int steps = (P.k + kBK - 1) / kBK;
  int turn = 0;  // step s is in buffer (turn + s) % kStages
  // every step's loads are issued, past the last one too, so that they can be counted
  auto fetch = [&](int s, int k0) {
    const bool past = k0 + chunk * 16 >= P.k;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int first = (i * kWaves + wave) * kPer;
      load_lds(first < kT ? xb : wb, lds + ((turn + s) % kStages * kRows + first) * kBK,
               past ? kNowhere : at[i], static_cast<uint32_t>(k0));
    }
  };
  i32x4 acc[kFn][kFt] = {};
  const int wt = (wave % kWt) * (kT / kWt), wn = (wave / kWt) * (kN / kWn);
  // the scales first where registers allow, so that nothing waits for them at the end
  constexpr bool kEarly = kFt * kFn <= 16;
  float xs[kFt];
  f32x4 ws[kFn];
  auto scales = [&] {
#pragma unroll
    for (int i = 0; i < kFt; ++i) xs[i] = scale_of(P, t0 + wt + 16 * i + col);
#pragma unroll
    for (int j = 0; j < kFn; ++j) ws[j] = scales_of(P, n0 + wn + 16 * j + 4 * quad);
  };
  if (kEarly) scales();
  struct Operands {  // of 64 values of k
    i32x4 x[kFt], w[kFn];
  };
  auto read = [&](Operands &o, int s, int ks) {
    const int8_t *m = lds + (turn + s) % kStages * kRows * kBK;
#pragma unroll
    for (int i = 0; i < kFt; ++i) {
      const int row = wt + 16 * i + col;
      o.x[i] = *reinterpret_cast<const i32x4 *>(m + row * kBK + place_of(row, ks * 4 + quad) * 16);
    }
#pragma unroll
    for (int j = 0; j < kFn; ++j) {
      const int row = kT + wn + 16 * j + col;
      o.w[j] = *reinterpret_cast<const i32x4 *>(m + row * kBK + place_of(row, ks * 4 + quad) * 16);
    }
  };
  auto multiply = [&](const Operands &o) {
#pragma unroll
    for (int j = 0; j < kFn; ++j)
#pragma unroll
      for (int i = 0; i < kFt; ++i) acc[j][i] = mfma(o.w[j], o.x[i], acc[j][i]);
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
#pragma unroll
  for (int s = 0; s < kStages; ++s) fetch(s, s * kBK);
  wait_and_meet<(kStages - 1) * kLoads>();
  Operands now, then;
  read(now, 0, 0);
  for (bool again = false;;) {
    int t1 = t0, n1 = n0;
    const bool more = next(t1, n1);
    for (int s = 0; s < steps; ++s) {
      // `now` has the first 64 values of step s, and is left with those of step s + 1
      read(then, s, 1);
      multiply(now);
      interleave(false);
      // step s + 1 is here, step s in registers; of another tile than the first, its first two
      // steps are, and only stores are under way
      if (again && s == 0) wait_and_meet<63>();
      else wait_and_meet<(kStages - 2) * kLoads>();
      int k0 = (s + kStages) * kBK;
      if (more && s + kStages >= steps) {
        k0 -= steps * kBK;
        if (k0 == 0) {
          xb = x_rows(t1);
          wb = w_rows(n1);
        }
      }
      fetch(s + kStages, k0);
      read(now, s + 1, 0);
      multiply(then);
      interleave(true);
    }
    if (!kEarly) scales();
    wait_loads();  // the next tile's, or LDS belongs to the next workgroup from here on
#pragma unroll
    for (int i = 0; i < kFt; ++i) {
      const int t = t0 + wt + 16 * i + col, n = n0 + wn;
      if (kFn % 2 == 0 && P.y_on16) {
#pragma unroll
        for (int j = 0; j + 1 < kFn; j += 2)
          put_pair<kType>(P, t, n + 16 * j, acc[j][i], acc[j + 1][i], xs[i], ws[j], ws[j + 1]);
      } else {
#pragma unroll
        for (int j = 0; j < kFn; ++j)
          put<kType>(P, t, n + 16 * j + 4 * quad, acc[j][i], xs[i], ws[j]);
      }
    }
    if (!more) return;
    t0 = t1;
    n0 = n1;
    turn = (turn + steps) % kStages;
    again = true;
#pragma unroll
    for (int j = 0; j < kFn; ++j)
#pragma unroll
      for (int i = 0; i < kFt; ++i) acc[j][i] = i32x4{};
    if (kEarly) scales();
  }
}

struct OneTile {
  __device__ bool operator()(int &, int &) const { return false; }
};

template <int kType, int kT, int kN, int kWt, int kWn, int kStages>
__global__ __launch_bounds__(kWt *kWn * 64, 2) void tile_kernel(const ProjectParams P) {
  __shared__ __attribute__((aligned(16))) int8_t lds[kLds<kT, kN, kStages>];
  int tt, tn;
  tile_at(run_of(blockIdx.x, P.tiles_t * P.tiles_n), P.tiles_t, P.tiles_n, tt, tn);
  tiles<kType, kT, kN, kWt, kWn, kStages>(P, tt * kT, tn * kN, lds, OneTile());
}

// Tiles of 256 x 256, one a CU; those past the last whole round of the CUs by quarters, so that a
// round of few tiles does not take as long as a whole one. All 256 registers are in use, and 8
// bytes a lane go to scratch.
template <int kType>
__global__ __launch_bounds__(512, 2) void tile_and_rest_kernel(const ProjectParams P) {
  __shared__ __attribute__((aligned(16))) int8_t lds[kLds<256, 256, 2>];
  static_assert(kLds<128, 128, 4> <= kLds<256, 256, 2>, "one LDS for both");
  int id = blockIdx.x, tt, tn;
  if (id < P.first) {
    tile_at(run_of(id, P.whole), P.tiles_t, P.tiles_n, tt, tn);
    return tiles<kType, 256, 256, 2, 4, 2>(P, tt * 256, tn * 256, lds, [&](int &t, int &n) {
      id += P.first;
      if (id >= P.whole) return false;
      tile_at(run_of(id, P.whole), P.tiles_t, P.tiles_n, tt, tn);
      t = tt * 256;
      n = tn * 256;
      return true;
    });
  }
  id -= P.first;  // quarters of one tile on one XCD
  const int k = P.whole + id % kXcds + id / (4 * kXcds) * kXcds, quarter = id / kXcds % 4;
  if (k >= P.tiles_t * P.tiles_n) return;
  tile_at(k, P.tiles_t, P.tiles_n, tt, tn);
  const int t0 = tt * 256 + quarter % 2 * 128, n0 = tn * 256 + quarter / 2 * 128;
  if (t0 < P.n_tokens && n0 < P.n) tiles<kType, 128, 128, 2, 4, 4>(P, t0, n0, lds, OneTile());
}

// ------------------------------------------------------------------------------- the host

constexpr int kCus = 256;

// Tiles of 256 x 256 past the whole rounds, where quarters of them fit the CUs.
int64_t rest_of(int64_t tiles) {
  const int64_t rest = tiles % kCus;
  return tiles > kCus && rest <= kCus / 4 ? rest : 0;
}

template <int kType, int kT, int kN, int kWt, int kWn, int kStages>
int launch_tiles(ProjectParams P, hipStream_t s) {
  const int64_t tiles_t = (int64_t(P.n_tokens) + kT - 1) / kT;
  const int64_t tiles_n = (int64_t(P.n) + kN - 1) / kN;
  int64_t blocks = tiles_t * tiles_n;
  constexpr bool kRest = kT == 256 && kN == 256;
  const int64_t rest = kRest ? rest_of(blocks) : 0;
  P.whole = static_cast<int32_t>(std::min<int64_t>(blocks - rest, INT32_MAX));
  if (rest > 0) blocks += (rest + kXcds - 1) / kXcds * kXcds * 4 - rest;
  // threads that a launch takes in one direction
  if (blocks * (kWt * kWn * 64) >= int64_t(1) << 32) return TG_E_INVAL;
  // steps of two tiles are under way at once where a tile has two
  P.first = kRest && P.k > kBK ? std::min(P.whole, kCus) : P.whole;
  blocks -= P.whole - P.first;
  P.tiles_t = static_cast<int32_t>(tiles_t);
  P.tiles_n = static_cast<int32_t>(tiles_n);
  const dim3 grid(static_cast<uint32_t>(blocks)), threads(kWt * kWn * 64);
  if constexpr (kRest)
    hipLaunchKernelGGL(tile_and_rest_kernel<kType>, grid, threads, 0, s, P);
  else
    hipLaunchKernelGGL((tile_kernel<kType, kT, kN, kWt, kWn, kStages>), grid, threads, 0, s, P);
  return hipGetLastError() == hipSuccess ? TG_OK : TG_E_HIP;
}

template <int kType>
int launch_few(ProjectParams P, hipStream_t s) {
  const int64_t tiles_t = (int64_t(P.n_tokens) + 15) / 16;
  P.tiles_n = static_cast<int32_t>((int64_t(P.n) + 15) / 16);
  if (tiles_t * P.tiles_n > kMaxWorkgroups) return TG_E_INVAL;
  hipLaunchKernelGGL(few_kernel<kType>, grid_of(tiles_t * P.tiles_n, kFewWaves * 64),
                     dim3(kFewWaves * 64), 0, s, P);
  return hipGetLastError() == hipSuccess ? TG_OK : TG_E_HIP;
}

// Few tokens go without LDS as long as their rows, which every 16 outputs read again, are less than
// the weights are worth: 16 x 4,096, k 4,096 5.5 us for 8.0 with tiles of 64 x 32, 64 x 1,536, k
// 1,024 3.9 for 4.4, but 32 x 4,096, k 4,096 10.2 for 8.3 and 16 x 8,192, k 8,192 16.7 for 13.4.
template <int kType>
int launch(const ProjectParams &P, hipStream_t s) {
  const int64_t weights = int64_t(P.n) * P.k;
  if ((P.n_tokens <= 16 && weights <= 1 << 25) || (P.n_tokens <= 64 && weights <= 1 << 21))
    return launch_few<kType>(P, s);
  const auto tiles = [&](int t, int n) {
    return ((int64_t(P.n_tokens) + t - 1) / t) * ((int64_t(P.n) + n - 1) / n);
  };
  // Large problems take the tile with the least time for its rounds of workgroups, one or two a CU;
  // a round of 192 x 128, 160 x 128, 192 x 256 and 256 x 256 takes 0.75, 1.13, 1.28 and 1.60 times
  // one of 128 x 128, the quarters that are left of 256 x 256 0.70. Fewer tiles than CUs: one a CU,
  // by 8 waves with more steps under way, and smaller ones where few even of those would be busy.
  // Measured (bfloat16, us; with results through the caches, 4 to 18 % more than now) with tiles of
  // 256 x 256, 192 x 256, 160 x 128, 128 x 128, 192 x 128, and one a CU 128 x 128, 128 x 64, 64 x
  // 64, 64 x 32:
  //   25,600 x 4,096, k 4,096: 411, 439, 449, 476
  //    8,192 x 8,192, k 4,096: 253,  -,   -,  338, 292
  //    6,400 x 1,536, k 1,024:  27,  23,  21,  26,   -,  27, 25, 27
  //    5,000 x 1,536, k 4,096:  53,   -,  41,  37,  50,  38, 42
  //    3,202 x 1,560, k 3,232:  48,   -,  37,  36,  27,  40, 37
  //    2,917 x 1,320, k 1,600:  30,   -,  19,  17,  16,  13, 15
  //    1,777 x 2,051, k 1,168:   -,  27,  19,   -,  18,  14, 15, 17, 21
  //      512 x 4,096, k 4,096:   -,  40,  28,   -,   -,  19, 15, 17, 22
  //    1,000 x 1,024, k 2,048:   -,  26,  19,   -,   -,  12, 10,  7,  8
  //      300 x   300, k 4,096:   -,  39,  25,   -,   -,  17, 13, 10,  8
  if (tiles(128, 128) > kCus) {
    const auto rounds = [&](int t, int n, int at_once) {
      return (tiles(t, n) + at_once - 1) / at_once;
    };
    const int64_t t256 = tiles(256, 256), rest = rest_of(t256);
    const int64_t c256 = 160 * ((t256 - rest + kCus - 1) / kCus) + (rest ? 70 : 0);
    const int64_t c192 = 128 * rounds(192, 256, kCus), half = 75 * rounds(192, 128, kCus);
    const int64_t c160 = 113 * rounds(160, 128, 2 * kCus), c128 = 100 * rounds(128, 128, 2 * kCus);
    const int64_t least = std::min({c256, c192, half, c160, c128});
    if (c256 == least) return launch_tiles<kType, 256, 256, 2, 4, 2>(P, s);
    if (c192 == least) return launch_tiles<kType, 192, 256, 4, 2, 2>(P, s);
    if (half == least) return launch_tiles<kType, 192, 128, 4, 2, 3>(P, s);
    if (c160 == least) return launch_tiles<kType, 160, 128, 2, 2, 2>(P, s);
    return launch_tiles<kType, 128, 128, 2, 2, 2>(P, s);
  }
  if (tiles(128, 128) >= 160) return launch_tiles<kType, 128, 128, 2, 4, 4>(P, s);
  if (tiles(64, 64) > kCus) return launch_tiles<kType, 128, 64, 2, 2, 3>(P, s);
  if (tiles(64, 64) > kCus / 2) return launch_tiles<kType, 64, 64, 2, 4, 4>(P, s);
  return launch_tiles<kType, 64, 32, 2, 2, 4>(P, s);
}

}  // namespace

extern "C" int tg_project_i8(const tg_project_i8_args *a, void *stream) {
  if (!a || a->n_tokens < 0 || a->k < 16 || a->k > TG_PROJECT_I8_MAX_K || a->k % 16 || a->n < 1 ||
      a->n_tokens > kMaxRows || a->n > kMaxRows || !type_ok(a->type))
    return TG_E_INVAL;
  if (a->x_stride < a->k || a->w_stride < a->k || a->y_stride < a->n || a->x_stride % 16 ||
      a->w_stride % 16 || a->x_stride > kMaxStride || a->w_stride > kMaxStride)
    return TG_E_INVAL;
  if (a->n_tokens == 0) return TG_OK;
  if (!a->x || !a->w || !a->y || !a->x_scale || !a->w_scale || !aligned16(a->x) ||
      !aligned16(a->w))
    return TG_E_INVAL;
  ProjectParams P = {};
  P.x = a->x;
  P.w = a->w;
  P.x_scale = a->x_scale;
  P.w_scale = a->w_scale;
  P.y = a->y;
  P.x_stride = a->x_stride;
  P.w_stride = a->w_stride;
  P.y_stride = a->y_stride;
  P.y_on16 = aligned16(a->y) && a->y_stride % 8 == 0;
  P.y_on64 = reinterpret_cast<uintptr_t>(a->y) % 64 == 0 && a->y_stride % 32 == 0;
  P.n_tokens = a->n_tokens;
  P.k = a->k;
  P.n = a->n;
  hipStream_t s = static_cast<hipStream_t>(stream);
  return a->type == TG_F16 ? launch<TG_F16>(P, s) : launch<TG_BF16>(P, s);
}
