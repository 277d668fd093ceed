// tg_norm: the norm after a block, its gate and the residual, and the norm before the next block.
//
// x and y are read once and the residual and its norm written once, 8 bytes a value, and everything
// between is kept in registers: that is what bounds it (25,600 x 4,096 in bfloat16, gates of 20
// cameras, a layer norm of y and a norm of the result: 157 us, 5.3 TB/s where a large copy reaches
// 4.9; 20 x 1,024: 3.7 us, a launch and two loads in a row). A row is 16 lanes', a wave's or a
// workgroup's, of 128 to 1,024 threads, so that a thread has 8 to 32 values. The variance is of the differences
// from the mean, which costs a second sum over the row but no digits, where sum and sum of squares
// at once would cancel; and what rounding the mean has left is taken off with it, as a row that
// hardly varies would show it (all 1,000: 0.06 for 0).
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "rows.h"
#include "tg.h"

namespace {

using namespace tok;

struct NormParams {
  const void *x, *y, *y_weight, *y_bias, *gate, *weight, *bias;
  void *x_out, *h;
  const int32_t *gate_row;
  int64_t x_stride, y_stride, gate_stride, x_out_stride, h_stride;
  float x_scale, y_scale, eps;
  int32_t y_norm, norm, n_tokens, n, n_gates;
  int32_t stream;  // past the caches
};

// Squares pass binary32 at both ends; such a row is brought near 1 by kFar or 1 / kFar first. Below
// kTiny, what the smallest squares have lost counts where eps does not hide it.
constexpr float kFar = 0x1p80f, kTiny = 0x1p-80f, kHides = 0x1p-60f;

// u of a row to weight * (u [- mean]) / sqrt(mean square + eps) + bias. `turns`: LDS of 6 sums.
template <int kType, int R, int kV, int W>
__device__ __forceinline__ void normalise(const NormParams &P, float (&u)[kV * 8], int kind,
                                          const void *weight, const void *bias,
                                          float (*turns)[16]) {
  typedef typename Num<kType>::E E;
  const int n = P.n;
  const float share = 1.0f / static_cast<float>(n);
  if (kind != TG_NORM_NONE) {
    const bool layer = kind == TG_NORM_LAYER;
    // what each value of the row, and nothing past it, is given to
    const auto each = [&](auto &&take) {
#pragma unroll
      for (int i = 0; i < kV; ++i) {
        if (W == 8 && place_in_row<R, W>(i, 0) >= n) continue;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (W == 8 || place_in_row<R, W>(i, e) < n) take(u[i * 8 + e]);
      }
    };
    const auto mean_of = [&](float up, float *turn) {
      float v = 0.0f;
      each([&](float x) { v += x * up; });
      return row_sum<R>(v, turn) * share;
    };
    // Of the differences from a mean, which is rounded: their mean (what that rounding left), and
    // their mean square less its square.
    const auto spread = [&](auto &&from, float &left, float *turn) {
      float v = 0.0f, w = 0.0f;
      left = 0.0f;
      if (!layer) {
        each([&](float x) {
          const float d = from(x);
          w += d * d;
        });
        return row_sum<R>(w, turn) * share;
      }
      each([&](float x) {
        const float d = from(x);
        v += d;
        w += d * d;
      });
      w = row_sum<R>(w, turn) * share;
      left = row_sum<R>(v, turn + 16) * share;
      // fused: `left` squared may pass binary32 where w does, and inf - inf would come out as 0
      return fmaxf(__builtin_fmaf(-left, left, w), 0.0f);  // of NaN, `left` is NaN
    };
    float left, mean = layer ? mean_of(1.0f, turns[0]) : 0.0f;
    float square = spread([&](float v) { return v - mean; }, left, turns[1]);
    const bool large = !(square < INFINITY) || !(fabsf(left) < INFINITY);
    if (large || (square < kTiny && P.eps < kHides)) {  // the same in the row's threads
      const float up = large ? 1.0f / kFar : kFar, before = large ? up : 1.0f;
      const float after = large ? 1.0f : up;
      if (large) mean = layer ? mean_of(up, turns[3]) : 0.0f;
      square = spread([&](float v) { return (v * before - mean) * after; }, left, turns[4]);
      const float inverse = rsqrtf(square + P.eps * up * up);
#pragma unroll
      for (int i = 0; i < kV * 8; ++i)
        u[i] = ((u[i] * before - mean) * after - left) * inverse;
    } else {
      const float inverse = rsqrtf(square + P.eps), shift = -left * inverse;
#pragma unroll
      for (int i = 0; i < kV * 8; ++i) u[i] = __builtin_fmaf(u[i] - mean, inverse, shift);
    }
  }
#pragma unroll
  for (int i = 0; i < kV; ++i) {
    if (weight) {
      const Chunk<kType> w = load_chunk<kType, R, W>(static_cast<const E *>(weight), i, n);
#pragma unroll
      for (int e = 0; e < 8; ++e) u[i * 8 + e] *= static_cast<float>(w[e]);
    }
    if (bias) {
      const Chunk<kType> b = load_chunk<kType, R, W>(static_cast<const E *>(bias), i, n);
#pragma unroll
      for (int e = 0; e < 8; ++e) u[i * 8 + e] += static_cast<float>(b[e]);
    }
  }
}

// kStream: x, y and the results go past the caches.
template <int kType, int R, int kV, int W, bool kStream>
__global__ __launch_bounds__(kGroupThreads<R>) void norm_kernel(const NormParams P) {
  typedef typename Num<kType>::E E;
  constexpr int kRows = kGroupThreads<R> / R;
  __shared__ float s_turns[R > 64 ? 12 : 1][16];
  const int64_t t = int64_t(workgroup()) * kRows + threadIdx.x / R;
  if (t >= P.n_tokens) return;  // 16 lanes, a whole wave, or the workgroup
  const int n = P.n;
  Chunk<kType> xv[kV];
  const E *x = static_cast<const E *>(P.x) + t * P.x_stride;
#pragma unroll
  for (int i = 0; i < kV; ++i) xv[i] = load_chunk<kType, R, W, kStream>(x, i, n);
  int g = P.y ? 0 : -1;
  if (P.gate_row) g = P.gate_row[t];
  if (P.gate && (g < 0 || g >= P.n_gates)) g = -1;
  float u[kV * 8];
  if (P.y && g >= 0) {
    const E *y = static_cast<const E *>(P.y) + t * P.y_stride;
#pragma unroll
    for (int i = 0; i < kV; ++i) {
      const Chunk<kType> v = load_chunk<kType, R, W, kStream>(y, i, n);
#pragma unroll
      for (int e = 0; e < 8; ++e) u[i * 8 + e] = static_cast<float>(v[e]);
    }
    normalise<kType, R, kV, W>(P, u, P.y_norm, P.y_weight, P.y_bias, s_turns);
    const E *gate = P.gate ? static_cast<const E *>(P.gate) + g * P.gate_stride : nullptr;
#pragma unroll
    for (int i = 0; i < kV; ++i) {
      if (gate) {
        const Chunk<kType> v = load_chunk<kType, R, W>(gate, i, n);
#pragma unroll
        for (int e = 0; e < 8; ++e) u[i * 8 + e] *= static_cast<float>(v[e]);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e)
        u[i * 8 + e] = P.x_scale * static_cast<float>(xv[i][e]) + P.y_scale * u[i * 8 + e];
    }
  } else {
#pragma unroll
    for (int i = 0; i < kV * 8; ++i) u[i] = P.x_scale * static_cast<float>(xv[i / 8][i % 8]);
  }
  const auto put = [&](void *to, int64_t stride) {
    E *row = static_cast<E *>(to) + t * stride;
#pragma unroll
    for (int i = 0; i < kV; ++i) {
      Chunk<kType> v;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = static_cast<E>(u[i * 8 + e]);
      store_chunk<kType, R, W, kStream>(row, i, n, v);
    }
  };
  if (P.x_out) put(P.x_out, P.x_out_stride);
  if (!P.h) return;
  normalise<kType, R, kV, W>(P, u, P.norm, P.weight, P.bias, s_turns + (R > 64 ? 6 : 0));
  put(P.h, P.h_stride);
}

template <int kType, int R, int kV>
int launch_rows(const NormParams &P, int piece, hipStream_t s) {
  constexpr int kThreads = kGroupThreads<R>, kRows = kThreads / R;
  const int64_t blocks = (int64_t(P.n_tokens) + kRows - 1) / kRows;
  if (blocks > kMaxWorkgroups) return TG_E_INVAL;
  const dim3 grid = grid_of(blocks, kThreads), threads(kThreads);
  if (piece == 8 && P.stream)
    hipLaunchKernelGGL((norm_kernel<kType, R, kV, 8, true>), grid, threads, 0, s, P);
  else if (piece == 8)
    hipLaunchKernelGGL((norm_kernel<kType, R, kV, 8, false>), grid, threads, 0, s, P);
  else if (piece == 4)
    hipLaunchKernelGGL((norm_kernel<kType, R, kV, 4, false>), grid, threads, 0, s, P);
  else
    hipLaunchKernelGGL((norm_kernel<kType, R, kV, 1, false>), grid, threads, 0, s, P);
  return hipGetLastError() == hipSuccess ? TG_OK : TG_E_HIP;
}

constexpr int64_t kFew = int64_t(1) << 22;
constexpr int kNarrow = 128;

template <int kType>
int launch(const NormParams &P, int piece, hipStream_t s) {
  // 8 values a thread where there is little to do and latency counts, 16 where there is more, as
  // far as that goes, and no more threads than that takes. Two layer norms, us with 8, 16 and 32
  // values a thread:
  //   20 x 1,024:      4.6,  5.4        64 x 8,192:      5.9,  6.6
  //   3,200 x 1,024:   9.2,  9.7        1,600 x 2,048:   9.8, 10.2
  //   6,400 x 1,024:  14.6, 13.4, 17.6  1,600 x 4,096:  15.5, 14.4
  //   25,600 x 2,048: 91.9, 81.2, 82.7  25,600 x 4,096: 186, 161, 172
  // Up to 256 values 16 lanes a row: 409,600 x 128 89 us, 261 with a wave a row, 14,768 x 19 5.5 for
  // 11.5; with 32 values a lane up to 512, 6,400 x 512 13.3 for 9.2, 102,400 x 512 83 for 89.
  // Over 16,384 values off 16 bytes, 15 to 28 registers go to scratch: a norm alone of 2,000 x 32,768
  // takes 46 us, by 4 values 51, of 32,767 one at a time 61.
  const bool few = int64_t(P.n_tokens) * P.n <= kFew;
  if (P.n <= kNarrow) return launch_rows<kType, 16, 1>(P, piece, s);
  if (P.n <= 2 * kNarrow) return launch_rows<kType, 16, 2>(P, piece, s);
  if (P.n <= 512) return launch_rows<kType, 64, 1>(P, piece, s);
  if (few && P.n <= 1024) return launch_rows<kType, 128, 1>(P, piece, s);
  if (few && P.n <= 2048) return launch_rows<kType, 256, 1>(P, piece, s);
  if (few && P.n <= 4096) return launch_rows<kType, 512, 1>(P, piece, s);
  if (few && P.n <= 8192) return launch_rows<kType, 1024, 1>(P, piece, s);
  if (P.n <= 1024) return launch_rows<kType, 64, 2>(P, piece, s);
  if (P.n <= 2048) return launch_rows<kType, 128, 2>(P, piece, s);
  if (P.n <= 4096) return launch_rows<kType, 256, 2>(P, piece, s);
  if (P.n <= 8192) return launch_rows<kType, 512, 2>(P, piece, s);
  if (P.n <= 16384) return launch_rows<kType, 1024, 2>(P, piece, s);
  return launch_rows<kType, 1024, 4>(P, piece, s);
}

bool kind_ok(int32_t k) { return k >= TG_NORM_NONE && k <= TG_NORM_LAYER; }

}  // namespace

extern "C" int tg_norm(const tg_norm_args *a, void *stream) {
  if (!a || a->n_tokens < 0 || a->n < 1 || a->n > TG_NORM_MAX_N || a->n_gates < 0 ||
      !type_ok(a->type) || !kind_ok(a->y_norm) || !kind_ok(a->norm) || !(a->eps >= 0.0f) ||
      !std::isfinite(a->eps) || !std::isfinite(a->x_scale) || !std::isfinite(a->y_scale))
    return TG_E_INVAL;
  if ((a->gate && (!a->y || a->n_gates < 1)) || (a->gate_row && !a->gate)) return TG_E_INVAL;
  if (a->n_tokens == 0) return TG_OK;
  if (!a->x || (!a->x_out && !a->h)) return TG_E_INVAL;
  int piece = piece_of(8, nullptr, a->n, 2);
  for (const void *v : {a->y_weight, a->y_bias, a->weight, a->bias})
    piece = piece_of(piece, v, 0, 2);
  const void *rows[5] = {a->x, a->y, a->gate, a->x_out, a->h};
  const int64_t strides[5] = {a->x_stride, a->y_stride, a->gate_stride, a->x_out_stride,
                              a->h_stride};
  int64_t arrays = 0;  // of n_tokens rows
  for (int i = 0; i < 5; ++i) {
    if (!rows[i]) continue;
    if (strides[i] < a->n) return TG_E_INVAL;
    piece = piece_of(piece, rows[i], strides[i], 2);
    arrays += i != 2;
  }
  NormParams P = {};
  P.x = a->x;
  P.y = a->y;
  P.y_weight = a->y_weight;
  P.y_bias = a->y_bias;
  P.gate = a->gate;
  P.weight = a->weight;
  P.bias = a->bias;
  P.x_out = a->x_out;
  P.h = a->h;
  P.gate_row = a->gate_row;
  P.x_stride = a->x_stride;
  P.y_stride = a->y_stride;
  P.gate_stride = a->gate_stride;
  P.x_out_stride = a->x_out_stride;
  P.h_stride = a->h_stride;
  P.x_scale = a->x_scale;
  P.y_scale = a->y_scale;
  P.eps = a->eps;
  P.y_norm = a->y_norm;
  P.norm = a->norm;
  P.n_tokens = a->n_tokens;
  P.n = a->n;
  P.n_gates = a->n_gates;
  // against the 256 MB that the last cache holds
  P.stream = arrays * a->n_tokens * a->n * 2 > (int64_t(256) << 20);
  hipStream_t s = static_cast<hipStream_t>(stream);
  return a->type == TG_F16 ? launch<TG_F16>(P, piece, s) : launch<TG_BF16>(P, piece, s);
}
