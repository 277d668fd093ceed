// tg_rotate: norm and position rotation of queries and keys, per head, in one pass.
//
// A head's d values are divided by their root mean square and multiplied by a weight; then
// pairs of the leading `rot` values turn by an angle that belongs to the token's position (the
// rotary embedding of Su et al. 2021, with a table of cosines and sines, so that the angle of a
// far position is as exact as the caller made it). Two axes give half of the pairs each: the x
// and y of a token on its frame.
//
// Nothing is reused but the table's row, so memory bounds it: a head is read once into
// registers, and written once, past the caches where they could not keep it (131,072 tokens, 18
// heads of 128, 1.2 GB in and out: 291 us, 4.2 TB/s where a large copy reaches 4.85; through the
// caches 313). Lanes hold 2 x 8 values, the two chunks whose values are each other's partners, so
// that a turn needs no exchange between lanes; the sum of squares is the only one. A wave takes a
// token and goes over its heads, which share the table's row; where a token's heads do not fill a
// wave it takes several tokens, and with few tokens the heads are spread over waves instead (20
// tokens, 24 heads: 4 us, a launch).
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "tg.h"
#include "token_math.h"

namespace {

using namespace tok;

constexpr int kThreads = 256;
constexpr int kMaxD = 512;

struct RotateParams {
  const void *in[3];        // q, k, v
  void *out[3];
  int64_t in_stride[3], in_head[3], out_stride[3], out_head[3];
  const void *weight[2];
  const float *table;
  const int32_t *pos;
  const int64_t *slot;
  int64_t n_rows;
  float eps;
  int32_t n_tokens, n_heads, n_kv_heads, d, rot, axes, n_positions;
  int32_t rows;             // heads of a token, over q, k and v
  int32_t passes;           // waves of a token, each takes rows / passes heads in turn
  int32_t lanes;            // lanes of a head, a power of two
  int32_t at_once;          // heads of a token that a wave takes at once, a power of two
};

// Which tensor (0 q, 1 k, 2 v) head row `r` of a token is in; r becomes the head there.
__device__ __forceinline__ int tensor_of(const RotateParams &P, int &r) {
  if (r < P.n_heads) return 0;
  r -= P.n_heads;
  if (r < P.n_kv_heads) return 1;
  r -= P.n_kv_heads;
  return 2;
}

__device__ __forceinline__ const float *table_row(const RotateParams &P, int64_t t, int pair) {
  const int half = P.rot >> 1;
  const int axis = P.axes == 2 && 2 * pair >= half ? 1 : 0;
  const int p = min(max(P.pos[t * P.axes + axis], 0), P.n_positions - 1);
  return P.table + (int64_t(p) * half + pair) * 2;
}

// Row of the output for token t, -1 for none.
__device__ __forceinline__ int64_t out_row(const RotateParams &P, int which, int64_t t) {
  if (which == 0 || !P.slot) return t;
  const int64_t r = P.slot[t];
  return r >= 0 && r < P.n_rows ? r : -1;
}

// 1 / sqrt(mean square + eps) of a head. Where the sum of squares has left binary32 it is formed
// from `small`, that of the values times kDown, as ordinary bfloat16 can be so large.
constexpr float kDown = 0x1p-70f;
__device__ __forceinline__ float inverse_norm(const RotateParams &P, float sum, float small) {
  const float d = static_cast<float>(P.d);
  if (sum < INFINITY) return rsqrtf(sum / d + P.eps);
  return rsqrtf(small / d + P.eps * kDown * kDown) * kDown;
}

// d a multiple of 16, rows and heads on 16-byte boundaries. Lane c of a head holds values 8 c ..
// and their partners rot / 2 later (half pairs, rot a multiple of 16), or values 16 c .. where
// pairs are neighbours.
template <int kType, bool kInterleaved, bool kStream>
__global__ __launch_bounds__(kThreads) void rotate_kernel(const RotateParams P) {
  typedef Num<kType> N;
  typedef typename N::E E;
  typedef typename N::V8 V8;
  const int64_t unit = int64_t(workgroup()) * (kThreads / 64) + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, sub = lane & (P.lanes - 1);
  const int slot = lane / P.lanes, step = P.at_once;
  // a wave has several tokens where one has fewer heads than the wave has room for
  const int64_t several = unit / P.passes;
  const int pass = static_cast<int>(unit - several * P.passes);
  const int64_t t = several * (64 / P.lanes / step) + slot / step;
  if (t >= P.n_tokens) return;
  const bool has = sub < P.d / 16;
  const bool turns = sub * 16 < P.rot;
  const bool part = P.rot % 16 != 0;  // a lane may hold pairs that turn and others
  int c0, c1;  // first values of the two chunks
  if (kInterleaved || !turns) {
    c0 = 16 * sub;
    c1 = c0 + 8;
  } else {
    c0 = 8 * sub;
    c1 = c0 + P.rot / 2;
  }
  float cs[8][2] = {};
  if (turns) {
    const int pair = kInterleaved ? c0 / 2 : c0;
    // the lane's 8 pairs are all turned, and on one axis
    if (P.rot % 16 == 0 && (P.axes == 1 || P.rot % 32 == 0)) {
      const f32x4 *row = reinterpret_cast<const f32x4 *>(table_row(P, t, pair));
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x4 v = row[i];
        cs[2 * i][0] = v[0], cs[2 * i][1] = v[1], cs[2 * i + 1][0] = v[2], cs[2 * i + 1][1] = v[3];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (2 * (pair + i) < P.rot) {
          const float *row = table_row(P, t, pair + i);
          cs[i][0] = row[0], cs[i][1] = row[1];
        }
      }
    }
  }
  for (int first = pass * step; first < P.rows; first += P.passes * step) {
    int h = first + (slot & (step - 1));
    const bool use = has && h < P.rows;
    const int which = use ? tensor_of(P, h) : 0;
    V8 a = {}, b = {};
    if (use) {
      const E *p = static_cast<const E *>(P.in[which]) + t * P.in_stride[which] +
                   h * P.in_head[which];
      const V8 *pa = reinterpret_cast<const V8 *>(p + c0);
      const V8 *pb = reinterpret_cast<const V8 *>(p + c1);
      a = kStream ? __builtin_nontemporal_load(pa) : *pa;
      b = kStream ? __builtin_nontemporal_load(pb) : *pb;
    }
    float u[16], sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      u[i] = static_cast<float>(a[i]);
      u[8 + i] = static_cast<float>(b[i]);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) sum += u[i] * u[i];
    for (int o = P.lanes >> 1; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    float small = sum;
    if (kType == TG_BF16 && __ballot(!(sum < INFINITY))) {
      small = 0.0f;
#pragma unroll
      for (int i = 0; i < 16; ++i) small += (u[i] * kDown) * (u[i] * kDown);
      for (int o = P.lanes >> 1; o > 0; o >>= 1) small += __shfl_xor(small, o);
    }
    if (!use) continue;
    const int64_t row = out_row(P, which, t);
    if (row < 0) continue;
    E *to = static_cast<E *>(P.out[which]) + row * P.out_stride[which] + h * P.out_head[which];
    if (which < 2) {
      const float inv = inverse_norm(P, sum, small);
      V8 wa, wb;
      const E *w = static_cast<const E *>(P.weight[which]);
      if (w) {
        wa = *reinterpret_cast<const V8 *>(w + c0);
        wb = *reinterpret_cast<const V8 *>(w + c1);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) wa[i] = wb[i] = static_cast<E>(1.0f);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        u[i] *= inv * static_cast<float>(wa[i]);
        u[8 + i] *= inv * static_cast<float>(wb[i]);
      }
      // a pair that does not turn stays as it is: 0 times an infinite partner would be NaN
      if (turns) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int x = kInterleaved ? 2 * i : i, y = kInterleaved ? 2 * i + 1 : 8 + i;
          const float p = u[x] * cs[i][0] - u[y] * cs[i][1];
          const float q = u[x] * cs[i][1] + u[y] * cs[i][0];
          if (kInterleaved && part && 2 * (8 * sub + i) >= P.rot) continue;
          u[x] = p;
          u[y] = q;
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        a[i] = static_cast<E>(u[i]);
        b[i] = static_cast<E>(u[8 + i]);
      }
    }
    V8 *ta = reinterpret_cast<V8 *>(to + c0), *tb = reinterpret_cast<V8 *>(to + c1);
    if (kStream) {
      __builtin_nontemporal_store(a, ta);
      __builtin_nontemporal_store(b, tb);
    } else {
      *ta = a;
      *tb = b;
    }
  }
}

// Any even d, any alignment: a wave takes one head, lane l pairs l, l + 64, ...
template <int kType>
__global__ __launch_bounds__(kThreads) void rotate_any_kernel(const RotateParams P,
                                                              int interleaved) {
  typedef typename Num<kType>::E E;
  const int64_t unit = int64_t(workgroup()) * (kThreads / 64) + (threadIdx.x >> 6);
  const int64_t t = unit / P.rows;
  if (t >= P.n_tokens) return;
  int h = static_cast<int>(unit - t * P.rows);
  const int which = tensor_of(P, h);
  const int lane = threadIdx.x & 63, half = P.rot >> 1;
  const E *p = static_cast<const E *>(P.in[which]) + t * P.in_stride[which] +
               h * P.in_head[which];
  constexpr int kMost = kMaxD / 128;  // pairs a lane may hold
  E va[kMost], vb[kMost];
  float sum = 0.0f, small = 0.0f;
#pragma unroll
  for (int k = 0; k < kMost; ++k) {
    const int i = lane + 64 * k;
    if (2 * i < P.d) {
      const bool split = i < half && !interleaved;
      const int x = split ? i : 2 * i, y = split ? i + half : 2 * i + 1;
      va[k] = p[x];
      vb[k] = p[y];
      const float fa = static_cast<float>(va[k]), fb = static_cast<float>(vb[k]);
      sum += fa * fa + fb * fb;
      small += (fa * kDown) * (fa * kDown) + (fb * kDown) * (fb * kDown);
    }
  }
  sum = wave_sum(sum);
  if (!(sum < INFINITY)) small = kType == TG_BF16 ? wave_sum(small) : sum;  // in every lane
  const int64_t row = out_row(P, which, t);
  if (row < 0) return;
  E *to = static_cast<E *>(P.out[which]) + row * P.out_stride[which] + h * P.out_head[which];
  const float inv = inverse_norm(P, sum, small);
  const E *w = which < 2 ? static_cast<const E *>(P.weight[which]) : nullptr;
#pragma unroll
  for (int k = 0; k < kMost; ++k) {
    const int i = lane + 64 * k;
    if (2 * i < P.d) {
      const bool split = i < half && !interleaved;
      const int x = split ? i : 2 * i, y = split ? i + half : 2 * i + 1;
      if (which == 2) {
        to[x] = va[k];
        to[y] = vb[k];
        continue;
      }
      const float fa = static_cast<float>(va[k]) * inv * (w ? static_cast<float>(w[x]) : 1.0f);
      const float fb = static_cast<float>(vb[k]) * inv * (w ? static_cast<float>(w[y]) : 1.0f);
      if (i >= half) {
        to[x] = static_cast<E>(fa);
        to[y] = static_cast<E>(fb);
        continue;
      }
      const float *r = table_row(P, t, i);
      to[x] = static_cast<E>(fa * r[0] - fb * r[1]);
      to[y] = static_cast<E>(fa * r[1] + fb * r[0]);
    }
  }
}

template <int kType>
void launch_vec(const RotateParams &P, bool interleaved, dim3 grid, hipStream_t s) {
  // what is read and written, against the 256 MB that the last cache holds
  const bool stream = int64_t(P.n_tokens) * P.rows * P.d * 4 > (int64_t(256) << 20);
  const dim3 threads(kThreads);
  if (interleaved && stream)
    hipLaunchKernelGGL((rotate_kernel<kType, true, true>), grid, threads, 0, s, P);
  else if (interleaved)
    hipLaunchKernelGGL((rotate_kernel<kType, true, false>), grid, threads, 0, s, P);
  else if (stream)
    hipLaunchKernelGGL((rotate_kernel<kType, false, true>), grid, threads, 0, s, P);
  else
    hipLaunchKernelGGL((rotate_kernel<kType, false, false>), grid, threads, 0, s, P);
}

bool on16(const void *p, int64_t stride, int64_t head) {
  return aligned16(p) && stride % 8 == 0 && head % 8 == 0;
}

}  // namespace

extern "C" int tg_rotate(const tg_rotate_args *a, void *stream) {
  if (!a || a->n_tokens < 0 || a->n_heads < 0 || a->n_kv_heads < 0) return TG_E_INVAL;
  if (!type_ok(a->type) || a->d < 2 || a->d > kMaxD || a->d % 2 || a->rot < 0 ||
      a->rot > a->d || a->rot % 2 || (a->axes != 1 && a->axes != 2) || !(a->eps >= 0.0f) ||
      !std::isfinite(a->eps))
    return TG_E_INVAL;
  if (a->rot > 0 && a->n_positions < 1) return TG_E_INVAL;
  if (a->slot && a->n_rows < 0) return TG_E_INVAL;
  if ((a->v == nullptr) != (a->v_out == nullptr)) return TG_E_INVAL;
  if (a->n_tokens == 0 || (a->n_heads == 0 && a->n_kv_heads == 0)) return TG_OK;
  if (a->n_heads > 0 && (!a->q || !a->q_out)) return TG_E_INVAL;
  if (a->n_kv_heads > 0 && (!a->k || !a->k_out)) return TG_E_INVAL;
  if (a->rot > 0 && (!a->table || !a->pos)) return TG_E_INVAL;
  const int64_t rows = int64_t(a->n_heads) + (a->v ? 2 : 1) * int64_t(a->n_kv_heads);
  if (rows > (1 << 20)) return TG_E_INVAL;

  RotateParams P = {};
  const void *in[3] = {a->q, a->k, a->v}, *out[3] = {a->q_out, a->k_out, a->v_out};
  const int64_t is[3] = {a->q_stride, a->k_stride, a->v_stride};
  const int64_t ih[3] = {a->q_head_stride, a->k_head_stride, a->v_head_stride};
  const int64_t os[3] = {a->q_out_stride, a->k_out_stride, a->v_out_stride};
  const int64_t oh[3] = {a->q_out_head_stride, a->k_out_head_stride, a->v_out_head_stride};
  bool vec = a->d % 16 == 0 && (a->rot % 16 == 0 || a->interleaved) && aligned16(a->table) &&
             aligned16(a->q_weight) && aligned16(a->k_weight);
  for (int i = 0; i < 3; ++i) {
    P.in[i] = in[i];
    P.out[i] = const_cast<void *>(out[i]);
    P.in_stride[i] = is[i];
    P.in_head[i] = ih[i];
    P.out_stride[i] = os[i];
    P.out_head[i] = oh[i];
    if (i == 0 ? a->n_heads > 0 : in[i] != nullptr && a->n_kv_heads > 0)
      vec = vec && on16(in[i], is[i], ih[i]) && on16(out[i], os[i], oh[i]);
  }
  P.weight[0] = a->q_weight;
  P.weight[1] = a->k_weight;
  P.table = a->table;
  P.pos = a->pos;
  P.slot = a->slot;
  P.n_rows = a->n_rows;
  P.eps = a->eps;
  P.n_tokens = a->n_tokens;
  P.n_heads = a->n_heads;
  P.n_kv_heads = a->n_kv_heads;
  P.d = a->d;
  P.rot = a->rot;
  P.axes = a->axes;
  P.n_positions = a->n_positions;
  P.rows = static_cast<int32_t>(rows);
  hipStream_t s = static_cast<hipStream_t>(stream);
  constexpr int kWaves = kThreads / 64;
  if (vec) {
    P.lanes = 1;
    while (P.lanes < a->d / 16) P.lanes *= 2;
    const int room = 64 / P.lanes;
    P.at_once = 1;
    while (P.at_once < room && P.at_once < P.rows) P.at_once *= 2;
    const int most = (P.rows + P.at_once - 1) / P.at_once;
    P.passes = a->n_tokens < 4096 ? most : 1;
    const int per = room / P.at_once;  // tokens of a wave
    const int64_t waves = (int64_t(a->n_tokens) + per - 1) / per * P.passes;
    const int64_t blocks = (waves + kWaves - 1) / kWaves;
    if (blocks > kMaxWorkgroups) return TG_E_INVAL;
    const dim3 grid = grid_of(blocks, kThreads);
    if (a->type == TG_F16)
      launch_vec<TG_F16>(P, a->interleaved != 0, grid, s);
    else
      launch_vec<TG_BF16>(P, a->interleaved != 0, grid, s);
  } else {
    const int64_t blocks = (int64_t(a->n_tokens) * P.rows + kWaves - 1) / kWaves;
    if (blocks > kMaxWorkgroups) return TG_E_INVAL;
    const dim3 grid = grid_of(blocks, kThreads);
    const int inter = a->interleaved != 0;
    if (a->type == TG_F16)
      hipLaunchKernelGGL(rotate_any_kernel<TG_F16>, grid, dim3(kThreads), 0, s, P, inter);
    else
      hipLaunchKernelGGL(rotate_any_kernel<TG_BF16>, grid, dim3(kThreads), 0, s, P, inter);
  }
  return hipGetLastError() == hipSuccess ? TG_OK : TG_E_HIP;
}
