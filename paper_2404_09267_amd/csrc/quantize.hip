// tg_quantize: rows of 16-bit values to 8-bit integers with a scale each.
//
// A row is read once into registers, its largest magnitude found, and the integers written: 3 bytes
// a value, which bounds it. The integer is that of the exact quotient x / scale. The product with
// the scale's inverse is off by 127 * 2^-23 at most, so only where it lies within kNear of a tie is
// the quotient looked at: x - r scale is exact in binary32 (both are multiples of the scale's last
// bit, and at most as far apart as the scale), and half the scale decides.
// bfloat16, 25,600 x 4,096: 50 us, 6.3 TB/s, as part of it stays in the last cache; 1,777 x 1,160:
// 3.7 us, a launch.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "rows.h"
#include "tg.h"

namespace {

using namespace tok;

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct QuantizeParams {
  const void *x;
  int8_t *q;
  float *scale;
  int64_t x_stride, q_stride;
  int32_t n_rows, k;
  int32_t stream;  // past the caches
};

constexpr float kNear = 4e-5f;
// Scales of bfloat16 rows below 2^-60 come near binary32's end; such a row is taken times 2^64.
constexpr float kSmall = 0x1p-60f, kUp = 0x1p64f;
// Adding it rounds to an integer (|t| < 2^22), which is then in the low bits.
constexpr float kRound = 12582912.0f;

// What a row's values are multiplied by, and the scale to decide ties with.
struct Scale {
  float up, scale, inverse;
};

// Of the largest magnitude's bits: magnitudes order as their bits do, infinity and NaN above all.
template <int kType>
__device__ __forceinline__ Scale scale_of(uint32_t bits, float &out) {
  constexpr uint32_t kInf = kType == TG_F16 ? 0x7C00u : 0x7F80u;
  if (bits >= kInf) {
    out = __builtin_nanf("");
    return {0.0f, 0.0f, 0.0f};
  }
  const float most =
      static_cast<float>(__builtin_bit_cast(typename Num<kType>::E, static_cast<uint16_t>(bits)));
  out = most / 127.0f;
  if (bits == 0) return {0.0f, 0.0f, 0.0f};
  const float up = most < kSmall ? kUp : 1.0f;
  return {up, out * up, 1.0f / (out * up)};
}

__device__ __forceinline__ float decided(float x, float t, const Scale &s) {
  float r = (t + kRound) - kRound;
  const float left = __builtin_fmaf(-r, s.scale, x), half = 0.5f * s.scale;
  const bool odd = __builtin_bit_cast(uint32_t, r + kRound) & 1;
  if (fabsf(left) > half || (fabsf(left) == half && odd)) r += left > 0.0f ? 1.0f : -1.0f;
  return r + kRound;
}

// NaN and infinity times 0 are left out: such rows have integers 0.
__device__ __forceinline__ float lifted(float x, const Scale &s) {
  return s.up == 0.0f ? 0.0f : x * s.up;
}

// The integers of 8 values, each as a float whose low byte it is.
template <int kType>
__device__ __forceinline__ void integers(const Chunk<kType> &v, const Scale &s, float (&r)[8]) {
  float far = 1.0f;  // rows of zeros, and those that are lifted, are not for the short way
  if (s.up == 1.0f) {
    far = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float x = static_cast<float>(v[e]);
      r[e] = __builtin_fmaf(x, s.inverse, kRound);
      far = fmaxf(far, fabsf(__builtin_fmaf(x, s.inverse, -(r[e] - kRound))));
    }
  }
  if (__ballot(far > 0.5f - kNear)) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float a = lifted(static_cast<float>(v[e]), s);
      r[e] = decided(a, a * s.inverse, s);
    }
  }
}

__device__ __forceinline__ uint32_t low_bytes(float a, float b, float c, float d) {
  const auto u = [](float v) { return __builtin_bit_cast(uint32_t, v); };
  const uint32_t lo = __builtin_amdgcn_perm(u(b), u(a), 0x0C0C0400u);
  const uint32_t hi = __builtin_amdgcn_perm(u(d), u(c), 0x04000C0Cu);
  return lo | hi;
}

// Largest over the R threads of a row.
template <int R>
__device__ __forceinline__ uint32_t row_max(uint32_t v, uint32_t *turn) {
  if constexpr (R == 16) return max16(v);
  v = lanes_max(v);
  if constexpr (R > 64) {
    if ((threadIdx.x & 63) == 0) turn[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int w = 0; w < R / 64; ++w) v = max(v, turn[w]);
  }
  return v;
}

template <int kType, int R, int kV, int W, bool kStream>
__global__ __launch_bounds__(kGroupThreads<R>) void quantize_kernel(const QuantizeParams P) {
  typedef typename Num<kType>::E E;
  constexpr int kRows = kGroupThreads<R> / R;
  __shared__ uint32_t s_turn[16];
  const int64_t t = int64_t(workgroup()) * kRows + threadIdx.x / R;
  if (t >= P.n_rows) return;  // 16 lanes, a whole wave, or the workgroup
  const E *x = static_cast<const E *>(P.x) + t * P.x_stride;
  Chunk<kType> v[kV];
#pragma unroll
  for (int i = 0; i < kV; ++i)
    v[i] = load_chunk<kType, R, W, kStream>(x, i, P.k);
  typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
  u16x8 most = {};
#pragma unroll
  for (int i = 0; i < kV; ++i) {
    const u32x4 bits = __builtin_bit_cast(u32x4, v[i]) & 0x7FFF7FFFu;
    most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x8, bits));
  }
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, static_cast<uint32_t>(most[e]));
  float scale;
  const Scale s = scale_of<kType>(row_max<R>(top, s_turn), scale);
  if (threadIdx.x % R == 0) P.scale[t] = scale;
  int8_t *q = P.q + t * P.q_stride;
#pragma unroll
  for (int i = 0; i < kV; ++i) {
    float r[8];
    integers<kType>(v[i], s, r);
    const u32x2 out = {low_bytes(r[0], r[1], r[2], r[3]), low_bytes(r[4], r[5], r[6], r[7])};
    typedef int8_t Bytes __attribute__((ext_vector_type(8)));
    typedef int8_t Piece __attribute__((ext_vector_type(W)));
    const Bytes all = __builtin_bit_cast(Bytes, out);
#pragma unroll
    for (int e = 0; e < 8; e += W) {
      const int c = place_in_row<R, W>(i, e);
      Piece piece;
#pragma unroll
      for (int f = 0; f < W; ++f) piece[f] = all[e + f];
      Piece *to = reinterpret_cast<Piece *>(q + c);
      if (c >= P.k) continue;
      if constexpr (kStream) __builtin_nontemporal_store(piece, to);
      else *to = piece;
    }
  }
}

// Rows longer than registers hold, value by value; the row is read twice. Left simple, as no layer
// here has such rows: 2,000 x 40,000 118 us, 2.4 times what its bytes take at a copy's rate, 200 x
// 100,003 66, 5.4 times (2,000 x 32,768, from registers, 37, 0.93 times).
template <int kType, int R>
__global__ __launch_bounds__(kGroupThreads<R>) void quantize_long_kernel(const QuantizeParams P) {
  typedef typename Num<kType>::E E;
  constexpr int kRows = kGroupThreads<R> / R;
  __shared__ uint32_t s_turn[16];
  const int64_t t = int64_t(workgroup()) * kRows + threadIdx.x / R;
  if (t >= P.n_rows) return;  // a whole wave, or the workgroup
  const int first = threadIdx.x % R;
  const E *x = static_cast<const E *>(P.x) + t * P.x_stride;
  uint32_t top = 0;
  for (int64_t c = first; c < P.k; c += R)
    top = max(top, static_cast<uint32_t>(__builtin_bit_cast(uint16_t, x[c])) & 0x7FFFu);
  float scale;
  const Scale s = scale_of<kType>(row_max<R>(top, s_turn), scale);
  if (first == 0) P.scale[t] = scale;
  int8_t *q = P.q + t * P.q_stride;
  for (int64_t c = first; c < P.k; c += R) {
    const float a = lifted(static_cast<float>(x[c]), s);
    const float r = decided(a, a * s.inverse, s);
    q[c] = static_cast<int8_t>(__builtin_bit_cast(uint32_t, r));
  }
}

template <int R, class Kernel>
int launch_rows(const QuantizeParams &P, Kernel kernel, hipStream_t s) {
  constexpr int kThreads = kGroupThreads<R>, kRows = kThreads / R;
  const int64_t blocks = (int64_t(P.n_rows) + kRows - 1) / kRows;
  if (blocks > kMaxWorkgroups) return TG_E_INVAL;
  hipLaunchKernelGGL(kernel, grid_of(blocks, kThreads), dim3(kThreads), 0, s, P);
  return hipGetLastError() == hipSuccess ? TG_OK : TG_E_HIP;
}

template <int kType, int R, int kV>
int launch_pieces(const QuantizeParams &P, int piece, hipStream_t s) {
  if (piece == 8 && P.stream) return launch_rows<R>(P, quantize_kernel<kType, R, kV, 8, true>, s);
  if (piece == 8) return launch_rows<R>(P, quantize_kernel<kType, R, kV, 8, false>, s);
  if (piece == 4) return launch_rows<R>(P, quantize_kernel<kType, R, kV, 4, false>, s);
  return launch_rows<R>(P, quantize_kernel<kType, R, kV, 1, false>, s);
}

constexpr int kLongest = 32768;  // of a row that is kept in registers
constexpr int kNarrow = 128;

template <int kType>
int launch(const QuantizeParams &P, int piece, hipStream_t s) {
  if (P.k > kLongest) return launch_rows<1024>(P, quantize_long_kernel<kType, 1024>, s);
  // 16 values a thread, as far as that goes. us with 8, 16 and 32:
  //   20 x 8,192:      3.5,  3.3,  4.1  1,600 x 2,048:  3.9,  4.1,  4.8
  //   25,600 x 1,024: 14.9, 13.7, 15.6  25,600 x 2,048: 31.5, 28.9, 29.4
  //   25,600 x 4,096: 58.7, 49.6, 49.9  25,600 x 8,192:  119, 95.9, 98.6
  // Up to 256 values 16 lanes a row: 409,600 x 128 31 us, 88 with a wave a row; with 32 values a lane
  // up to 512, 25,600 x 512 9.2 for 8.6, 102,400 x 333 35 for 29.
  if (P.k <= kNarrow) return launch_pieces<kType, 16, 1>(P, piece, s);
  if (P.k <= 2 * kNarrow) return launch_pieces<kType, 16, 2>(P, piece, s);
  if (P.k <= 512) return launch_pieces<kType, 64, 1>(P, piece, s);
  if (P.k <= 1024) return launch_pieces<kType, 64, 2>(P, piece, s);
  if (P.k <= 2048) return launch_pieces<kType, 128, 2>(P, piece, s);
  if (P.k <= 4096) return launch_pieces<kType, 256, 2>(P, piece, s);
  if (P.k <= 8192) return launch_pieces<kType, 512, 2>(P, piece, s);
  if (P.k <= 16384) return launch_pieces<kType, 1024, 2>(P, piece, s);
  return launch_pieces<kType, 1024, 4>(P, piece, s);
}

}  // namespace

extern "C" int tg_quantize(const tg_quantize_args *a, void *stream) {
  if (!a || a->n_rows < 0 || a->k < 1 || !type_ok(a->type) || a->x_stride < a->k ||
      a->q_stride < a->k)
    return TG_E_INVAL;
  if (a->n_rows == 0) return TG_OK;
  if (!a->x || !a->q || !a->scale) return TG_E_INVAL;
  QuantizeParams P = {};
  P.x = a->x;
  P.q = a->q;
  P.scale = a->scale;
  P.x_stride = a->x_stride;
  P.q_stride = a->q_stride;
  P.n_rows = a->n_rows;
  P.k = a->k;
  // against the 256 MB that the last cache holds
  P.stream = int64_t(a->n_rows) * a->k * 3 > (int64_t(256) << 20);
  const int piece = piece_of(piece_of(piece_of(8, nullptr, a->k, 2), a->x, a->x_stride, 2), a->q,
                             a->q_stride, 1);
  hipStream_t s = static_cast<hipStream_t>(stream);
  return a->type == TG_F16 ? launch<TG_F16>(P, piece, s) : launch<TG_BF16>(P, piece, s);
}
