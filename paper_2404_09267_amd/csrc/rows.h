// What the operators that take a row at a time share: a row's values in registers, 8 a chunk, of R
// threads a row, and sums over a row.
#pragma once

#include "token_math.h"

namespace tok {

// Threads of a workgroup: rows of 16 lanes or a wave each, or one row.
template <int R>
constexpr int kGroupThreads = R <= 64 ? 256 : R;

template <int kType>
using Chunk = typename Num<kType>::V8;

// A chunk is 8 / W pieces of W values that follow each other, as many as n and where rows start
// allow to load at once. Place in the row of value e of this thread's chunk i: the row's threads
// have pieces that follow each other.
template <int R, int W>
__device__ __forceinline__ int place_in_row(int i, int e) {
  return ((i * (8 / W) + e / W) * R + threadIdx.x % R) * W + e % W;
}

// Chunk i of a row; zeros past n. kStream: past the caches.
template <int kType, int R, int W, bool kStream = false>
__device__ __forceinline__ Chunk<kType> load_chunk(const typename Num<kType>::E *row, int i,
                                                   int n) {
  typedef typename Num<kType>::E Piece __attribute__((ext_vector_type(W)));
  Chunk<kType> v = {};
#pragma unroll
  for (int e = 0; e < 8; e += W) {
    const int c = place_in_row<R, W>(i, e);
    const auto *p = reinterpret_cast<const Piece *>(row + c);
    Piece piece = {};
    if (c < n) piece = kStream ? __builtin_nontemporal_load(p) : *p;
#pragma unroll
    for (int f = 0; f < W; ++f) v[e + f] = piece[f];
  }
  return v;
}

template <int kType, int R, int W, bool kStream = false>
__device__ __forceinline__ void store_chunk(typename Num<kType>::E *row, int i, int n,
                                            Chunk<kType> v) {
  typedef typename Num<kType>::E Piece __attribute__((ext_vector_type(W)));
#pragma unroll
  for (int e = 0; e < 8; e += W) {
    const int c = place_in_row<R, W>(i, e);
    Piece piece;
#pragma unroll
    for (int f = 0; f < W; ++f) piece[f] = v[e + f];
    auto *p = reinterpret_cast<Piece *>(row + c);
    if (c >= n) continue;
    if constexpr (kStream) __builtin_nontemporal_store(piece, p);
    else *p = piece;
  }
}

// 8, 4 or 1: the values of `size` bytes that can be loaded at once from rows at `p`, `stride`
// apart; `w`: what other rows allow. By 2 is slower than by 1 (a norm of 25,600 x 2,002: 172 us for
// 101; by 4 90, of 2,000 by 8 78).
inline int piece_of(int w, const void *p, int64_t stride, int size) {
  while (w > 1 && (reinterpret_cast<uintptr_t>(p) % (w * size) || stride % w)) w = w == 8 ? 4 : 1;
  return w;
}

// v of the lane that kCtrl says (1, 2, 4 or 8 before in a row of 16, or the last of the row or of
// the half before), 0 where there is none.
template <int kCtrl, int kRows>
__device__ __forceinline__ uint32_t before(uint32_t v) {
  return __builtin_amdgcn_update_dpp(0u, v, kCtrl, kRows, 0xF, false);
}

// Sum over the wave, in all lanes and in a set order; without LDS, whose six round trips a row
// of few values would wait for.
__device__ __forceinline__ float lanes_sum(float v) {
  const auto bits = [](float x) { return __builtin_bit_cast(uint32_t, x); };
  const auto value = [](uint32_t x) { return __builtin_bit_cast(float, x); };
  v += value(before<0x111, 0xF>(bits(v)));
  v += value(before<0x112, 0xF>(bits(v)));
  v += value(before<0x114, 0xF>(bits(v)));
  v += value(before<0x118, 0xF>(bits(v)));
  v += value(before<0x142, 0xA>(bits(v)));
  v += value(before<0x143, 0xC>(bits(v)));
  return value(__builtin_amdgcn_readlane(bits(v), 63));
}

__device__ __forceinline__ uint32_t lanes_max(uint32_t v) {
  v = max(v, before<0x111, 0xF>(v));
  v = max(v, before<0x112, 0xF>(v));
  v = max(v, before<0x114, 0xF>(v));
  v = max(v, before<0x118, 0xF>(v));
  v = max(v, before<0x142, 0xA>(v));
  v = max(v, before<0x143, 0xC>(v));
  return __builtin_amdgcn_readlane(v, 63);
}

// v of the lane 1 or 2 away, or of the mirrored lane among 8 or 16: the four of them together go
// over 16 lanes, in an order that is the same for all.
template <int kStep>
__device__ __forceinline__ uint32_t across(uint32_t v) {
  constexpr int kCtrl[4] = {0xB1, 0x4E, 0x141, 0x140};
  return __builtin_amdgcn_update_dpp(0u, v, kCtrl[kStep], 0xF, 0xF, false);
}

// Sum and largest over 16 lanes, in all of them.
__device__ __forceinline__ float sum16(float v) {
  const auto bits = [](float x) { return __builtin_bit_cast(uint32_t, x); };
  const auto value = [](uint32_t x) { return __builtin_bit_cast(float, x); };
  v += value(across<0>(bits(v)));
  v += value(across<1>(bits(v)));
  v += value(across<2>(bits(v)));
  v += value(across<3>(bits(v)));
  return v;
}

__device__ __forceinline__ uint32_t max16(uint32_t v) {
  v = max(v, across<0>(v));
  v = max(v, across<1>(v));
  v = max(v, across<2>(v));
  return max(v, across<3>(v));
}

// Sum over the R threads of a row, in all of them and in a set order. `turn`: LDS of this sum's
// own.
template <int R>
__device__ __forceinline__ float row_sum(float v, float *turn) {
  if constexpr (R == 16) return sum16(v);
  v = lanes_sum(v);
  if constexpr (R > 64) {
    if ((threadIdx.x & 63) == 0) turn[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0f;
#pragma unroll
    for (int w = 0; w < R / 64; ++w) v += turn[w];
  }
  return v;
}

}  // namespace tok
