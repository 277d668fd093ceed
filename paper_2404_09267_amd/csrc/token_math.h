// What the token operators share: the two 16-bit types, their matrix instructions, and loads
// that go from memory to LDS without passing through registers.
//
// Operand layouts of the matrix instructions used here, for lane l of a wave:
//   16x16x32: A row l % 16, B column l % 16, both with k = 8 (l / 16) + 0..7; result register r
//             is row 4 (l / 16) + r, column l % 16.
//   32x32x16: A row l % 32, B column l % 32, both with k = 8 (l / 32) + 0..7; result register r
//             is row 8 (r / 4) + 4 (l / 32) + r % 4, column l % 32.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "tg.h"

namespace tok {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int32_t i32x2 __attribute__((ext_vector_type(2)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

template <int kType>
struct Num;

template <>
struct Num<TG_F16> {
  typedef _Float16 E;
  typedef E V2 __attribute__((ext_vector_type(2)));
  typedef E V4 __attribute__((ext_vector_type(4)));
  typedef E V8 __attribute__((ext_vector_type(8)));
  static __device__ __forceinline__ f32x4 mfma16(V8 a, V8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x16 mfma32(V8 a, V8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
};

template <>
struct Num<TG_BF16> {
  typedef __bf16 E;
  typedef E V2 __attribute__((ext_vector_type(2)));
  typedef E V4 __attribute__((ext_vector_type(4)));
  typedef E V8 __attribute__((ext_vector_type(8)));
  static __device__ __forceinline__ f32x4 mfma16(V8 a, V8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x16 mfma32(V8 a, V8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
};

// Two values rounded to nearest-even, as one register.
template <int kType>
__device__ __forceinline__ typename Num<kType>::V2 pack2(float a, float b) {
  const f32x2 v = {a, b};
  return __builtin_convertvector(v, typename Num<kType>::V2);
}

// Memory as a buffer: reads past `bytes` give zero. The offset of a read that must give zero
// is kNowhere, beyond every buffer made here (bytes < 2^31).
constexpr uint32_t kNowhere = 0xC0000000u;

__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const void *p, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, bytes, 0x00020000);
}

// 16 bytes per lane from offset + base of the buffer into LDS at `to` + 16 * lane (`to` is the
// same in every lane of the wave). The caller waits (vmcnt) before LDS is read.
__device__ __forceinline__ void load_lds(__amdgpu_buffer_rsrc_t r, void *to, uint32_t offset,
                                         uint32_t base) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(
      r, reinterpret_cast<__attribute__((address_space(3))) void *>(
             reinterpret_cast<uintptr_t>(to)),
      16, offset, base, 0, 0);
}

// The same with 4 bytes per lane, to `to` + 4 * lane.
__device__ __forceinline__ void load_lds4(__amdgpu_buffer_rsrc_t r, void *to, uint32_t offset) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(
      r, reinterpret_cast<__attribute__((address_space(3))) void *>(
             reinterpret_cast<uintptr_t>(to)),
      4, offset, 0, 0, 0);
}

// Waits until at most `left` of the wave's loads are under way.
template <int left = 0>
__device__ __forceinline__ void wait_loads() {
  // vmcnt in bits 0-3 and 14-15; the counters of exports (4-6) and of LDS (8-11) at their most
  __builtin_amdgcn_s_waitcnt((left & 15) | ((left >> 4) << 14) | 0x0F70);
}

// The same, and for the wave's LDS accesses; then the workgroup's barrier. Nothing moves across.
template <int left>
__device__ __forceinline__ void wait_and_meet() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((left & 15) | ((left >> 4) << 14) | 0x0070);
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  return v;
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// `blocks` workgroups: in one row, or in several of kRow where their threads would pass the 2^32
// that a launch takes in one direction. A kernel's own place is workgroup(), which asks for no
// size of the grid (its load adds 0.1 us to a call); the last row may have more than asked for, and
// even those are numbered in 31 bits.
constexpr int kRow = 1 << 20;
constexpr int64_t kMaxWorkgroups = INT32_MAX - kRow;
inline dim3 grid_of(int64_t blocks, int threads) {
  if (blocks * threads < int64_t(1) << 32) return dim3(static_cast<uint32_t>(blocks));
  return dim3(kRow, static_cast<uint32_t>((blocks + kRow - 1) / kRow));
}
__device__ __forceinline__ int workgroup() {
  return static_cast<int>(blockIdx.y * kRow + blockIdx.x);
}

inline bool aligned16(const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }
inline bool type_ok(int32_t t) { return t == TG_F16 || t == TG_BF16; }

}  // namespace tok
