// tg_attend_pages: attention of one new token a sequence over the pages of a cache.
//
// The query heads that share a key head are rows of one matrix tile, so that keys and values are
// read once, and reading them bounds it: each wave has a tile of 32 keys and their values under way
// to LDS while it works on the one before. A key's row in the cache is looked up by a lane, a tile
// ahead of its loads. Tiles whose keys are all seen are loaded by runs of rows; in the others
// rows that are not seen (past the end, before the window, on a page that is none) are loaded from
// zeros instead, so that whatever lies there stays out, and have no weight.
//
// Softmax in one pass over the keys (Milakov and Gimelshein 2018): a running maximum m in units of
// log2, the sum l of 2^(z - m) and the weighted sum of values, the latter two multiplied by
// 2^(m_old - m_new) when a score passes m by kSlack. Scores are computed transposed, S^T = K Q^T,
// so that a lane's scores are of one query and the weights come out where the second product, O^T =
// V^T P^T, takes them as an operand. That product takes 16-bit operands; where values of both signs
// cancel, weights of 8 or 11 bits would show long before the result's own rounding does, so they
// go in as two parts, a rounding and, rounded too, what that leaves. Up to 8 query heads a key head
// leave half the tile's columns free, and those take the second part of the same heads (20 sequences
// of 1,600, 16 heads of 64 over 4: 12.6 -> 13.2 us for it, 8 of 100,003 the same 107); more heads
// take a second product (8 of 60,000, 32 heads of 128 over 1: 39 -> 44; the paired columns would
// read keys once for every 8).
//
// Few keys, or many sequences: a workgroup a sequence and key head. Else all sequences' keys are
// cut into as many ranges of one length as there is room for workgroups, found on the device, so
// that each has as much to read whatever the lengths are; a workgroup goes from sequence to
// sequence, and join_kernel joins what a sequence has in several ranges, in a set order. bfloat16:
// 8 sequences of up to 100,003 keys, 16 heads of 128 over 2, 583 MB: 107 to 111 us, 5.3 TB/s; 256
// of up to 4,096, 32 heads over 8, 2.4 GB: 440 to 467 us by card, 5.1 to 5.4; 20 of up to 1,600, 16
// heads of 64 over 4: 13.4 us with a cap and 10.6 without, a launch and a chain of loads (length,
// pages, keys, and those of 6 tiles a wave) and of what each tile is put through.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <climits>
#include <cmath>
#include <cstdint>

#include "tg.h"
#include "token_math.h"

namespace {

using namespace tok;

constexpr int kMaxStride = 1 << 22, kMaxKeys = 1 << 30;
constexpr float kSlack = 8.0f;
// Weights are kept times 2^kLift: binary16's smallest number is 2^-24, and what lies below 2^-25 of
// the largest weight, of a second part too, would be lost, however many such keys there are. With kSlack they reach
// 2^15, which binary16 holds.
template <int kType>
constexpr float kLift = kType == TG_F16 ? 7.0f : 0.0f;
constexpr float kLog2e = 1.4426950408889634f;

struct AttendParams {
  const void *q, *k, *v;
  void *out;
  int64_t q_stride, q_head, k_stride, k_head, v_stride, v_head, out_stride, out_head;
  int64_t table_stride;
  const int32_t *table, *kv_len, *q_begin;
  const float *slope;
  float to_log2;   // scale * log2(e): a raw score's factor
  float cap_arg;   // scale / cap
  float cap_out;   // cap * log2(e), 0: no cap
  int32_t window, n_seqs, n_q_rows, n_pages, page_size;
  int32_t page_log2;  // of page_size, -1: it is no power of two
  int32_t most;    // keys of a sequence at most
  int32_t n_heads, n_kv_heads, group, d;
  int32_t row_tiles;
  int32_t near;    // workgroups of a sequence or range go to one XCD
  int32_t width;   // ranges that all keys are cut into at most, 0: a workgroup a sequence
  int32_t least;   // tiles of a range at least; a multiple of
  int32_t unit;    // the tiles that a workgroup takes at once
  float *part;     // [width + n_seqs][n_heads][d] weighted sums, and
  float *part_ml;  // [..][..][2] maximum (log2 units) and sum of weights
};

// A sequence's query and its keys; no row, no keys where it has no query.
struct Query {
  int row, keys;
};

__device__ __forceinline__ Query query_of(const AttendParams &P, int s) {
  Query r = {s, P.kv_len[s]};
  if (P.q_begin) {
    const int begin = P.q_begin[s], end = P.q_begin[s + 1];
    r.row = end > begin && end > 0 && end <= P.n_q_rows ? end - 1 : -1;
  }
  r.keys = r.row < 0 ? 0 : max(r.keys, 0);
  return r;
}

// Keys [lo, hi) of a sequence are seen by its query; a tile has 32 keys from a multiple of 32 on.
struct Span {
  int lo, hi;
};

__device__ __forceinline__ Span span_of(const AttendParams &P, int len) {
  Span r;
  r.hi = min(max(len, 0), P.most);
  // the query stands at the last key there is, whatever of them is left out at the end
  r.lo = P.window > 0 && len > P.window ? min(len - P.window, r.hi) : 0;
  return r;
}

// tanh(x) in binary32: the quotient where 1 and 2 / (1 + e^2x) hardly cancel, else the series x -
// x^3 / 3 + 2 x^5 / 15 - 17 x^7 / 315. Off by 2.1e-7 at most, which is 1.7e-6 of it just above 1 / 8
// and less on; below 1 / 8 by 9e-8 of it (exponential and reciprocal off by a last bit each, either
// way).
__device__ __forceinline__ float bend(float x) {
  const float e = __builtin_amdgcn_exp2f(x * (2.0f * kLog2e));
  const float z = __builtin_fmaf(-2.0f, __builtin_amdgcn_rcpf(1.0f + e), 1.0f);
  const float x2 = x * x;
  const float p = __builtin_fmaf(
      x2, __builtin_fmaf(x2, __builtin_fmaf(x2, -17.0f / 315, 2.0f / 15), -1.0f / 3), 1.0f);
  return fabsf(x) < 0.125f ? x * p : z;
}

// a[0] + a[1] + c of two values of the type.
template <int kType>
__device__ __forceinline__ float add2(typename Num<kType>::V2 a, float c);
template <>
__device__ __forceinline__ float add2<TG_F16>(Num<TG_F16>::V2 a, float c) {
  const Num<TG_F16>::V2 one = {static_cast<_Float16>(1.0f), static_cast<_Float16>(1.0f)};
  return __builtin_amdgcn_fdot2(a, one, c, false);
}
template <>
__device__ __forceinline__ float add2<TG_BF16>(Num<TG_BF16>::V2 a, float c) {
  const Num<TG_BF16>::V2 one = {static_cast<__bf16>(1.0f), static_cast<__bf16>(1.0f)};
  return __builtin_amdgcn_fdot2_f32_bf16(a, one, c, false);
}

// What the second product takes of four blocks of 16 of d and 32 keys: transposing reads at the
// four places, and kHigh bytes further for the upper 16 keys. They wait for themselves: the
// compiler would have them wait for every load to LDS under way, the next tile's too.
template <int kType, int kHigh>
__device__ __forceinline__ void read_transposed(const uint32_t (&at)[4],
                                                typename Num<kType>::V8 (&out)[4]) {
  i32x2 v[8];
  asm volatile(
      "ds_read_b64_tr_b16 %0, %8\n\t"
      "ds_read_b64_tr_b16 %1, %8 offset:%12\n\t"
      "ds_read_b64_tr_b16 %2, %9\n\t"
      "ds_read_b64_tr_b16 %3, %9 offset:%12\n\t"
      "ds_read_b64_tr_b16 %4, %10\n\t"
      "ds_read_b64_tr_b16 %5, %10 offset:%12\n\t"
      "ds_read_b64_tr_b16 %6, %11\n\t"
      "ds_read_b64_tr_b16 %7, %11 offset:%12\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3]), "=&v"(v[4]), "=&v"(v[5]),
        "=&v"(v[6]), "=&v"(v[7])
      : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]), "n"(kHigh)
      : "memory");
#pragma unroll
  for (int b = 0; b < 4; ++b) {
    const i32x4 both = {v[2 * b][0], v[2 * b][1], v[2 * b + 1][0], v[2 * b + 1][1]};
    out[b] = __builtin_bit_cast(typename Num<kType>::V8, both);
  }
}

// 16 bytes per lane, each from its own address, into LDS at `to` + 16 * lane. The caller waits.
__device__ __forceinline__ void gather_lds(uint64_t from, void *to) {
  __builtin_amdgcn_global_load_lds(
      reinterpret_cast<const __attribute__((address_space(1))) void *>(from),
      reinterpret_cast<__attribute__((address_space(3))) void *>(reinterpret_cast<uintptr_t>(to)),
      16, 0, 0);
}

// Waits for the wave's loads; LDS is not read before.
__device__ __forceinline__ void wait_tile() {
  wait_loads();
  asm volatile("" ::: "memory");
}

// Waits for the wave's LDS reads; no load to LDS is issued before.
__device__ __forceinline__ void wait_lds() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// What rows that are not seen are read from.
__device__ const uint32_t kZeros[4] __attribute__((aligned(16))) = {};

// Place of 16-byte chunk c of row r in a tile of rows of kChunks chunks (8 or 16). Matrix
// operands take one chunk of 16 rows at once, transposing reads 2 chunks of 8 rows: both fall on
// 16 different places of the 256 bytes that LDS serves at once.
template <int kChunks>
__device__ __forceinline__ int place_of(int r, int c) {
  if (kChunks == 16) return c ^ (((r & 7) << 1) | ((r >> 3) & 1));
  return c ^ ((((r >> 1) & 3) << 1) | ((r >> 3) & 1));
}

// ------------------------------------------------------------------------ the cut of all keys

constexpr int kKeys = 32;      // of a tile
// Sequences, where any is cut: a wave has them in registers. Of more, a long one among short ones
// is one workgroup's for each key head (one of 100,003 keys, 16 heads of 128 over 2, among 1,024: 150
// us, among 1,025: 544).
constexpr int kMaxCut = 1024;

// All sequences' tiles one after the other are cut into ranges of `length`; a workgroup has one,
// whatever it holds of how many sequences. What range w has of sequence s is part w + s: from one
// part to the next, one of the two grows.
struct Cut {
  int length;  // tiles of a range
  int ranges;  // that there are
  int seq;     // the sequence asked for, and
  int at;      // its first tile
};

__device__ __forceinline__ int tiles_of(const Span &s) {
  return s.hi > s.lo ? (s.hi + kKeys - 1) / kKeys - s.lo / kKeys : 0;
}

// Sum of `v` over the wave's lanes up to and with this one.
__device__ __forceinline__ int sum_up(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);  // the lanes 1, 2, 4 and 8 before
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);  // in a row of 16
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);  // the last of the row before
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);  // the last of the half before
  return v;
}

// `range` >= 0: the first sequence that has a part in that range (a sequence of no keys counts
// where it starts); otherwise sequence `seq`. A wave works it out.
__device__ __forceinline__ Cut find_cut(const AttendParams &P, int range, int seq) {
  const int lane = threadIdx.x & 63;
  constexpr int kEach = kMaxCut / 64, kAtOnce = 4;
  int tiles[kEach], upto[kEach], total = 0;  // of a sequence, and with all before it
#pragma unroll
  for (int u0 = 0; u0 < kEach; u0 += kAtOnce) {
    if (u0 * 64 >= P.n_seqs) continue;
    int len[kAtOnce];  // loads of one turn without a branch between them
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u)
      len[u] = query_of(P, min((u0 + u) * 64 + lane, P.n_seqs - 1)).keys;
#pragma unroll
    for (int u = u0; u < u0 + kAtOnce; ++u) {
      tiles[u] = u * 64 + lane < P.n_seqs ? tiles_of(span_of(P, len[u - u0])) : 0;
      if (u * 64 >= P.n_seqs) continue;
      upto[u] = total + sum_up(tiles[u]);
      total = __builtin_amdgcn_readlane(upto[u], 63);
    }
  }
  Cut r;
  const int even = (total + P.width - 1) / P.width;
  r.length = max((even + P.unit - 1) / P.unit * P.unit, P.least);
  r.ranges = max((total + r.length - 1) / r.length, 1);
  r.seq = -1;
  r.at = 0;
  if (range >= r.ranges) return r;
  const int start = range * r.length;
#pragma unroll
  for (int u = 0; u < kEach; ++u) {
    if (u * 64 >= P.n_seqs || r.seq >= 0) continue;
    const bool in = u * 64 + lane < P.n_seqs;
    const uint64_t here =
        range < 0 ? (seq >= u * 64 && seq < u * 64 + 64 ? 1ull << (seq & 63) : 0)
                  : __ballot(in && (upto[u] > start || (tiles[u] == 0 && upto[u] == start)));
    if (!here) continue;
    const int l = __builtin_amdgcn_readfirstlane(__builtin_ctzll(here));
    r.seq = u * 64 + l;
    r.at = __builtin_amdgcn_readlane(upto[u], l) - __builtin_amdgcn_readlane(tiles[u], l);
  }
  return r;
}

// A result from its sum of weights: a query that sees no key has no maximum, one whose scores are
// all minus infinity the least number as one.
__device__ __forceinline__ float weighted(float sum, float m, float l) {
  return l == 0.0f ? (m == -INFINITY ? 0.0f : NAN) : sum / l;
}

// v of the lane 8 on in a row of 16 lanes, which goes round.
__device__ __forceinline__ float eight_on(float v) {
  const int bits = __builtin_bit_cast(int, v);
  return __builtin_bit_cast(float,
                            __builtin_amdgcn_update_dpp(bits, bits, 0x128, 0xF, 0xF, false));
}

constexpr int kXcds = 8;  // that workgroups go round

// Waves of a SIMD that registers are to have room for: as many as LDS has where keys are not cut.
// Heads of 64 get 4 with 3 asked for (126 registers); asked for 4, more than 8 a key head spill
// two.
constexpr int per_simd(int d, int bufs) { return bufs > 1 ? 1 : d == 64 ? 3 : 2; }

// Rows of a workgroup: 16 query heads that share a key head. Each of its waves takes every
// kWaves-th 32 keys of what the workgroup has of a sequence, through LDS of its own. kPair: 8 heads
// at most, which columns 8 to 15 are once more: they take what the weights' roundings leave.
template <int kType, int kD, int kWaves, int kBufs, bool kPair>
__global__ __launch_bounds__(kWaves * 64, per_simd(kD, kBufs)) void attend_pages_kernel(
    const AttendParams P) {
  typedef Num<kType> N;
  typedef typename N::E E;
  typedef typename N::V4 V4;
  typedef typename N::V8 V8;
  constexpr int kChunks = kD / 8, kSteps = kD / 32, kBlocks = kD / 16;
  constexpr int kPer = 64 / kChunks, kLoads = kKeys / kPer;  // rows of one load, loads of a tile
  constexpr int kRows = kPair ? 8 : 16;
  // keys and values of a step; the waves' sums at the end
  __shared__ __attribute__((aligned(16))) E tile[kWaves][kBufs][2][kKeys * kD];
  __shared__ float s_m[kWaves][16], s_l[kWaves][16];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, quad = lane >> 4;
  int id = workgroup(), xcd = 0;
  if (P.near) {  // those of a sequence or range go to one XCD, whose L2 has what they share
    xcd = id % kXcds;
    id /= kXcds;
  }
  const int kvh = id % P.n_kv_heads;
  id /= P.n_kv_heads;
  const int rt = id % P.row_tiles;
  id /= P.row_tiles;
  if (P.near) id = id * kXcds + xcd;
  // tiles of all sequences that are this workgroup's, and where its first sequence starts
  int seq = id, at_tile = 0, begin_tile = 0, end_tile = INT_MAX;
  bool to_end = false;  // sequences of no keys at the end of all, too
  if (P.width > 0) {
    const Cut cut = find_cut(P, id, -1);
    if (cut.seq < 0) return;
    seq = cut.seq;
    at_tile = cut.at;
    begin_tile = id * cut.length;
    end_tile = begin_tile + cut.length;
    to_end = id == cut.ranges - 1;
  } else if (id >= P.n_seqs) {
    return;
  }
  const uint64_t zeros = reinterpret_cast<uintptr_t>(kZeros);
  const uint64_t k_at = reinterpret_cast<uintptr_t>(static_cast<const E *>(P.k) +
                                                    kvh * P.k_head);
  const uint64_t v_at = reinterpret_cast<uintptr_t>(static_cast<const E *>(P.v) + kvh * P.v_head);
  const uint32_t k_bytes = static_cast<uint32_t>(P.k_stride) * 2;
  const uint32_t v_bytes = static_cast<uint32_t>(P.v_stride) * 2;
  // Lane r of each half of the wave looks after key r of a tile: its page, and its row there.
  auto page_at = [&](const int32_t *table, int j0, int lo, int end) {
    const int j = j0 + (lane & 31);
    const uint32_t at = P.page_log2 >= 0 ? static_cast<uint32_t>(j) >> P.page_log2
                                         : static_cast<uint32_t>(j) / P.page_size;
    return j >= lo && j < end ? table[at] : -1;
  };
  auto row_at = [&](int j0, int page) {
    const uint32_t j = j0 + (lane & 31);
    const uint32_t in = P.page_log2 >= 0 ? j & (P.page_size - 1) : j % P.page_size;
    return static_cast<uint32_t>(page) < static_cast<uint32_t>(P.n_pages)
               ? page * P.page_size + static_cast<int>(in)
               : -1;
  };
  // The loads of a tile's keys or values to LDS. Where all its keys are seen, and pages are whole
  // times kRun rows, that many rows lie one after the other: a lane's place among them stays the
  // same, and only where they start is looked up. Else every lane has addresses of its own. Runs of
  // 8 cost wide heads nothing (33 sequences of 3,001, pages of 24: 17.4 -> 15.5 us), those of 64 5
  // % where pages are of 16 (20 of 1,600: 13.7 for 13.0), which is why pages of 8 and 24 go row by
  // row there (20 of 1,600 without a cap: 12.0 and 12.3, pages of 16 to 64 10.6 to 10.4).
  constexpr int kRun = kD > 64 ? 8 : 16, kRuns = kKeys / kRun;
  uint32_t piece[2][kLoads / 2];
  const auto pieces = [&](uint32_t bytes, uint32_t(&to)[kLoads / 2]) {
#pragma unroll
    for (int i = 0; i < kLoads / 2; ++i) {
      const int r = i * kPer + lane / kChunks;  // of 16
      const int c = place_of<kChunks>(r, lane & (kChunks - 1)) * 8;
      to[i] = c < P.d ? r % kRun * bytes + c * 2 : kNowhere;
    }
  };
  pieces(k_bytes, piece[0]);
  pieces(v_bytes, piece[1]);
  const bool even_pages = P.page_size % kRun == 0;
  int rows[kLoads];
  auto spread = [&](uint32_t all, int row) {
    if (all == 0xFFFFFFFFu && even_pages) {
#pragma unroll
      for (int g = 0; g < kRuns; ++g) rows[g] = __builtin_amdgcn_readlane(row, kRun * g);
      return;
    }
#pragma unroll
    for (int i = 0; i < kLoads; ++i) rows[i] = __shfl(row, i * kPer + lane / kChunks);
  };
  auto fetch = [&](int which, uint32_t all, E *to) {
    const uint64_t base = which ? v_at : k_at;
    const uint32_t bytes = which ? v_bytes : k_bytes;
    if (all == 0xFFFFFFFFu && even_pages) {
#pragma unroll
      for (int g = 0; g < kRuns; ++g) {
        const uint32_t at = __builtin_amdgcn_readfirstlane(rows[g]);
        const auto b = buffer(reinterpret_cast<const void *>(base + uint64_t(at) * bytes),
                              (kRun - 1) * bytes + P.d * 2);
#pragma unroll
        for (int i = g * kLoads / kRuns; i < (g + 1) * kLoads / kRuns; ++i)
          load_lds(b, to + i * kPer * kD, piece[which][i % (kLoads / 2)], 0);
      }
      return;
    }
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int c = place_of<kChunks>(i * kPer + lane / kChunks, lane & (kChunks - 1)) * 8;
      const uint64_t p = base + uint64_t(static_cast<uint32_t>(rows[i])) * bytes + c * 2;
      gather_lds(rows[i] >= 0 && c < P.d ? p : zeros, to + i * kPer * kD);
    }
  };
  E(*const own)[2][kKeys * kD] = tile[wave];
  // where a lane's transposing reads of a tile start
  uint32_t place[kBlocks];
#pragma unroll
  for (int b = 0; b < kBlocks; ++b) {
    const int r = 4 * quad + (col >> 2), c = 2 * b + ((col & 3) >> 1);
    place[b] = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(own[0][1])) +
               (r * kD + place_of<kChunks>(r, c) * 8 + (col & 1) * 4) * sizeof(E);
  }
  constexpr int kStep = kWaves * kKeys;
  const int my = kPair ? col & 7 : rt * 16 + col;  // this lane's row
  const float less = kPair && col < 8 ? 0.0f : -1.0f;  // times a weight's rounding: its second part
  const bool live = my < P.group;
  const int head = kvh * P.group + min(my, P.group - 1);
  const float slope2 = P.slope ? P.slope[head] * kLog2e : 0.0f;
  Query query = query_of(P, seq);
  for (;;) {
    const Span span = span_of(P, query.keys);
    const int tiles = tiles_of(span), last = query.keys - 1, q_row = query.row;
    const int first = max(begin_tile - at_tile, 0);        // of the sequence's tiles, up to
    const int beyond = min(end_tile - at_tile, tiles);
    const bool whole = first == 0 && beyond == tiles;
    const int base_key = span.lo / kKeys * kKeys;
    const int from = base_key + first * kKeys, end = min(base_key + beyond * kKeys, span.hi);
    const bool again = P.width > 0 && seq + 1 < P.n_seqs && (to_end || at_tile + tiles < end_tile);
    if (again) query = query_of(P, seq + 1);
    const int32_t *table = P.table + seq * P.table_stride;
    int j0 = from + wave * kKeys, buf = 0;
    const int page0 = page_at(table, j0, span.lo, end);
    int page = page_at(table, j0 + kStep, span.lo, end);
    const E *qr = static_cast<const E *>(P.q) + max(q_row, 0) * P.q_stride + head * P.q_head;
    V8 qf[kSteps];
#pragma unroll
    for (int k = 0; k < kSteps; ++k) {
      qf[k] = V8{};
      if (live && k * 32 + quad * 8 < P.d)
        qf[k] = *reinterpret_cast<const V8 *>(qr + k * 32 + quad * 8);
    }
    uint32_t seen = 0;
    if (j0 < end) {
      const int row = row_at(j0, page0);
      seen = static_cast<uint32_t>(__ballot(row >= 0));
      spread(seen, row);
      fetch(0, seen, own[0][0]);
      fetch(1, seen, own[0][1]);
    }
    f32x4 acc[kBlocks] = {}, low[kPair ? 1 : kBlocks] = {};
    float m = -INFINITY, l = 0.0f;
    bool any = false;
    for (; j0 < end; j0 += kStep) {
      wait_tile();
      const uint32_t now = seen;
      const bool more = j0 + kStep < end;
      if (more) {
        // nothing may ask for the page before the wait: the tile's loads are older
        asm volatile("" : "+v"(page));
        const int row = row_at(j0 + kStep, page);
        page = page_at(table, j0 + 2 * kStep, span.lo, end);
        seen = static_cast<uint32_t>(__ballot(row >= 0));
        spread(seen, row);
        if (kBufs > 1) {
          fetch(0, seen, own[buf ^ 1][0]);
          fetch(1, seen, own[buf ^ 1][1]);
        }
      }
      const E *tk = own[buf][0];
      f32x4 z[2] = {};
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
          const int r = b * 16 + col;
          const V8 kf = *reinterpret_cast<const V8 *>(
              tk + r * kD + place_of<kChunks>(r, 4 * k + quad) * 8);
          z[b] = N::mfma16(kf, qf[k], z[b]);
        }
      if (kBufs == 1 && more) {
        wait_lds();  // the keys are in registers, or done with
        fetch(0, seen, own[0][0]);
      }
      if (P.cap_out > 0.0f) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          z[e >> 2][e & 3] = P.cap_out * bend(z[e >> 2][e & 3] * P.cap_arg);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e >> 2][e & 3] *= P.to_log2;
      }
      if (P.slope) {
        const int far = last - j0 - 4 * quad;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          z[e >> 2][e & 3] -= slope2 * static_cast<float>(far - ((e >> 2) * 16 + (e & 3)));
      }
      if (now != 0xFFFFFFFFu) {
        const uint32_t mine = now >> (4 * quad);
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (!(mine >> ((e >> 2) * 16 + (e & 3)) & 1)) z[e >> 2][e & 3] = -INFINITY;
      }
      any = any || now != 0;
      float big = -INFINITY;
#pragma unroll
      for (int e = 0; e < 8; ++e) big = fmaxf(big, z[e >> 2][e & 3]);
      if (__ballot(big > m + kSlack)) {
        big = fmaxf(big, __shfl_xor(big, 16));
        big = fmaxf(big, __shfl_xor(big, 32));
        const float to = fmaxf(m, big);
        const float fix = to == m ? 1.0f : __builtin_amdgcn_exp2f(m - to);
        m = to;
        l *= fix;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            acc[b][r] *= fix;
            if (!kPair) low[b][r] *= fix;
          }
      }
      // the difference first: with scores of 2^24 and more the sum of m and kLift would be off
      const float base = m == -INFINITY ? 0.0f : m;
      V8 pf, pl;  // weights, first and second parts; kPair: the one that this column takes
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const float p0 = __builtin_amdgcn_exp2f((z[e >> 2][e & 3] - base) + kLift<kType>);
        const float p1 = __builtin_amdgcn_exp2f((z[e >> 2][(e & 3) + 1] - base) + kLift<kType>);
        auto two = pack2<kType>(p0, p1);
        const auto left = pack2<kType>(__builtin_fmaf(static_cast<float>(two[0]), less, p0),
                                       __builtin_fmaf(static_cast<float>(two[1]), less, p1));
        if (kPair) two = left;
        l = add2<kType>(two, l);
        pf[e] = two[0];
        pf[e + 1] = two[1];
        if (kPair) continue;
        l = add2<kType>(left, l);
        pl[e] = left[0];
        pl[e + 1] = left[1];
      }
#pragma unroll
      for (int b0 = 0; b0 < kBlocks; b0 += 4) {
        uint32_t at[4];
        V8 vf[4];
#pragma unroll
        for (int b = 0; b < 4; ++b) at[b] = place[b0 + b] + buf * 2 * kKeys * kD * sizeof(E);
        read_transposed<kType, 16 * kD * sizeof(E)>(at, vf);
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          acc[b0 + b] = N::mfma16(vf[b], pf, acc[b0 + b]);
          if (!kPair) low[b0 + b] = N::mfma16(vf[b], pl, low[b0 + b]);
        }
      }
      if (more) {
        if (kBufs == 1) fetch(1, seen, own[0][1]);
        buf ^= kBufs - 1;
      }
    }
    // the waves' ranges are joined through LDS
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (kPair) l += eight_on(l);
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) {
      f32x4 more = kPair ? acc[b] : low[b];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        if (kPair) more[r] = eight_on(more[r]);
        // may be an infinite value times 0, and such a value goes by its weight's rounding alone
        if (fabsf(acc[b][r]) < INFINITY) acc[b][r] += more[r];
      }
    }
    if (any && m == -INFINITY) m = -FLT_MAX;
    wait_loads();
    __syncthreads();  // the tiles are done with
    float *sums = reinterpret_cast<float *>(&tile[0][0][0][0]);  // [kWaves][kRows][kD]
    if (quad == 0) {
      s_m[wave][col] = m;
      s_l[wave][col] = l;
    }
    if (col < kRows) {
#pragma unroll
      for (int b = 0; b < kBlocks; ++b)
        *reinterpret_cast<f32x4 *>(sums + (wave * kRows + col) * kD + b * 16 + quad * 4) = acc[b];
    }
    __syncthreads();
    constexpr int kMost = kWaves * 64 / kRows;
    constexpr int kLanes = kMost < kD / 4 ? kMost : kD / 4;  // threads of a row
    const int r = threadIdx.x / kLanes, c0 = threadIdx.x % kLanes;
    const int mine = rt * 16 + r;
    if (r < kRows && mine < P.group && q_row >= 0) {
      float top = -INFINITY;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) top = fmaxf(top, s_m[w][r]);
      float f[kWaves], sum = 0.0f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        f[w] = s_m[w][r] == top ? 1.0f : __builtin_amdgcn_exp2f(s_m[w][r] - top);
        sum += f[w] * s_l[w][r];
      }
      const int ohead = kvh * P.group + mine;
      const int64_t flat = int64_t(id + seq) * P.n_heads + ohead;
      E *o = static_cast<E *>(P.out) + q_row * P.out_stride + ohead * P.out_head;
#pragma unroll
      for (int b = 0; b < kD / 4 / kLanes; ++b) {
        const int c = (b * kLanes + c0) * 4;
        if (c >= P.d) continue;
        f32x4 v = {};
#pragma unroll
        for (int w = 0; w < kWaves; ++w)
          v += f[w] * *reinterpret_cast<const f32x4 *>(sums + (w * kRows + r) * kD + c);
        if (whole) {
#pragma unroll
          for (int q = 0; q < 4; ++q) v[q] = weighted(v[q], top, sum);
          *reinterpret_cast<V4 *>(o + c) = __builtin_convertvector(v, V4);
        } else {
          *reinterpret_cast<f32x4 *>(P.part + flat * P.d + c) = v;
        }
      }
      if (!whole && c0 == 0) {
        P.part_ml[flat * 2] = top;
        P.part_ml[flat * 2 + 1] = sum;
      }
    }
    if (!again) return;
    at_tile += tiles;
    ++seq;
    __syncthreads();  // the sums are read
  }
}

// Joins the parts of a query head: a workgroup each, 32 lanes a part with 4 values each. Up to 64
// parts have all their loads under way at once; of more, the weights are found first (1 sequence of
// 100,003 keys, 4 heads over one, 391 parts: 28 -> 22 us in all).
constexpr int kPlaces = 512;  // ranges at most
constexpr int kJoinThreads = 256;

template <int kType>
__global__ __launch_bounds__(kJoinThreads, 4) void join_kernel(const AttendParams P) {
  typedef typename Num<kType>::E E;
  typedef typename Num<kType>::V4 V4;
  constexpr int kAtOnce = kJoinThreads / 32, kWaves = kJoinThreads / 64;
  __shared__ f32x4 s_sum[kAtOnce][32];
  __shared__ float s_w[kPlaces];
  __shared__ float s_top[kWaves], s_total[kWaves];
  const int tid = threadIdx.x, lane = tid & 63, group = tid >> 5, c = (tid & 31) * 4;
  const int id = workgroup(), head = id % P.n_heads, seq = id / P.n_heads;
  if (seq >= P.n_seqs) return;
  const Cut cut = find_cut(P, -1, seq);
  const Query query = query_of(P, seq);
  const int tiles = tiles_of(span_of(P, query.keys));
  const int first = cut.at / cut.length, n = (cut.at + tiles - 1) / cut.length - first + 1;
  if (tiles == 0 || n <= 1) return;  // in one range: the result is there
  const int64_t flat = int64_t(first + seq) * P.n_heads + head;
  const float *part = P.part + flat * P.d + c, *ml = P.part_ml + flat * 2;
  const int64_t step = int64_t(P.n_heads) * P.d, step_ml = int64_t(P.n_heads) * 2;
  float top = -INFINITY, total = 0.0f;
  f32x4 sum = {};
  if (n <= 64) {  // lane k of every wave has part k's maximum and sum
    float m = -INFINITY, l = 0.0f;
    if (lane < n) {
      m = ml[lane * step_ml];
      l = ml[lane * step_ml + 1];
    }
    f32x4 v[64 / kAtOnce];
#pragma unroll
    for (int u = 0; u < 64 / kAtOnce; ++u) {
      const int k = u * kAtOnce + group;
      v[u] = f32x4{};
      if (k < n && c < P.d) v[u] = *reinterpret_cast<const f32x4 *>(part + k * step);
    }
    top = wave_max(m);
    const float f = m == top ? 1.0f : __builtin_amdgcn_exp2f(m - top);
    total = wave_sum(f * l);
    if (tid < 64) s_w[lane] = f;
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 64 / kAtOnce; ++u) {
      const int k = u * kAtOnce + group;
      if (k < n) sum += s_w[k] * v[u];
    }
  } else {
    constexpr int kEach = kPlaces / kJoinThreads;
    float m[kEach], l[kEach];
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
      const int k = u * kJoinThreads + tid;
      m[u] = -INFINITY;
      l[u] = 0.0f;
      if (k < n) {
        m[u] = ml[k * step_ml];
        l[u] = ml[k * step_ml + 1];
      }
      top = fmaxf(top, m[u]);
    }
    top = wave_max(top);
    if (lane == 0) s_top[tid >> 6] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, s_top[w]);
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
      const float f = m[u] == top ? 1.0f : __builtin_amdgcn_exp2f(m[u] - top);
      s_w[u * kJoinThreads + tid] = f;
      total += f * l[u];
    }
    total = wave_sum(total);
    if (lane == 0) s_total[tid >> 6] = total;
    __syncthreads();
    total = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) total += s_total[w];
    if (c < P.d) {
#pragma unroll 8
      for (int k = group; k < n; k += kAtOnce)
        sum += s_w[k] * *reinterpret_cast<const f32x4 *>(part + k * step);
    }
  }
  s_sum[group][tid & 31] = sum;
  __syncthreads();
  if (group == 0 && c < P.d) {
#pragma unroll
    for (int g = 1; g < kAtOnce; ++g) sum += s_sum[g][tid];
#pragma unroll
    for (int q = 0; q < 4; ++q) sum[q] = weighted(sum[q], top, total);
    E *o = static_cast<E *>(P.out) + query.row * P.out_stride + head * P.out_head;
    *reinterpret_cast<V4 *>(o + c) = __builtin_convertvector(sum, V4);
  }
}

// ------------------------------------------------------------------------------- the host

// How a call is done: by a workgroup a sequence and key head, of `waves` waves, or with all keys
// cut into ranges for one workgroup a place (512: two a CU with heads of 128), which a second
// launch joins.
struct Form {
  int waves, width, least;
};

constexpr int kCutWaves = 2, kNear = 32;

int64_t each_of(int n_heads, int n_kv_heads) {  // workgroups of a sequence
  return int64_t(n_kv_heads) * ((n_heads / n_kv_heads + 15) / 16);
}

// Whether a sequence's keys are left to one workgroup: where there are few, since the join costs a
// launch, and up to more of them the more workgroups the sequences alone make; beyond, a long one
// among short ones would keep all waiting. us by a workgroup of 8 waves (4) and cut, with weights in
// one part (the second adds up to 5 % to either):
//       1 sequence,    900 keys, 16 heads of 128 over 4: 12.3, 12.0;   2,048: 16, 12
//       4 sequences, 1,200, 16 heads of 128 over 4:      13.9, 12.3;   2,048: 19, 16
//       8 sequences, 1,600, 16 heads of 128 over 4:      17.0, 17.3;   2,048: 20, 18
//      14 sequences, 2,048, 16 heads of 128 over 4:      20.3, 20.8;   2,560: 23, 21
//      30 sequences, 2,048, 16 heads of 128 over 4:      22.2, 25.3;   3,500: 49, 37
//       1 sequence,  1,600, 16 heads of 64 over 4:        9.8, 10.7;   2,048: 11.4, 10.7
//       4 sequences, 2,560, 16 heads of 64 over 4:       13.9, 14.1;   3,500: 19, 14
//       8 sequences, 2,560, 16 heads of 64 over 4:       14.9, 15.6;   3,500: 19, 16
//      20 sequences, 1,600, 16 heads of 64 over 4:         13 (19), 18
//      30 sequences, 3,500, 16 heads of 64 over 4:       19.9, 23.1
//      64 sequences, 2,200, 16 heads of 128 over 4:        41 (40), 46
//     256 sequences, 4,096, 32 heads of 128 over 8:       439 (442), 439
//     256 sequences,   500, 16 heads of 64 over 2:         12 (11), 35
//   1,000 sequences,   900, 8 heads of 128 over 1:         64 (58), 106
//       8 sequences, 100,003, 16 heads of 128 over 2:     937 (1,107), 111
// 16 waves, of heads of 64: 13.3 for 13.1 where 20 have 1,600 keys, 73.8 for 65.8 where 256 have
// 2,000.
struct Whole {
  int alone;         // from so many workgroups on
  int narrow, wide;  // keys of heads up to 64, and of wider ones
};
constexpr int kWholeLeast = 768;
constexpr Whole kWhole[] = {{256, 4096, 4096}, {64, 3584, 2048}, {32, 2816, 1664},
                            {16, 2560, 1408},  {8, 2048, 1024},  {0, 1792, kWholeLeast}};

Form form_of(int n_seqs, int max_kv, int64_t each, int d) {
  const int64_t alone = n_seqs * each;
  const Whole *limit = kWhole;
  while (alone < limit->alone) ++limit;
  const int whole = d <= 64 ? limit->narrow : limit->wide;
  const int waves = max_kv <= (alone > 256 ? 1024 : 512) ? 4 : 8;
  // tiles are counted in 30 bits
  if (n_seqs > kMaxCut || max_kv <= whole || n_seqs * (int64_t(max_kv) / kKeys + 2) > 1 << 30)
    return {waves, 0, 0};
  return {kCutWaves, static_cast<int>(std::max<int64_t>(kPlaces / each, 1)), kCutWaves};
}

template <int kType, int kD, int kWaves, int kBufs, bool kPair>
int launch_waves(const AttendParams &P, hipStream_t s) {
  int64_t blocks = P.width ? P.width : P.n_seqs;
  if (P.near) blocks = (blocks + kXcds - 1) / kXcds * kXcds;
  blocks *= int64_t(P.n_kv_heads) * P.row_tiles;
  const int64_t joined = P.width > 0 ? int64_t(P.n_seqs) * P.n_heads : 0;
  if (blocks > kMaxWorkgroups || joined > kMaxWorkgroups) return TG_E_INVAL;
  hipLaunchKernelGGL((attend_pages_kernel<kType, kD, kWaves, kBufs, kPair>),
                     grid_of(blocks, kWaves * 64), dim3(kWaves * 64), 0, s, P);
  if (joined > 0)
    hipLaunchKernelGGL(join_kernel<kType>, grid_of(joined, kJoinThreads), dim3(kJoinThreads), 0, s,
                       P);
  return hipGetLastError() == hipSuccess ? TG_OK : TG_E_HIP;
}

template <int kType, int kD, bool kPair>
int launch_form(const AttendParams &P, hipStream_t s) {
  if (P.width > 0) return launch_waves<kType, kD, kCutWaves, 2, kPair>(P, s);
  return P.unit == 4 ? launch_waves<kType, kD, 4, 1, kPair>(P, s)
                     : launch_waves<kType, kD, 8, 1, kPair>(P, s);
}

template <int kType, int kD>
int launch(const AttendParams &P, hipStream_t s) {
  return P.group <= 8 ? launch_form<kType, kD, true>(P, s) : launch_form<kType, kD, false>(P, s);
}

bool layout_ok(const void *p, int64_t stride, int64_t head) {
  return p && aligned16(p) && stride >= 0 && stride <= kMaxStride && stride % 8 == 0 &&
         head >= 0 && head % 8 == 0;
}

bool sizes_ok(int n_seqs, int max_kv, int n_heads, int n_kv_heads, int d) {
  return n_seqs >= 0 && n_seqs <= TG_PAGES_MAX_SEQS && max_kv >= 0 &&
         max_kv <= kMaxKeys && n_heads >= 1 &&
         n_kv_heads >= 1 && n_heads % n_kv_heads == 0 && d >= 8 && d <= TG_ATTEND_MAX_D &&
         d % 8 == 0;
}

}  // namespace

// Parts of a call, and of every call of fewer sequences or shorter ones with it: those may have
// more parts than this one, which may have none.
extern "C" size_t tg_attend_pages_workspace_bytes(int32_t n_seqs, int32_t max_kv_len,
                                                  int32_t n_heads, int32_t n_kv_heads,
                                                  int32_t d) {
  if (!sizes_ok(n_seqs, max_kv_len, n_heads, n_kv_heads, d) || n_seqs == 0) return 0;
  const int64_t each = each_of(n_heads, n_kv_heads);
  if (max_kv_len <= kWholeLeast) return 0;
  const int64_t cut = std::min<int64_t>(n_seqs, kMaxCut);
  const int64_t parts = std::max<int64_t>(kPlaces / each, 1) + cut;
  return static_cast<size_t>(parts) * n_heads * (d + 2) * sizeof(float);
}

extern "C" int tg_attend_pages(const tg_attend_pages_args *a, void *stream) {
  if (!a || !type_ok(a->type) ||
      !sizes_ok(a->n_seqs, a->max_kv_len, a->n_heads, a->n_kv_heads, a->d) || a->n_pages < 0 ||
      (a->q_begin && a->n_q_rows < 0) || a->page_size < 1 || a->max_pages < 1 || a->window < 0 ||
      int64_t(a->n_pages) * a->page_size > INT32_MAX || a->table_stride < a->max_pages ||
      !std::isfinite(a->scale) || !std::isfinite(a->cap) || a->cap < 0.0f)
    return TG_E_INVAL;
  if (a->n_seqs == 0 || (a->q_begin && a->n_q_rows == 0)) return TG_OK;
  if (!a->table || !a->kv_len || !layout_ok(a->q, a->q_stride, a->q_head_stride) ||
      !layout_ok(a->out, a->out_stride, a->out_head_stride))
    return TG_E_INVAL;
  if (a->n_pages > 0 && (!layout_ok(a->k, a->k_stride, a->k_head_stride) ||
                         !layout_ok(a->v, a->v_stride, a->v_head_stride)))
    return TG_E_INVAL;
  const size_t need = tg_attend_pages_workspace_bytes(a->n_seqs, a->max_kv_len, a->n_heads,
                                                      a->n_kv_heads, a->d);
  if (need > 0 && (!a->workspace || a->workspace_bytes < need || !aligned16(a->workspace)))
    return TG_E_WORKSPACE;
  AttendParams P = {};
  P.q = a->q;
  P.k = a->k;
  P.v = a->v;
  P.out = a->out;
  P.q_stride = a->q_stride;
  P.q_head = a->q_head_stride;
  P.k_stride = a->k_stride;
  P.k_head = a->k_head_stride;
  P.v_stride = a->v_stride;
  P.v_head = a->v_head_stride;
  P.out_stride = a->out_stride;
  P.out_head = a->out_head_stride;
  P.table = a->table;
  P.table_stride = a->table_stride;
  P.kv_len = a->kv_len;
  P.q_begin = a->q_begin;
  P.n_q_rows = a->n_q_rows;
  P.slope = a->slope;
  // factors at the ends of binary32 are its largest numbers
  const auto factor = [](double v) {
    return static_cast<float>(std::min(std::max(v, -double(FLT_MAX)), double(FLT_MAX)));
  };
  P.to_log2 = factor(double(a->scale) * kLog2e);
  if (a->cap > 0.0f) {
    // of a cap so large that no score reaches tanh's bend, any other such will do
    const double cap = std::min<double>(
        a->cap, 0x1p100 * std::min(std::max(std::fabs(double(a->scale)), 1.0), 0x1p26));
    P.cap_arg = factor(a->scale / cap);
    P.cap_out = static_cast<float>(cap * kLog2e);
  }
  P.window = a->window;
  P.n_seqs = a->n_seqs;
  P.n_pages = a->n_pages;
  P.page_size = a->page_size;
  P.page_log2 = -1;
  if ((a->page_size & (a->page_size - 1)) == 0) P.page_log2 = __builtin_ctz(a->page_size);
  P.most = static_cast<int32_t>(
      std::min<int64_t>(int64_t(a->max_pages) * a->page_size, a->max_kv_len));
  P.n_heads = a->n_heads;
  P.n_kv_heads = a->n_kv_heads;
  P.group = a->n_heads / a->n_kv_heads;
  P.d = a->d;
  const int64_t each = each_of(a->n_heads, a->n_kv_heads);
  P.row_tiles = static_cast<int32_t>(each / a->n_kv_heads);
  const int seen = a->window > 0 ? std::min(P.most, a->window) : P.most;
  const Form form = form_of(a->n_seqs, seen, each, a->d);
  P.unit = form.waves;
  P.width = form.width;
  P.least = form.least;
  // Heads that share lines of 128 bytes, or more than 16 query heads that share a key head, would
  // have them read once for each XCD; with few sequences all XCDs are wanted. us without and with:
  // 8 sequences of 100,003 keys, 16 heads of 96 over 2: 95, 86; 8 of 60,000, 32 heads of 128 over
  // 1: 68, 51; 64 of 900, 16 heads of 80 over 4: 17.2, 14.8.
  const bool share = P.row_tiles > 1 ||
                     (a->n_kv_heads > 1 && (a->k_head_stride % 64 || a->v_head_stride % 64));
  P.near = share && (P.width > 0 ? P.width : P.n_seqs) >= kNear;
  P.part = static_cast<float *>(a->workspace);
  P.part_ml = P.part + (static_cast<size_t>(P.width) + a->n_seqs) * a->n_heads * a->d;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (a->d <= 64) return a->type == TG_F16 ? launch<TG_F16, 64>(P, s) : launch<TG_BF16, 64>(P, s);
  return a->type == TG_F16 ? launch<TG_F16, 128>(P, s) : launch<TG_BF16, 128>(P, s);
}
