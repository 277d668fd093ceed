// tg_attend: attention over a ragged batch, with capped scores, a bias by distance, a document
// mask and a prefix mask.
//
// Softmax in one pass over the keys (Milakov and Gimelshein 2018; tiled as by Dao et al. 2022):
// a running maximum m, the sum l of 2^(z - m) and the weighted sum of values, the latter two
// multiplied by 2^(m_old - m_new) when m grows. Scores are kept in units of log2, so that a
// weight is one exponential. m is only moved when a score passes it by more than kSlack: weights
// then reach 2^kSlack times what they would, which neither binary16 nor the sums mind, and the
// accumulators are seldom touched.
//
// Scores are computed transposed, S^T = K Q^T: a lane holds scores of ONE query, so that m, l
// and the correction are plain registers, and the weights come out where the second product,
// O^T = V^T P^T, takes them as an operand. That operand's key slots are then not in key order
// (a lane has the keys 4 h + 0..3 of every 8, h its half of the wave); the sum over keys does
// not care, as long as V is taken in the same order, which the transposing LDS reads do.
//
// attend_tile_kernel takes 128 queries of a head at a time, attend_few_kernel the few queries of
// all heads that share keys. Both cut long key ranges over workgroups where there are few, joined
// by join_tile_kernel and join_kernel.
//
// A key that a query does not see has weight 0, and 0 times infinity or NaN would still reach
// the query's sum. Such sums stay NaN, so each result is looked at once, at the end; a row that
// is not finite is computed again by strict_row, which leaves unseen keys out one by one. So is a
// row that has no maximum though it sees keys, and one whose scores are so large (2^24 and more)
// that the maximum, which is rounded, lies so far from the score that it comes from that the
// largest weight is lost (full_sum).
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

constexpr int kMaxStride = 1 << 22;
constexpr float kSlack = 8.0f;
// Weights are kept times 2^kLift: binary16's smallest number is 2^-24, and without it what lies
// below 2^-25 of the largest weight would be lost, however many such keys there are. With kSlack
// they reach 2^15, which binary16 holds.
template <int kType>
constexpr float kLift = kType == TG_F16 ? 7.0f : 0.0f;
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
// Caps up to here use 1 - 2 / (1 + 2^x) for tanh, whose error of a few 2^-24 times the cap stays
// below 1e-4 in the exponent; with larger ones small arguments, where 1 and the quotient cancel,
// take the series.
constexpr float kFastCap = 256.0f;

struct AttendParams {
  const void *q, *k, *v;
  void *out;
  int64_t q_stride, q_head, k_stride, k_head, v_stride, v_head, out_stride, out_head;
  const int32_t *q_begin, *kv_len, *prefix, *q_doc, *k_doc, *q_pos, *k_pos;
  const int64_t *kv_begin;
  const float *slope;
  float to_log2;    // scale * log2(e): a raw score's factor
  float cap_in;     // raw score -> exponent of 2 inside tanh: 2 log2(e) scale / cap
  float cap_out;    // cap * log2(e)
  float cap_arg;    // scale / cap
  int32_t capped;   // 0 none, 1 up to kFastCap, 2 above
  int32_t shaped;   // scores are brought to log2 units before the softmax (cap, bias, scale <= 0)
  int32_t causal, n_seqs, n_q_rows;
  int64_t n_k_rows;
  int32_t max_q, max_kv, n_heads, n_kv_heads, group, d;
  // attend_tile_kernel
  int32_t turns;    // workgroups of a head
  int32_t splits;   // workgroups that share a tile's keys; with more than one, parts are laid out
                    // as [splits][n_q_rows][n_heads][d], and [..][..][..][2]
  // attend_few_kernel
  int32_t row_tiles;
  int32_t width;    // parts that all keys are cut into, 0: no sequence is cut
  float *part;      // [width + n_seqs][n_kv_heads][16 row_tiles][d] weighted sums, and
  float *part_ml;   // [..][..][..][2] maximum (log2 units) and sum of weights
};

struct Seq {
  int q0, nq;       // first query row, queries
  int64_t k0;       // first key row
  int nk, place0;   // keys, place of the first query
  int prefix;
};

// A sequence, clamped to the tensors and to the caller's bounds.
__device__ __forceinline__ Seq sequence(const AttendParams &P, int s) {
  Seq r;
  const int a = min(max(P.q_begin[s], 0), P.n_q_rows);
  const int b = min(max(P.q_begin[s + 1], a), P.n_q_rows);
  r.q0 = a;
  r.k0 = P.kv_begin[s];
  int64_t nk = P.kv_len[s];
  if (r.k0 < 0 || r.k0 >= P.n_k_rows) {
    r.k0 = 0;
    nk = 0;
  }
  nk = min(max(nk, int64_t(0)), P.n_k_rows - r.k0);
  r.place0 = static_cast<int>(nk) - (b - a);
  r.nk = min(static_cast<int>(nk), P.max_kv);
  r.nq = min(b - a, P.max_q);
  r.prefix = P.prefix ? P.prefix[s] : 0;
  return r;
}

// v < 0, looked at here and not where v was loaded: the compiler would wait for the load before
// it issues those that follow (single tokens of 250 keys 9.1 us for 8.7).
__device__ __forceinline__ bool below_zero(int v) {
  asm volatile("" : "+v"(v));
  return v < 0;
}

// Lane `l`'s sequence, for every lane.
__device__ __forceinline__ Seq broadcast(const Seq &s, int l) {
  const auto take = [&](int v) { return __builtin_amdgcn_readlane(v, l); };
  Seq r;
  r.q0 = take(s.q0);
  r.nq = take(s.nq);
  const uint32_t hi = static_cast<uint32_t>(take(static_cast<int>(s.k0 >> 32)));
  const uint32_t lo = static_cast<uint32_t>(take(static_cast<int>(s.k0)));
  r.k0 = static_cast<int64_t>(static_cast<uint64_t>(hi) << 32 | lo);
  r.nk = take(s.nk);
  r.place0 = take(s.place0);
  r.prefix = take(s.prefix);
  return r;
}

// The sequence that has a tile of `rows` queries, and the tile's first query in it (none of its
// own where that is outside). Sequence b owns the tiles from q_begin[b] / rows + b on, room for
// all of its queries. Up to 64 sequences are looked at at once, one a lane.
__device__ __forceinline__ Seq sequence_of(const AttendParams &P, int tile, int rows, int &first) {
  if (P.n_seqs <= 64) {
    const int lane = threadIdx.x & 63;
    const Seq mine = sequence(P, min(lane, P.n_seqs - 1));
    const uint64_t before = __ballot(lane < P.n_seqs && mine.q0 / rows + lane <= tile);
    const int at = before ? 63 - __builtin_clzll(before) : 0;
    const Seq s = broadcast(mine, __builtin_amdgcn_readfirstlane(at));
    first = (tile - (s.q0 / rows + at)) * rows;
    return s;
  }
  int lo = 0, hi = P.n_seqs - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (min(max(P.q_begin[mid], 0), P.n_q_rows) / rows + mid <= tile) lo = mid; else hi = mid - 1;
  }
  const Seq s = sequence(P, lo);
  first = (tile - (s.q0 / rows + lo)) * rows;
  return s;
}

// Keys before this one are the ones that query i may see, documents aside.
__device__ __forceinline__ int key_limit(const AttendParams &P, const Seq &s, int i) {
  if (!P.causal) return s.nk;
  return min(s.nk, max(s.place0 + i + 1, s.prefix));
}

// 1 / (1 + 2^x), which is (1 - tanh) / 2 of the argument that x stands for.
__device__ __forceinline__ float fall(float x) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x));
}

// a - b of any two, rounded once: by halves, as the difference can pass 32 bits.
__device__ __forceinline__ float apart(int a, int b) {
  return __builtin_fmaf(static_cast<float>((a >> 16) - (b >> 16)), 65536.0f,
                        static_cast<float>((a & 0xFFFF) - (b & 0xFFFF)));
}

// A raw score capped, in log2 units.
__device__ __forceinline__ float cap_score(const AttendParams &P, float s) {
  const float z = __builtin_fmaf(-2.0f * P.cap_out, fall(s * P.cap_in), P.cap_out);
  if (P.capped == 1) return z;
  // x - x^3 / 3 + 2 x^5 / 15 - 17 x^7 / 315: to 2e-9 below 1 / 8
  const float x = s * P.cap_arg, x2 = x * x;
  const float p = __builtin_fmaf(
      x2, __builtin_fmaf(x2, __builtin_fmaf(x2, -17.0f / 315, 2.0f / 15), -1.0f / 3), 1.0f);
  return fabsf(x) < 0.125f ? P.cap_out * (x * p) : z;
}

// A raw score in log2 units; `far` is the distance. (The tile kernel does the same steps.)
__device__ __forceinline__ float shape(const AttendParams &P, float s, float slope2, float far) {
  const float z = P.capped ? cap_score(P, s) : s * P.to_log2;
  return z - slope2 * far;
}

// The largest, or smallest, of three in one instruction; NaN is left out where there is another.
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
__device__ __forceinline__ float min3(float a, float b, float c) {
  float r;
  asm("v_min3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
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

// The larger of a lane's value and that of its partner in the other half of the wave.
__device__ __forceinline__ float both_halves(float v) {
  const unsigned u = __builtin_bit_cast(unsigned, v);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__builtin_bit_cast(float, static_cast<unsigned>(r[0])),
               __builtin_bit_cast(float, static_cast<unsigned>(r[1])));
}

__device__ __forceinline__ float abs_diff(int a, int b) {  // of any two
  const uint32_t d = static_cast<uint32_t>(a) - static_cast<uint32_t>(b);
  return static_cast<float>(a > b ? d : 0u - d);
}

// Whether a row's sum holds its largest weight, which is 1 at least if it was not rounded away;
// without a maximum, whether it sees no key (`none`: it may see none).
__device__ __forceinline__ bool full_sum(float m, float l, bool none) {
  return l >= 0.5f || (m == -INFINITY && none);
}

// One query row of one head, by one wave, unseen keys left out one by one: a lane a key's score,
// then 8 or 16 lanes a key's values. A NaN that is seen in the query or a key is all of the result,
// so that the rest is not looked at. bfloat16, the 7 prompts of up to 2,077 with a cap below, all
// of whose rows come here: 17 ms for 0.15 with a NaN in every value, 1.3 in every query.
template <int kType>
__device__ __forceinline__ void strict_row(const AttendParams &P, const Seq &s, int i,
                                           int head) {
  typedef typename Num<kType>::E E;
  typedef typename Num<kType>::V8 V8;
  const int lane = threadIdx.x & 63;
  const int64_t row = int64_t(s.q0) + i;
  const E *q = static_cast<const E *>(P.q) + row * P.q_stride + head * P.q_head;
  const E *k = static_cast<const E *>(P.k) + (head / P.group) * P.k_head + s.k0 * P.k_stride;
  const int limit = key_limit(P, s, i), place = s.place0 + i;
  const int doc = P.q_doc ? P.q_doc[row] : 0;
  const float slope2 = P.slope ? P.slope[head] * kLog2e : 0.0f;
  const int wide = P.d <= 64 ? 8 : 16, c = lane % wide * 8, own = lane / wide;
  const E *v = static_cast<const E *>(P.v) + (head / P.group) * P.v_head + s.k0 * P.v_stride + c;
  float m = -INFINITY, l = 0.0f, sum[8] = {};
  bool lost = false, any = false;
  for (int j0 = 0; j0 < limit && !lost; j0 += 64) {
    const int j = j0 + lane;
    const bool seen = j < limit && doc >= 0 && (!P.k_doc || P.k_doc[s.k0 + j] == doc);
    const uint64_t all = __ballot(seen);
    if (!all) continue;
    any = true;
    float z = -INFINITY;
    if (seen) {
      const E *kr = k + j * P.k_stride;
      float dot = 0.0f;
      for (int e0 = 0; e0 < P.d; e0 += 8) {
        const V8 a = *reinterpret_cast<const V8 *>(q + e0);
        const V8 b = *reinterpret_cast<const V8 *>(kr + e0);
#pragma unroll
        for (int e = 0; e < 8; ++e) dot += static_cast<float>(a[e]) * static_cast<float>(b[e]);
      }
      float far = abs_diff(place, j);
      if (P.k_pos)
        far = abs_diff(P.q_pos[2 * row], P.k_pos[2 * (s.k0 + j)]) +
              abs_diff(P.q_pos[2 * row + 1], P.k_pos[2 * (s.k0 + j) + 1]);
      z = shape(P, dot, slope2, P.slope ? far : 0.0f);
    }
    lost = __ballot(z != z) != 0;
    const float to = fmaxf(m, wave_max(z));
    const float fix = to == m ? 1.0f : __builtin_amdgcn_exp2f(m - to);
    m = to;
    const float p = seen ? __builtin_amdgcn_exp2f(z - (m == -INFINITY ? 0.0f : m)) : 0.0f;
    l = l * fix + p;
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] *= fix;
    for (int u = own; u < 64; u += 64 / wide) {
      const float w = __shfl(p, u);
      if (!(all >> u & 1) || c >= P.d) continue;
      const V8 x = *reinterpret_cast<const V8 *>(v + int64_t(j0 + u) * P.v_stride);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[e] += w * static_cast<float>(x[e]);
    }
  }
  lost = lost || (any && m == -INFINITY);  // all scores minus infinity: no weights
  l = wave_sum(l);
  V8 out;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    for (int o = wide; o < 64; o <<= 1) sum[e] += __shfl_xor(sum[e], o);
    out[e] = static_cast<E>(lost ? NAN : l == 0.0f ? 0.0f : sum[e] / l);
  }
  E *o = static_cast<E *>(P.out) + row * P.out_stride + head * P.out_head;
  if (own == 0 && c < P.d) *reinterpret_cast<V8 *>(o + c) = out;
}

// Place of 16-byte chunk c of row r in a tile of rows of kChunks chunks (8 or 16). Matrix
// operands take one chunk of 16 rows at once, transposing reads 4 chunks of 4 rows (the tile
// kernel) or 2 chunks of 8 rows (kPairs, the kernel for few rows): all fall on 16 different
// places of the 256 bytes that LDS serves at once.
template <int kChunks, bool kPairs>
__device__ __forceinline__ int place_of(int r, int c) {
  if (kChunks == 16) {
    const int g = kPairs ? ((r & 7) << 1) | ((r >> 3) & 1) : ((r & 3) << 2) | ((r >> 2) & 3);
    return c ^ g;
  }
  const int g = kPairs ? (((r >> 1) & 3) << 1) | ((r >> 3) & 1)
                       : (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
  return c ^ g;
}

// Loads kRows rows of a head's keys or values, from `row` on, into an LDS tile, shared by kShare
// waves; rows from `rows` on and values past d are 0. `offset` is that of the wave's first load,
// which row_offset gives: rows of later loads lie kShare * 64 / kChunks further, and take their
// chunks from the same places where that is a multiple of 16.
template <int kChunks, bool kPairs>
__device__ __forceinline__ uint32_t row_offset(int64_t stride, int d, int r) {
  const int c = place_of<kChunks, kPairs>(r, (threadIdx.x & 63) & (kChunks - 1));
  return c * 8 < d ? static_cast<uint32_t>((r * stride + c * 8) * 2) : kNowhere;
}

template <int kRows, int kChunks, bool kPairs, int kShare>
__device__ __forceinline__ void load_rows(const void *base, int64_t stride, int64_t row, int rows,
                                          int d, void *tile, int wave, uint32_t offset) {
  constexpr int kPer = 64 / kChunks, kStep = kPer * kShare;  // rows of one load, of one turn
  const auto b = buffer(static_cast<const char *>(base) + row * stride * 2,
                        static_cast<uint32_t>(((min(rows, kRows) - 1) * stride + d) * 2));
#pragma unroll
  for (int i = 0; i < kRows / kStep; ++i) {
    uint32_t off = offset + static_cast<uint32_t>(i * kStep * stride * 2);
    if (kStep % 16)
      off = row_offset<kChunks, kPairs>(stride, d, i * kStep + (threadIdx.x & 63) / kChunks);
    load_lds(b, static_cast<char *>(tile) + (i * kShare + wave) * 1024, off, 0);
  }
}

// A key's document, or a coordinate (`part`) of its position, of up to kRows keys from `row` on:
// one lane a key.
template <int kRows>
__device__ __forceinline__ void load_marks(const int32_t *base, int64_t row, int rows, int width,
                                           int part, int *to) {
  const int lane = threadIdx.x & 63;
  const auto b = buffer(base + row * width, static_cast<uint32_t>(min(rows, kRows) * width * 4));
  load_lds4(b, to, lane < kRows ? static_cast<uint32_t>((lane * width + part) * 4) : kNowhere);
}

template <int kType>
__device__ __forceinline__ typename Num<kType>::V4 read_transposed(const void *p) {
  typedef __attribute__((address_space(3))) s16x4 *P3;
  return __builtin_bit_cast(
      typename Num<kType>::V4,
      __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<P3>(
          reinterpret_cast<uintptr_t>(p))));
}

// ------------------------------------------------------------------- 128 queries of a head

constexpr int kBM = 128, kBN = 64;
constexpr int kCus = 256;
constexpr int kMaskTiles = 4096;  // key tiles whose documents are looked through at once

// What is done to a score between the products, decided when compiled where it is common.
enum Mode {
  kPlain = 0,  // the factor only
  kCapped = 1, // a cap up to kFastCap
  kSloped = 2, // a bias by the distance of indexes
  kAny = 3     // any of the above at once, positions, documents, a factor <= 0
};

// A wave takes 32 queries and a workgroup's 4 waves share tiles of 64 keys and values, two of them
// in LDS by turns, so that a tile's loads run while the one before it is worked on: 69 KB with
// heads of 128 and 2 workgroups a CU, 3 with heads of 64. The weights never leave the registers.
// A tile has about as many cycles of matrix as of vector instructions, and they hardly overlap:
// that, and not memory, bounds it, so the vector work a score costs is what the modes are for.
// bfloat16, one sequence of 16,384 tokens, 16 heads of 128 over 4, causal, a bias: 1.12 to 1.22 ms
// by card, 900 to 980 TFLOP/s of the products that are seen, matrix units 48 % of the time at
// work, vector units 57 %; 7 of up to 2,077 with a cap and prefixes 0.15 ms, 620 (33 %, 58 %).
// binary16, 4 canvases of up to 6,400 tokens, 16 heads of 64, 32 documents each and a bias by
// position: 0.11 ms (12 %, 59 %, and waves that wait 47 % of their time, as a workgroup has about 7
// tiles and looks through all documents first; 0.26 with the tokens in raster order, where few
// keys of a tile are of a query's document).
// 64 queries a wave (half the LDS reads) spilled registers and took three times as long; one
// tile's products between the other's exponentials, by half tiles, 1.30 ms for 1.20.
template <int kType, int kD, int kMode>
__global__ __launch_bounds__(kThreads, kD == 64 ? 3 : 2) void attend_tile_kernel(const AttendParams P) {
  typedef Num<kType> N;
  typedef typename N::E E;
  typedef typename N::V4 V4;
  typedef typename N::V8 V8;
  constexpr int kChunks = kD / 8, kSteps = kD / 16, kBlocks = kD / 32;
  __shared__ __attribute__((aligned(16))) E tk[2][kBN * kD];
  __shared__ __attribute__((aligned(16))) E tv[2][kBN * kD];
  constexpr bool kAnyMode = kMode == kAny;
  __shared__ int s_doc[2][kAnyMode ? kBN : 1];
  __shared__ int s_pos[2][2][kAnyMode ? kBN : 1];
  __shared__ float s_far[kWaves][2][kAnyMode ? kBN : 1];  // the keys' places from the wave's first
  __shared__ uint64_t s_use[kAnyMode ? kMaskTiles / 64 : 1];
  __shared__ int s_range[kWaves][2];
  const bool with_docs = kAnyMode && P.k_doc, with_pos = kAnyMode && P.k_pos;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int id = workgroup(), head = id % P.n_heads;
  // Long rows first; workgroups 256 to 511 the other way round, as they share a CU with those 256
  // before them (4 causal prompts of 2,048, 8 heads of 128: 57 us for 63; 1 of 4,096, 16 heads:
  // 101 for 104)
  const int turns = P.turns, round = kCus / P.n_heads;
  int turn = id / P.n_heads;
  if (turn >= turns) return;
  if (turn >= round && turn < 2 * round) turn = round + min(2 * round, turns) - 1 - turn;
  const int split = turn % P.splits, tile = (turns - 1 - turn) / P.splits;
  int first;
  const Seq s = sequence_of(P, tile, kBM, first);
  if (first < 0 || first >= s.nq) return;
  const int i = first + wave * 32 + col;       // this lane's query
  const bool live = i < s.nq;
  const int64_t row = int64_t(s.q0) + min(i, s.nq - 1);
  const E *qr = static_cast<const E *>(P.q) + row * P.q_stride + head * P.q_head;
  V8 qf[kSteps];
#pragma unroll
  for (int k = 0; k < kSteps; ++k) {
    qf[k] = V8{};
    if (k * 16 + half * 8 < P.d) qf[k] = *reinterpret_cast<const V8 *>(qr + k * 16 + half * 8);
  }
  const void *kb = static_cast<const E *>(P.k) + (head / P.group) * P.k_head;
  const void *vb = static_cast<const E *>(P.v) + (head / P.group) * P.v_head;
  const int limit = live ? key_limit(P, s, i) : 0;
  const int wave_first = first + wave * 32;
  // every key before `all` is seen by all of the wave's queries, none from `end` on by any of
  // the workgroup's (limits do not fall with i)
  const int all = key_limit(P, s, min(wave_first, s.nq - 1));
  const int end = key_limit(P, s, min(first + kBM, s.nq) - 1);
  const int wave_end = wave_first < s.nq ? key_limit(P, s, min(wave_first + 32, s.nq) - 1) : 0;
  int doc = with_docs && live ? P.q_doc[row] : -1;
  const float slope2 = kMode >= kSloped && P.slope ? P.slope[head] * kLog2e : 0.0f;
  const int place = s.place0 + i;
  int px = 0, py = 0;
  if (with_pos) {
    px = P.q_pos[2 * row];
    py = P.q_pos[2 * row + 1];
  }
  const int x0 = __builtin_amdgcn_readfirstlane(px), y0 = __builtin_amdgcn_readfirstlane(py);
  const float fx = apart(px, x0), fy = apart(py, y0);
  // queries so far apart that the wave's first is no origin for exact differences
  const bool scattered = with_pos && __ballot(fmaxf(fabsf(fx), fabsf(fy)) > 0x1p23f) != 0;
  const bool late = !P.capped && P.to_log2 >= 0x1p-20f;
  const float rate = late ? slope2 / P.to_log2 : slope2;
  int wave_lo = INT_MAX, wave_hi = -1;  // the documents of the wave's queries
  int block_lo = INT_MAX, block_hi = -1;
  if (with_docs) {
    int a = doc >= 0 ? doc : INT_MAX, b = doc;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      a = min(a, __shfl_xor(a, o));
      b = max(b, __shfl_xor(b, o));
    }
    wave_lo = a;
    wave_hi = b;
    if (lane == 0) {
      s_range[wave][0] = a;
      s_range[wave][1] = b;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      block_lo = min(block_lo, s_range[w][0]);
      block_hi = max(block_hi, s_range[w][1]);
    }
    if (doc < 0) doc = INT_MIN;  // hardly any key's
  }
  const int first_row = wave * (64 / kChunks) + lane / kChunks;
  const uint32_t k_off = row_offset<kChunks, false>(P.k_stride, P.d, first_row);
  const uint32_t v_off = row_offset<kChunks, false>(P.v_stride, P.d, first_row);
  f32x16 acc[kBlocks] = {};
  float m = -INFINITY, l = 0.0f;
  int tiles = (end + kBN - 1) / kBN, from = 0;
  if (P.splits > 1) {
    from = static_cast<int>(int64_t(tiles) * split / P.splits);
    tiles = static_cast<int>(int64_t(tiles) * (split + 1) / P.splits);
  }

  for (int seg = from; seg < tiles; seg += kMaskTiles) {
    const int seg_end = min(tiles, seg + kMaskTiles);
    if (with_docs) {  // which tiles hold a key whose document is in the queries' range
      __syncthreads();
      for (int t = threadIdx.x; t < kMaskTiles / 64; t += kThreads) s_use[t] = 0;
      __syncthreads();
      // 4 keys a lane and 4 tiles a load, 8 loads under way
      constexpr int kAhead = 8, kTurn = 4 * kAhead;
      for (int t0 = seg + wave * kTurn; t0 < seg_end; t0 += kWaves * kTurn) {
        i32x4 kd[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
          const int j = (t0 + 4 * u) * kBN + 4 * lane;
          kd[u] = i32x4{-1, -1, -1, -1};
          if (t0 + 4 * u < seg_end) {
            if (j + 3 < end) {
              __builtin_memcpy(&kd[u], P.k_doc + s.k0 + j, 16);
            } else {
#pragma unroll
              for (int e = 0; e < 3; ++e)
                if (j + e < end) kd[u][e] = P.k_doc[s.k0 + j + e];
            }
          }
        }
        uint32_t used = 0;
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
          bool in = false;
#pragma unroll
          for (int e = 0; e < 4; ++e) in = in || (kd[u][e] >= block_lo && kd[u][e] <= block_hi);
          const uint64_t lanes = __ballot(in);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            used |= ((lanes >> (16 * e)) & 0xFFFF ? 1u : 0u) << (4 * u + e);
        }
        if (used && lane == 0)  // 32 tiles from a multiple of 32 on: within one word
          atomicOr(reinterpret_cast<unsigned long long *>(&s_use[(t0 - seg) >> 6]),
                   static_cast<unsigned long long>(used) << ((t0 - seg) & 63));
      }
      __syncthreads();
    }
    auto next = [&](int t) {  // the first tile to visit from t on
      if (!with_docs) return t;
      while (t < seg_end) {
        const uint64_t w = s_use[(t - seg) >> 6] >> ((t - seg) & 63);
        if (w) {
          t += __builtin_ctzll(w);
          break;
        }
        t = seg + (((t - seg) >> 6) + 1) * 64;
      }
      return __builtin_amdgcn_readfirstlane(t);
    };
    auto fetch = [&](int t, int to) {
      const int j0 = t * kBN;
      load_rows<kBN, kChunks, false, kWaves>(kb, P.k_stride, s.k0 + j0, s.nk - j0, P.d, tk[to],
                                             wave, k_off);
      load_rows<kBN, kChunks, false, kWaves>(vb, P.v_stride, s.k0 + j0, s.nk - j0, P.d, tv[to],
                                             wave, v_off);
      if (with_docs && wave == 0)
        load_marks<kBN>(P.k_doc, s.k0 + j0, s.nk - j0, 1, 0, s_doc[to]);
      if (with_pos && (wave == 1 || wave == 2))
        load_marks<kBN>(P.k_pos, s.k0 + j0, s.nk - j0, 2, wave - 1, s_pos[to][wave - 1]);
    };
    int t = next(seg), buf = 0;
    if (t < seg_end) fetch(t, 0);
    while (t < seg_end) {
      const int j0 = t * kBN;
      const int after = next(t + 1);
      wait_loads();
      __syncthreads();
      if (after < seg_end) fetch(after, buf ^ 1);
      bool skip = j0 >= wave_end, docs = false;
      if (with_docs && !skip) {
        const int kd = s_doc[buf][lane];
        skip = __ballot(kd >= wave_lo && kd <= wave_hi) == 0;
        docs = !(wave_lo == wave_hi && __ballot(kd == wave_lo) == ~0ull &&
                 __ballot(doc == wave_lo) == ~0ull);
      }
      if (!skip) {
        f32x16 z[2] = {};
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int k = 0; k < kSteps; ++k) {
            const int r = b * 32 + col;
            const V8 kf = *reinterpret_cast<const V8 *>(
                tk[buf] + r * kD + place_of<kChunks, false>(r, 2 * k + half) * 8);
            z[b] = N::mfma32(kf, qf[k], z[b]);
          }
        __builtin_amdgcn_s_setprio(1);  // a wave that is at its exponentials goes first
        const bool edge = j0 + kBN > all;  // some query does not see some key, documents aside
        // A weight is 2^(z factor - (m - shift)): what is left of a score's way to log2 units,
        // and what all of a lane's scores of the tile have in common.
        float factor = 1.0f, shift = 0.0f;
        if constexpr (kMode == kPlain) {
          factor = P.to_log2;
        } else if constexpr (kMode == kCapped) {
          // cap (1 - 2 f): with f in the place of the score the cap is one more factor
#pragma unroll
          for (int e = 0; e < 32; ++e) z[e >> 4][e & 15] = fall(z[e >> 4][e & 15] * P.cap_in);
          factor = -2.0f * P.cap_out;
          shift = P.cap_out;
        } else if constexpr (kMode == kSloped) {
          const float here = static_cast<float>(place - j0 - 4 * half);
          if (!edge && j0 + kBN <= s.place0 + wave_first + 1) {  // all keys at or before all queries
            shift = -slope2 * here;
#pragma unroll
            for (int e = 0; e < 32; ++e)
              z[e >> 4][e & 15] = __builtin_fmaf(
                  z[e >> 4][e & 15], P.to_log2,
                  slope2 * static_cast<float>((e >> 2) * 8 + (e & 3)));
          } else {
#pragma unroll
            for (int e = 0; e < 32; ++e)
              z[e >> 4][e & 15] = __builtin_fmaf(
                  z[e >> 4][e & 15], P.to_log2,
                  -slope2 * fabsf(here - static_cast<float>((e >> 2) * 8 + (e & 3))));
          }
        } else {
          // what brings a score to log2 units comes with the weight, if it can be undone in the bias
          if (P.capped) {
#pragma unroll
            for (int e = 0; e < 32; ++e) z[e >> 4][e & 15] = cap_score(P, z[e >> 4][e & 15]);
          } else if (late) {
            factor = P.to_log2;
          } else {
#pragma unroll
            for (int e = 0; e < 32; ++e) z[e >> 4][e & 15] *= P.to_log2;
          }
          if (P.slope && !with_pos) {
            const float here = static_cast<float>(place - j0 - 4 * half);
#pragma unroll
            for (int e = 0; e < 32; ++e)
              z[e >> 4][e & 15] = __builtin_fmaf(
                  -rate, fabsf(here - static_cast<float>((e >> 2) * 8 + (e & 3))),
                  z[e >> 4][e & 15]);
          } else if (P.slope) {
            s_far[wave][0][lane] = apart(s_pos[buf][0][lane], x0);
            s_far[wave][1][lane] = apart(s_pos[buf][1][lane], y0);
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
            for (int e = 0; e < 32; e += 4) {
              const int j = (e >> 2) * 8 + 4 * half;
              const f32x4 kx = *reinterpret_cast<const f32x4 *>(&s_far[wave][0][j]);
              const f32x4 ky = *reinterpret_cast<const f32x4 *>(&s_far[wave][1][j]);
#pragma unroll
              for (int r = 0; r < 4; ++r)
                z[e >> 4][(e & 15) + r] =
                    __builtin_fmaf(-rate, fabsf(kx[r] - fx) + fabsf(ky[r] - fy),
                                   z[e >> 4][(e & 15) + r]);
            }
          }
        }
        // a factor < 0 turns the order round
        constexpr float kNone = kMode == kCapped ? INFINITY : -INFINITY;
        if (edge) {
          const int last = limit - j0 - 4 * half;
#pragma unroll
          for (int e = 0; e < 32; ++e)
            if ((e >> 2) * 8 + (e & 3) >= last) z[e >> 4][e & 15] = kNone;
        }
        if (docs) {
#pragma unroll
          for (int e = 0; e < 32; ++e)
            if (s_doc[buf][(e >> 2) * 8 + 4 * half + (e & 3)] != doc) z[e >> 4][e & 15] = kNone;
        }
        float big = kNone;
#pragma unroll
        for (int e = 0; e < 32; e += 2)
          big = kMode == kCapped ? min3(big, z[e >> 4][e & 15], z[e >> 4][(e & 15) + 1])
                                 : max3(big, z[e >> 4][e & 15], z[e >> 4][(e & 15) + 1]);
        big = both_halves(__builtin_fmaf(big, factor, shift));
        if (__ballot(big > m + kSlack)) {
          const float to = fmaxf(m, big);
          const float fix = to == m ? 1.0f : __builtin_amdgcn_exp2f(m - to);
          m = to;
          l *= fix;
#pragma unroll
          for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[b][r] *= fix;
        }
        const float base = shift - (m == -INFINITY ? 0.0f : m) + kLift<kType>;
        __builtin_amdgcn_s_setprio(0);
#pragma unroll
        for (int k = 0; k < 4; ++k) {  // 16 keys
          V8 pf;
#pragma unroll
          for (int e = 0; e < 8; e += 2) {
            const float p0 = __builtin_amdgcn_exp2f(
                __builtin_fmaf(z[k >> 1][(k & 1) * 8 + e], factor, base));
            const float p1 = __builtin_amdgcn_exp2f(
                __builtin_fmaf(z[k >> 1][(k & 1) * 8 + e + 1], factor, base));
            const auto two = pack2<kType>(p0, p1);
            l = add2<kType>(two, l);
            pf[e] = two[0];
            pf[e + 1] = two[1];
          }
          const int i16 = lane & 15, g = (lane >> 4) & 1;
#pragma unroll
          for (int b = 0; b < kBlocks; ++b) {
            const int r0 = k * 16 + 4 * half + (i16 >> 2);
            const int c = 4 * b + 2 * g + ((i16 & 3) >> 1);
            const V4 v0 = read_transposed<kType>(
                tv[buf] + r0 * kD + place_of<kChunks, false>(r0, c) * 8 + (i16 & 1) * 4);
            const V4 v1 = read_transposed<kType>(
                tv[buf] + (r0 + 8) * kD + place_of<kChunks, false>(r0 + 8, c) * 8 +
                (i16 & 1) * 4);
            const V8 vf = __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
            acc[b] = N::mfma32(vf, pf, acc[b]);
          }
        }
      }
      t = after;
      buf ^= 1;
    }
  }

  l += __shfl_xor(l, 32);
  if (with_docs && below_zero(doc)) {  // keys of document INT_MIN are not seen either
    m = -INFINITY;
    l = 0.0f;
  }
  if (scattered) l = NAN;  // for strict_row: a second formula in the loop spilled registers
  if (P.splits > 1) {
    const int64_t to = (int64_t(split) * P.n_q_rows + row) * P.n_heads + head;
    if (!live) return;
    if (half == 0) {
      P.part_ml[to * 2] = m;
      P.part_ml[to * 2 + 1] = l;
    }
    if (m == -INFINITY) return;  // the sums are not looked at
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        const int c = b * 32 + r4 * 8 + 4 * half;
        if (c < P.d)
          *reinterpret_cast<f32x4 *>(P.part + to * P.d + c) =
              f32x4{acc[b][r4 * 4], acc[b][r4 * 4 + 1], acc[b][r4 * 4 + 2], acc[b][r4 * 4 + 3]};
      }
    return;
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  bool fine = full_sum(m, l, with_docs || limit <= 0);
  E *o = static_cast<E *>(P.out) + row * P.out_stride + head * P.out_head;
#pragma unroll
  for (int b = 0; b < kBlocks; ++b)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
      const int c = b * 32 + r4 * 8 + 4 * half;
      f32x4 v;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        v[r] = l == 0.0f ? 0.0f : acc[b][r4 * 4 + r] * inv;
        fine = fine && fabsf(v[r]) < INFINITY;
      }
      if (live && c < P.d) *reinterpret_cast<V4 *>(o + c) = __builtin_convertvector(v, V4);
    }
  uint64_t bad = __ballot(!fine && live);
  bad = (bad | (bad >> 32)) & 0xFFFFFFFFull;
  for (; bad; bad &= bad - 1)
    strict_row<kType>(P, s, wave_first + __builtin_ctzll(bad), head);
}

// Joins the parts of a tile's rows, 32 rows of a head a workgroup, 32 lanes a row with 4 values
// each.
constexpr int kMaxSplits = 16, kJoinRows = 32;
template <int kType>
__global__ __launch_bounds__(kThreads) void join_tile_kernel(const AttendParams P) {
  typedef typename Num<kType>::E E;
  typedef typename Num<kType>::V4 V4;
  constexpr int kEach = kJoinRows * 32 / kThreads, kStep = kThreads / 32;
  const int c = (threadIdx.x & 31) * 4, group = threadIdx.x >> 5;
  const int head = blockIdx.x % P.n_heads, id = blockIdx.x / P.n_heads;
  int first;
  const Seq s = sequence_of(P, id / (kBM / kJoinRows), kBM, first);
  if (first < 0) return;
  first += id % (kBM / kJoinRows) * kJoinRows;
  if (first >= s.nq) return;
  float pm[kEach][kMaxSplits], pl[kEach][kMaxSplits];
  f32x4 sum[kEach];
  uint32_t bad = 0;
#pragma unroll
  for (int u = 0; u < kEach; ++u) {
    const int i = min(first + u * kStep + group, s.nq - 1);
    const int64_t at = (int64_t(s.q0) + i) * P.n_heads + head;
    const int64_t step = int64_t(P.n_q_rows) * P.n_heads;
#pragma unroll
    for (int k = 0; k < kMaxSplits; ++k) {
      pm[u][k] = -INFINITY;
      pl[u][k] = 0.0f;
      if (k < P.splits) {
        pm[u][k] = P.part_ml[(k * step + at) * 2];
        pl[u][k] = P.part_ml[(k * step + at) * 2 + 1];
      }
    }
  }
#pragma unroll
  for (int u = 0; u < kEach; ++u) {
    const int i = first + u * kStep + group;
    const int64_t at = (int64_t(s.q0) + min(i, s.nq - 1)) * P.n_heads + head;
    const int64_t step = int64_t(P.n_q_rows) * P.n_heads;
    float top = -INFINITY, total = 0.0f;
#pragma unroll
    for (int k = 0; k < kMaxSplits; ++k) top = fmaxf(top, pm[u][k]);
    sum[u] = f32x4{};
#pragma unroll
    for (int k = 0; k < kMaxSplits; ++k)
      if (pm[u][k] != -INFINITY) {
        const float f = __builtin_amdgcn_exp2f(pm[u][k] - top);
        total += f * pl[u][k];
        if (c < P.d)
          sum[u] += f * *reinterpret_cast<const f32x4 *>(P.part + (k * step + at) * P.d + c);
      } else {
        total += pl[u][k];  // 0, or NaN where NaN is all that was seen of the part
      }
    bool fine = full_sum(top, total, key_limit(P, s, i) <= 0);  // no documents here
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      sum[u][q] = total == 0.0f ? 0.0f : sum[u][q] / total;
      fine = fine && fabsf(sum[u][q]) < INFINITY;
    }
    E *o = static_cast<E *>(P.out) + (int64_t(s.q0) + i) * P.out_stride + head * P.out_head;
    if (i < s.nq && c < P.d) *reinterpret_cast<V4 *>(o + c) = __builtin_convertvector(sum[u], V4);
    const uint64_t worse = __ballot(!fine && i < s.nq && c < P.d);
    bad |= ((worse & 0xFFFFFFFFull ? 1u : 0u) | (worse >> 32 ? 2u : 0u)) << (2 * u);
  }
  const int low = __builtin_amdgcn_readfirstlane(group);  // the row of the wave's first half
  for (; bad; bad &= bad - 1) {
    const int at = __builtin_ctz(bad);
    strict_row<kType>(P, s, first + (at >> 1) * kStep + low + (at & 1), head);
  }
}

// ------------------------------------------------------------------------ few queries

// How the keys of all sequences are cut: parts of one length, so that every workgroup has as much
// to read, whatever the lengths are. A wave works it out; the host knows bounds only.
constexpr int kMaxCut = 256;   // sequences, where any is cut
// Parts have 128 keys at least; where that makes more than one workgroup a place, up to 512, for
// one workgroup a place; beyond, for three (20 queries, 16 heads of 64 over 4, 1,600 keys each, 256
// keys a part and not 128: 15.0 us for 17.5; 64 queries, 8 heads of 128 over 2, 1,200 keys each:
// 27 for 33; 64 queries, 16 heads of 128 over 4, 2,200 keys each, 512 and not 384: 63 for 62).
constexpr int kMinPart = 128, kOneRound = 512;

struct Parts {
  int chunk;   // keys of a part
  int seq;     // the sequence asked for, -1: there is none
  int first;   // its first part
  int count;   // its parts
  Seq s;       // what else is known of it
};

// `part` >= 0: the sequence that has it; otherwise sequence `seq`.
__device__ __forceinline__ Parts find_parts(const AttendParams &P, int part, int seq) {
  const int lane = threadIdx.x & 63;
  constexpr int kEach = kMaxCut / 64;
  int nk[kEach];
  Seq all[kEach];
  int64_t total = 0;
#pragma unroll
  for (int u = 0; u < kEach; ++u) {
    nk[u] = -1;  // no queries: no part
    if (u * 64 >= P.n_seqs) continue;
    if (u * 64 + lane < P.n_seqs) {
      all[u] = sequence(P, u * 64 + lane);
      if (all[u].nq > 0) nk[u] = all[u].nk;
    }
    total += max(nk[u], 0);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) total += __shfl_xor(total, o);
  Parts r = {kMinPart, -1, 0, 0, {}};
  const auto even = [&](int parts) {
    return static_cast<int>(((total + parts - 1) / parts + 63) / 64 * 64);
  };
  const int one = even((P.width + 2) / 3);
  if (one >= 2 * kMinPart) r.chunk = min(one, kOneRound);
  r.chunk = max(r.chunk, even(P.width));
  int before = 0;
#pragma unroll
  for (int u = 0; u < kEach; ++u) {
    if (u * 64 >= P.n_seqs) continue;
    const int mine = nk[u] < 0 ? 0 : max((nk[u] + r.chunk - 1) / r.chunk, 1);
    int upto = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(upto, o);
      if (lane >= o) upto += v;
    }
    const uint64_t at = part >= 0 ? __ballot(before + upto > part)
                                  : (seq >= u * 64 && seq < u * 64 + 64 ? 1ull << (seq & 63) : 0);
    if (at && r.seq < 0) {
      const int l = __builtin_amdgcn_readfirstlane(__builtin_ctzll(at));
      r.seq = u * 64 + l;
      r.count = __shfl(mine, l);
      r.first = before + __shfl(upto, l) - r.count;
      r.s = broadcast(all[u], l);
    }
    before += __shfl(upto, 63);
  }
  r.seq = __builtin_amdgcn_readfirstlane(r.seq);
  r.first = __builtin_amdgcn_readfirstlane(r.first);
  r.count = __builtin_amdgcn_readfirstlane(r.count);
  r.chunk = __builtin_amdgcn_readfirstlane(r.chunk);
  return r;
}

// Rows of a workgroup: 16 (query, head) pairs that share a key head, query-major. Each of its two
// waves takes every second 32 keys of the workgroup's range through LDS of its own; two waves, so
// that several workgroups fit a CU and one's start and end fall into another's loads. The query
// heads of a key head are rows of one tile, so keys are read once: memory bounds it. bfloat16, 16
// heads of 128 over 2, 8 queries against up to 100,003 keys each, 467 MB: 93 us, 5.0 TB/s, and 9
// for the join; 20 queries, heads of 64 over 4, up to 1,600 keys, 18 MB: 9 us and 5, where a chain
// of loads (lengths, then queries, then keys) takes most of it.
constexpr int kFewWaves = 2;
constexpr int kFewWorkgroups = 1536;  // that the keys are cut for: 3 for each of the 512 places

template <int kType, int kD>
__global__ __launch_bounds__(kFewWaves * 64) void attend_few_kernel(const AttendParams P) {
  typedef Num<kType> N;
  typedef typename N::E E;
  typedef typename N::V4 V4;
  typedef typename N::V8 V8;
  constexpr int kChunks = kD / 8, kSteps = kD / 32, kBlocks = kD / 16, kKeys = 32;
  __shared__ __attribute__((aligned(16))) E tile[kFewWaves][2][2][kKeys * kD];
  __shared__ int s_marks[kFewWaves][2][3][64];  // documents and positions of a step's keys
  __shared__ float s_m[kFewWaves][16], s_l[kFewWaves][16];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, quad = lane >> 4;
  int id = workgroup();
  const int kvh = id % P.n_kv_heads;
  id /= P.n_kv_heads;
  const int rt = id % P.row_tiles;
  id /= P.row_tiles;
  Parts parts = {0, id, id, 1, {}};
  if (P.width > 0) {
    parts = find_parts(P, id, -1);
    if (parts.seq < 0) return;
  } else {
    if (id >= P.n_seqs) return;
    parts.s = sequence(P, id);
  }
  const Seq s = parts.s;
  const int rows = s.nq * P.group;
  if (rt * 16 >= rows) return;
  const int from = (id - parts.first) * parts.chunk;
  const int my = rt * 16 + col;  // this lane's row
  const bool live = my < rows;
  const int i = (live ? my : rows - 1) / P.group;
  const int head = kvh * P.group + (live ? my : rows - 1) % P.group;
  int end = key_limit(P, s, (min(rt * 16 + 16, rows) - 1) / P.group);
  if (parts.count > 1) end = min(end, from + parts.chunk);
  const int all = key_limit(P, s, rt * 16 / P.group);
  const int64_t row = int64_t(s.q0) + i;
  const void *kb = static_cast<const E *>(P.k) + kvh * P.k_head;
  const void *vb = static_cast<const E *>(P.v) + kvh * P.v_head;
  auto fetch = [&](int j0, int to) {
    load_rows<kKeys, kChunks, true, 1>(kb, P.k_stride, s.k0 + j0, s.nk - j0, P.d,
                                       tile[wave][to][0], 0, 0);
    load_rows<kKeys, kChunks, true, 1>(vb, P.v_stride, s.k0 + j0, s.nk - j0, P.d,
                                       tile[wave][to][1], 0, 0);
    if (P.k_doc) load_marks<kKeys>(P.k_doc, s.k0 + j0, s.nk - j0, 1, 0, s_marks[wave][to][0]);
    if (P.k_pos) {
      load_marks<kKeys>(P.k_pos, s.k0 + j0, s.nk - j0, 2, 0, s_marks[wave][to][1]);
      load_marks<kKeys>(P.k_pos, s.k0 + j0, s.nk - j0, 2, 1, s_marks[wave][to][2]);
    }
  };
  int j0 = from + wave * kKeys, buf = 0;
  if (j0 < end) fetch(j0, 0);
  const E *qr = static_cast<const E *>(P.q) + row * P.q_stride + head * P.q_head;
  V8 qf[kSteps];
#pragma unroll
  for (int k = 0; k < kSteps; ++k) {
    qf[k] = V8{};
    if (k * 32 + quad * 8 < P.d) qf[k] = *reinterpret_cast<const V8 *>(qr + k * 32 + quad * 8);
  }
  const int limit = live ? key_limit(P, s, i) : 0;
  int doc = P.q_doc ? P.q_doc[row] : 0;
  const float slope2 = P.slope ? P.slope[head] * kLog2e : 0.0f;
  const int place = s.place0 + i;
  int px = 0, py = 0;
  if (P.q_pos) {
    px = P.q_pos[2 * row];
    py = P.q_pos[2 * row + 1];
  }
  if (doc < 0) doc = INT_MIN;
  f32x4 acc[kBlocks] = {};
  float m = -INFINITY, l = 0.0f;
  const float unit = P.shaped ? 1.0f : P.to_log2;
  for (; j0 < end; j0 += kFewWaves * kKeys) {
    wait_loads();
    const E *tk = tile[wave][buf][0], *tv = tile[wave][buf][1];
    const int(*marks)[64] = s_marks[wave][buf];
    if (j0 + kFewWaves * kKeys < end) fetch(j0 + kFewWaves * kKeys, buf ^ 1);
    f32x4 z[2] = {};
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int k = 0; k < kSteps; ++k) {
        const int r = b * 16 + col;
        const V8 kf = *reinterpret_cast<const V8 *>(
            tk + r * kD + place_of<kChunks, true>(r, 4 * k + quad) * 8);
        z[b] = N::mfma16(kf, qf[k], z[b]);
      }
    if (P.shaped) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int at = (e >> 2) * 16 + 4 * quad + (e & 3);
        float far = 0.0f;
        if (P.slope)
          far = P.k_pos ? abs_diff(px, marks[1][at]) + abs_diff(py, marks[2][at])
                        : abs_diff(place, j0 + at);
        z[e >> 2][e & 3] = shape(P, z[e >> 2][e & 3], slope2, far);
      }
    }
    if (j0 + kKeys > all) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (j0 + (e >> 2) * 16 + 4 * quad + (e & 3) >= limit) z[e >> 2][e & 3] = -INFINITY;
    }
    if (P.k_doc) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (marks[0][(e >> 2) * 16 + 4 * quad + (e & 3)] != doc) z[e >> 2][e & 3] = -INFINITY;
    }
    float big = -INFINITY;
#pragma unroll
    for (int e = 0; e < 8; e += 2) big = max3(big, z[e >> 2][e & 3], z[e >> 2][(e & 3) + 1]);
    big *= unit;
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
        for (int r = 0; r < 4; ++r) acc[b][r] *= fix;
    }
    const float base = (m == -INFINITY ? 0.0f : m) - kLift<kType>;
    V8 pf;
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const float p0 =
          __builtin_amdgcn_exp2f(__builtin_fmaf(z[e >> 2][e & 3], unit, -base));
      const float p1 =
          __builtin_amdgcn_exp2f(__builtin_fmaf(z[e >> 2][(e & 3) + 1], unit, -base));
      const auto two = pack2<kType>(p0, p1);
      l = add2<kType>(two, l);
      pf[e] = two[0];
      pf[e + 1] = two[1];
    }
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) {
      const int r0 = 4 * quad + (col >> 2), c = 2 * b + ((col & 3) >> 1);
      const V4 v0 = read_transposed<kType>(
          tv + r0 * kD + place_of<kChunks, true>(r0, c) * 8 + (col & 1) * 4);
      const V4 v1 = read_transposed<kType>(
          tv + (r0 + 16) * kD + place_of<kChunks, true>(r0 + 16, c) * 8 + (col & 1) * 4);
      const V8 vf = __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
      acc[b] = N::mfma16(vf, pf, acc[b]);
    }
    buf ^= 1;
  }
  // the waves' ranges are joined through LDS
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  if (below_zero(doc)) {  // sees nothing, nor keys of document INT_MIN
    m = -INFINITY;
    l = 0.0f;
  }
  __syncthreads();  // the tiles are done with
  float *sums = reinterpret_cast<float *>(&tile[0][0][0][0]);  // [kFewWaves][16][kD]
  if (quad == 0) {
    s_m[wave][col] = m;
    s_l[wave][col] = l;
  }
#pragma unroll
  for (int b = 0; b < kBlocks; ++b)
    *reinterpret_cast<f32x4 *>(sums + (wave * 16 + col) * kD + b * 16 + quad * 4) = acc[b];
  __syncthreads();
  constexpr int kLanes = kFewWaves * 4;  // threads of a row
  const int r = threadIdx.x / kLanes, c0 = threadIdx.x % kLanes;
  const int mine = rt * 16 + r;
  float top = -INFINITY;
#pragma unroll
  for (int w = 0; w < kFewWaves; ++w) top = fmaxf(top, s_m[w][r]);
  float f[kFewWaves], total = 0.0f;
#pragma unroll
  for (int w = 0; w < kFewWaves; ++w) {
    f[w] = s_m[w][r] == top ? 1.0f : __builtin_amdgcn_exp2f(s_m[w][r] - top);
    total += f[w] * s_l[w][r];
  }
  const int64_t orow = int64_t(s.q0) + min(mine, rows - 1) / P.group;
  const int ohead = kvh * P.group + min(mine, rows - 1) % P.group;
  const int64_t flat = (int64_t(id) * P.n_kv_heads + kvh) * P.row_tiles * 16 + mine;
  float *part = P.part + flat * P.d;
  E *o = static_cast<E *>(P.out) + orow * P.out_stride + ohead * P.out_head;
  bool fine = full_sum(top, total, P.k_doc || mine >= rows ||
                                       key_limit(P, s, static_cast<int>(orow - s.q0)) <= 0);
#pragma unroll
  for (int b = 0; b < kD / 4 / kLanes; ++b) {
    const int c = (b * kLanes + c0) * 4;
    f32x4 v = {};
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w)
      v += f[w] * *reinterpret_cast<const f32x4 *>(sums + (w * 16 + r) * kD + c);
    if (mine < rows && c < P.d) {
      if (parts.count == 1) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          v[q] = total == 0.0f ? 0.0f : v[q] / total;
          fine = fine && fabsf(v[q]) < INFINITY;
        }
        *reinterpret_cast<V4 *>(o + c) = __builtin_convertvector(v, V4);
      } else {
        *reinterpret_cast<f32x4 *>(part + c) = v;
      }
    }
  }
  if (parts.count > 1) {
    if (mine < rows && c0 == 0) {
      P.part_ml[flat * 2] = top;
      P.part_ml[flat * 2 + 1] = total;
    }
    return;
  }
  for (uint64_t bad = __ballot(!fine); bad;) {
    const int w = __builtin_ctzll(bad) / kLanes;  // row of the wave
    bad &= ~(((1ull << kLanes) - 1) << (kLanes * w));
    const int rr = rt * 16 + wave * (64 / kLanes) + w;
    strict_row<kType>(P, s, rr / P.group, kvh * P.group + rr % P.group);
  }
}

// Joins the parts of a row: a workgroup a row, 32 lanes a part with 4 values each.
template <int kType>
__global__ __launch_bounds__(kThreads, 4) void join_kernel(const AttendParams P) {
  typedef typename Num<kType>::E E;
  typedef typename Num<kType>::V4 V4;
  constexpr int kAtOnce = kThreads / 32;
  __shared__ f32x4 s_sum[kAtOnce][32];
  __shared__ float s_w[64];
  __shared__ int s_bad;
  const int tid = threadIdx.x, lane = tid & 63, group = tid >> 5, c = (tid & 31) * 4;
  const int per = P.row_tiles * 16;       // rows of a sequence and key head in the parts
  const int most = P.max_q * P.group;     // and those that may be in use
  int id = blockIdx.x;
  const int my = id % most;
  id /= most;
  const int kvh = id % P.n_kv_heads, si = id / P.n_kv_heads;
  const Parts parts = find_parts(P, -1, si);
  const Seq s = parts.s;
  const int rows = s.nq * P.group;
  if (my >= rows || parts.count <= 1) return;
  const int i = my / P.group, head = kvh * P.group + my % P.group;
  const int n = parts.count;
  const int64_t step = int64_t(P.n_kv_heads) * per;  // rows of a part
  const int64_t flat = (int64_t(parts.first) * P.n_kv_heads + kvh) * per + my;
  float top = -INFINITY, total = 0.0f;
  f32x4 sum = {};
  for (int k0 = 0; k0 < n; k0 += 64) {  // lane k of every wave has part k's maximum and sum
    float pm = -INFINITY, pl = 0.0f;
    if (k0 + lane < n) {
      pm = P.part_ml[((k0 + lane) * step + flat) * 2];
      pl = P.part_ml[((k0 + lane) * step + flat) * 2 + 1];
    }
    f32x4 v[64 / kAtOnce];
#pragma unroll
    for (int u = 0; u < 64 / kAtOnce; ++u) {
      const int k = k0 + u * kAtOnce + group;
      v[u] = f32x4{};
      if (k < n && c < P.d)
        v[u] = *reinterpret_cast<const f32x4 *>(P.part + (k * step + flat) * P.d + c);
    }
    const float to = fmaxf(top, wave_max(pm));
    const float fix = top == to ? 1.0f : __builtin_amdgcn_exp2f(top - to);
    const float f = pm == to ? 1.0f : __builtin_amdgcn_exp2f(pm - to);
    top = to;
    total = total * fix + wave_sum(f * pl);
    sum *= fix;
    if (k0 > 0) __syncthreads();
    if (tid < 64) s_w[lane] = f;
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 64 / kAtOnce; ++u) {
      const int k = u * kAtOnce + group;
      if (k0 + k < n) sum += s_w[k] * v[u];
    }
  }
  s_sum[group][tid & 31] = sum;
  if (tid == 0) s_bad = 0;
  __syncthreads();
  if (group == 0 && c < P.d) {
#pragma unroll
    for (int g = 1; g < kAtOnce; ++g) sum += s_sum[g][tid];
    bool fine = full_sum(top, total, P.k_doc || key_limit(P, s, i) <= 0);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      sum[q] = total == 0.0f ? 0.0f : sum[q] / total;
      fine = fine && fabsf(sum[q]) < INFINITY;
    }
    E *o = static_cast<E *>(P.out) + (int64_t(s.q0) + i) * P.out_stride + head * P.out_head;
    *reinterpret_cast<V4 *>(o + c) = __builtin_convertvector(sum, V4);
    if (!fine) s_bad = 1;
  }
  __syncthreads();
  if (s_bad && tid < 64) strict_row<kType>(P, s, i, head);
}

// ------------------------------------------------------------------------------- the host

// The form for few queries: 16-row tiles of a key head's rows, and into how many parts the keys
// of all sequences are cut; or into how many those of a tile of the other form are.
struct Few {
  bool use;
  int row_tiles, width;
  int splits;  // of the other form
};

constexpr int kFewRows = 64;
// Of the form for few queries, keys that are not cut, as the join's launch costs more: up to 512,
// or 1,024 where the sequences alone make 64 workgroups. 16 heads, us cut and not: 20 queries of
// heads of 64 over 4, 500 keys 12.4, 8.8, 1,000 keys 13.0, 13.1; of heads of 128, 700 keys 17.7,
// 15.0; 64 queries, 8 heads of 128 over 2, 1,000 keys 28, 20; but 1 query, 32 heads over 8, 1,000
// keys 12.7, 18.6.
constexpr int kWhole = 512, kWholeOfMany = 1024, kManyWorkgroups = 64;
int whole_keys(int64_t workgroups) {
  return workgroups >= kManyWorkgroups ? kWholeOfMany : kWhole;
}
// Of the other form, the workgroups that tiles' keys are cut for, and the key tiles of a part.
constexpr int kTileWorkgroups = 768, kTilesOfPart = 12;
int64_t key_tiles(int max_kv) { return (int64_t(max_kv) + kBN - 1) / kBN; }

Few few_of(int n_seqs, int n_q_rows, int max_q, int max_kv, int n_heads, int n_kv_heads,
            bool causal, bool docs) {
  Few r = {};
  const int64_t rows = int64_t(max_q) * (n_heads / n_kv_heads);
  const int64_t each = n_kv_heads * ((rows + 15) / 16);
  r.use = rows <= kFewRows;
  if (!r.use) {
    // Tiles' keys are cut where the tiles alone would leave CUs idle: for 768 workgroups, or for 512
    // where most rows see about half of the keys, of 12 key tiles or more each, since the join
    // and the parts' way through memory cost about as much as 7. Not with documents, which leave
    // most tiles out. bfloat16, causal, heads of 128 over a quarter as many, us with 1, 2, 4, 8
    // and 16 parts:
    //    16 tiles, 64 queries, 32,768 keys: 591, 310, 166, 100, 77
    //    96 tiles, 4 times the same:        602, 332, 231, 179, 198
    //   384 tiles, 16 times the same:       909, 629, 639, 673, 716
    //    72 tiles, 1,024 queries of 16,384: 303, 169, 101,  92, 113
    //   132 tiles, 4,096 queries and keys:   79,  54,  43,  52
    //   272 tiles, 2,048:                    45,  40,  49,  71
    //   144 tiles, 1,024:                    25,  24,  28,  42
    //   528 tiles, 4,096:                    92,  97, 115, 182
    const int64_t blocks = (int64_t(n_q_rows) / kBM + n_seqs) * n_heads;
    const int64_t want = causal && max_q > max_kv / 2 ? 512 : kTileWorkgroups;
    const int64_t splits = std::min(
        {(want + blocks / 2) / blocks, key_tiles(max_kv) / kTilesOfPart, int64_t(kMaxSplits)});
    r.splits = docs || splits < 1 ? 1 : static_cast<int>(splits);
    return r;
  }
  r.row_tiles = static_cast<int>((rows + 15) / 16);
  const int64_t want = kFewWorkgroups;
  if (n_seqs <= kMaxCut && n_seqs * each < want && max_kv > whole_keys(n_seqs * each))
    r.width = static_cast<int>((want + each - 1) / each);
  return r;
}

template <int kType, int kD>
int launch(AttendParams P, const Few &few, hipStream_t s) {
  if (few.use) {
    const int64_t blocks = (int64_t(P.n_seqs) + P.width) * P.n_kv_heads * P.row_tiles;
    const int64_t joined = int64_t(P.n_seqs) * P.n_heads * P.max_q;
    if (blocks > kMaxWorkgroups || joined > INT32_MAX) return TG_E_INVAL;
    hipLaunchKernelGGL((attend_few_kernel<kType, kD>), grid_of(blocks, kFewWaves * 64),
                       dim3(kFewWaves * 64), 0, s, P);
    if (P.width > 0)
      hipLaunchKernelGGL(join_kernel<kType>, dim3(static_cast<uint32_t>(joined)), dim3(kThreads), 0,
                         s, P);
  } else {
    const int64_t tiles = (int64_t(P.n_q_rows) / kBM + P.n_seqs) * P.n_heads;
    if (tiles * P.splits > kMaxWorkgroups) return TG_E_INVAL;
    P.turns = static_cast<int32_t>(tiles / P.n_heads * P.splits);
    const dim3 grid = grid_of(tiles * P.splits, kThreads), threads(kThreads);
    const bool any = P.k_doc || P.k_pos || P.capped == 2 || !(P.to_log2 > 0.0f);
    if (any || (P.capped && P.slope))
      hipLaunchKernelGGL((attend_tile_kernel<kType, kD, kAny>), grid, threads, 0, s, P);
    else if (P.capped)
      hipLaunchKernelGGL((attend_tile_kernel<kType, kD, kCapped>), grid, threads, 0, s, P);
    else if (P.slope)
      hipLaunchKernelGGL((attend_tile_kernel<kType, kD, kSloped>), grid, threads, 0, s, P);
    else
      hipLaunchKernelGGL((attend_tile_kernel<kType, kD, kPlain>), grid, threads, 0, s, P);
    if (P.splits > 1)
      hipLaunchKernelGGL(join_tile_kernel<kType>,
                         dim3(static_cast<uint32_t>(tiles * (kBM / kJoinRows))), threads, 0, s, P);
  }
  return hipGetLastError() == hipSuccess ? TG_OK : TG_E_HIP;
}

bool layout_ok(const void *p, int64_t stride, int64_t head) {
  return p && aligned16(p) && stride >= 0 && stride <= kMaxStride && stride % 8 == 0 &&
         head >= 0 && head % 8 == 0;
}

bool sizes_ok(int n_seqs, int n_q_rows, int max_q, int max_kv, int n_heads, int n_kv_heads,
              int d) {
  return n_seqs >= 0 && n_q_rows >= 0 && max_q >= 0 && max_kv >= 0 && n_heads >= 1 &&
         n_kv_heads >= 1 && n_heads % n_kv_heads == 0 && d >= 8 && d <= TG_ATTEND_MAX_D &&
         d % 8 == 0;
}

}  // namespace

// What a call needs, and every call of fewer sequences, rows or shorter ones with it: those have
// more parts, or take the other form. The largest product of parts and rows is looked for per rows
// of 16 in the form for few queries, and per number of parts in the other.
extern "C" size_t tg_attend_workspace_bytes(int32_t n_seqs, int32_t n_q_rows, int32_t max_q_len,
                                            int32_t max_kv_len, int32_t n_heads,
                                            int32_t n_kv_heads, int32_t d) {
  if (!sizes_ok(n_seqs, n_q_rows, max_q_len, max_kv_len, n_heads, n_kv_heads, d)) return 0;
  if (n_seqs == 0 || n_q_rows == 0 || max_q_len == 0) return 0;
  const int64_t group = n_heads / n_kv_heads;
  int64_t rows = 0;  // rows of d sums, a maximum and a sum of weights
  const int64_t few_q = std::min<int64_t>(max_q_len, kFewRows / group);
  for (int64_t row_tiles = 1; row_tiles <= (few_q * group + 15) / 16; ++row_tiles) {
    const int64_t each = n_kv_heads * row_tiles;
    if (max_kv_len <= whole_keys(each)) continue;
    const int64_t most = max_kv_len <= kWholeOfMany ? kManyWorkgroups : kFewWorkgroups;
    const int64_t seqs = std::min<int64_t>({n_seqs, kMaxCut, (most - 1) / each});
    if (seqs > 0) rows = std::max(rows, ((kFewWorkgroups + each - 1) / each + seqs) * each * 16);
  }
  if (max_q_len * group > kFewRows) {
    const int64_t most = std::min<int64_t>(key_tiles(max_kv_len) / kTilesOfPart, kMaxSplits);
    for (int64_t splits = 2; splits <= most; ++splits) {
      // the most tiles that are cut into so many, and the most rows that these can have
      const int64_t tiles = 2 * kTileWorkgroups / (2 * splits - 1) / n_heads;
      if (tiles > 0)
        rows = std::max(rows, splits * std::min<int64_t>(n_q_rows, tiles * kBM - 1) * n_heads);
    }
  }
  return static_cast<size_t>(rows) * (d + 2) * sizeof(float);
}

extern "C" int tg_attend(const tg_attend_args *a, void *stream) {
  if (!a || !type_ok(a->type) ||
      !sizes_ok(a->n_seqs, a->n_q_rows, a->max_q_len, a->max_kv_len, a->n_heads, a->n_kv_heads,
                a->d) ||
      a->n_k_rows < 0 || !std::isfinite(a->scale) || !std::isfinite(a->cap) || a->cap < 0.0f)
    return TG_E_INVAL;
  if (a->prefix && !a->causal) return TG_E_INVAL;
  if (a->n_seqs == 0 || a->n_q_rows == 0 || a->max_q_len == 0) return TG_OK;
  // arrays of no rows may be null; where there is no key, nothing asks for the queries' either
  const bool keys = a->n_k_rows > 0;
  if (keys && ((a->q_doc == nullptr) != (a->k_doc == nullptr) ||
               (a->q_pos == nullptr) != (a->k_pos == nullptr)))
    return TG_E_INVAL;
  if (!a->q_begin || !a->kv_begin || !a->kv_len || !layout_ok(a->q, a->q_stride, a->q_head_stride) ||
      !layout_ok(a->out, a->out_stride, a->out_head_stride))
    return TG_E_INVAL;
  if (keys && (!layout_ok(a->k, a->k_stride, a->k_head_stride) ||
               !layout_ok(a->v, a->v_stride, a->v_head_stride)))
    return TG_E_INVAL;
  const Few few = few_of(a->n_seqs, a->n_q_rows, a->max_q_len, a->max_kv_len, a->n_heads,
                         a->n_kv_heads, a->causal != 0, a->q_doc != nullptr);
  // rows of the parts that this call writes
  const size_t parts =
      few.use ? few.width == 0 ? 0
                               : (static_cast<size_t>(few.width) + a->n_seqs) * a->n_kv_heads *
                                     few.row_tiles * 16
              : few.splits == 1 ? 0 : static_cast<size_t>(few.splits) * a->n_q_rows * a->n_heads;
  const size_t written = parts * (a->d + 2) * sizeof(float);
  const size_t need = tg_attend_workspace_bytes(a->n_seqs, a->n_q_rows, a->max_q_len,
                                                a->max_kv_len, a->n_heads, a->n_kv_heads, a->d);
  if (need > 0 && (!a->workspace || a->workspace_bytes < std::max(need, written) ||
                   !aligned16(a->workspace)))
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
  P.q_begin = a->q_begin;
  P.kv_begin = a->kv_begin;
  P.kv_len = a->kv_len;
  P.prefix = a->prefix;
  P.q_doc = keys ? a->q_doc : nullptr;
  P.k_doc = keys ? a->k_doc : nullptr;
  P.q_pos = keys && a->slope ? a->q_pos : nullptr;  // nothing else asks for places
  P.k_pos = keys && a->slope ? a->k_pos : nullptr;
  P.slope = a->slope;
  // Scales and caps at the ends of binary32: a factor past it is its largest number (a score that
  // is not 0 is past tanh's range with either, and 0 stays 0). Of a cap so large that no score
  // reaches tanh's bend, any other such will do.
  const auto factor = [](double v) {
    return static_cast<float>(std::min(std::max(v, -double(FLT_MAX)), double(FLT_MAX)));
  };
  P.to_log2 = factor(double(a->scale) * kLog2e);
  if (a->cap > 0.0f) {
    const double cap = std::min<double>(
        a->cap, 0x1p100 * std::min(std::max(std::fabs(double(a->scale)), 1.0), 0x1p26));
    P.capped = cap <= kFastCap ? 1 : 2;
    P.cap_arg = factor(a->scale / cap);
    P.cap_in = factor(2.0 * kLog2e * a->scale / cap);
    P.cap_out = static_cast<float>(cap * kLog2e);
  }
  P.shaped = P.capped || a->slope || !(P.to_log2 > 0.0f);
  P.causal = a->causal != 0;
  P.n_seqs = a->n_seqs;
  P.n_q_rows = a->n_q_rows;
  P.n_k_rows = a->n_k_rows;
  P.max_q = a->max_q_len;
  P.max_kv = a->max_kv_len;
  P.n_heads = a->n_heads;
  P.n_kv_heads = a->n_kv_heads;
  P.group = a->n_heads / a->n_kv_heads;
  P.d = a->d;
  P.row_tiles = few.row_tiles;
  P.width = few.width;
  P.part = static_cast<float *>(a->workspace);
  P.splits = few.splits;
  P.part_ml = P.part + parts * a->d;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (a->d <= 64)
    return a->type == TG_F16 ? launch<TG_F16, 64>(P, few, s) : launch<TG_BF16, 64>(P, few, s);
  return a->type == TG_F16 ? launch<TG_F16, 128>(P, few, s) : launch<TG_BF16, 128>(P, few, s);
}
