// tg_pages: the pages of a cache given back and taken, page tables, and a cache row for every new
// token of a step, from lengths that stay on the device.
//
// What each sequence gets depends on what all before it have asked for, so one workgroup goes over
// the sequences, kThreads at a time, with a prefix sum of pages each: first of those that go back,
// which are pushed on the stack, then of those that are asked for, which come off its top. No
// sequence waits for another's write: a page that is taken is read from the stack by whoever needs
// it. The rows of new tokens come with it where they are few; many are a second kernel's, a thread
// a few tokens, which finds a token's sequence by bisection. There is next to nothing to read, so a
// chain of loads bounds it (lengths, stack, then the stores).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <cstdint>

#include "tg.h"
#include "token_math.h"

namespace {

using namespace tok;

constexpr int kThreads = 1024, kWaves = kThreads / 64;
// Tokens up to here are given their rows by the first kernel.
constexpr int kFewTokens = 4096;

struct PagesParams {
  const int32_t *q_begin, *kv_len, *release, *n_free;
  int32_t *kv_len_out, *table, *free_pages, *n_free_out, *pos, *refused;
  int64_t table_stride;
  int64_t *slot;
  int32_t *start;    // [n_seqs]: place of a sequence's first new token, -1: refused. NULL: the
                     // first kernel gives the tokens their rows
  int32_t n_seqs, n_tokens, n_pages, page_size;
  int32_t most;      // rows that a sequence may hold
};

__device__ __forceinline__ int clamp(int v, int lo, int hi) { return min(max(v, lo), hi); }

__device__ __forceinline__ int pages_of(const PagesParams &P, int rows) {
  return static_cast<int>((static_cast<uint32_t>(rows) + P.page_size - 1) / P.page_size);
}

// The cache row at `place` of a sequence whose page there is `page`.
__device__ __forceinline__ int64_t row_of(const PagesParams &P, int page, int place) {
  if (page < 0 || page >= P.n_pages) return -1;
  return int64_t(page) * P.page_size + static_cast<uint32_t>(place) % P.page_size;
}

__device__ __forceinline__ void put(const PagesParams &P, int t, int64_t slot, int place) {
  P.slot[t] = slot;
  if (P.pos) P.pos[t] = slot < 0 ? 0 : place;
}

// Sum of `v` over the workgroup's threads up to and with this one; `total` over all. 64 bits:
// q_begin may be anything, and the sums decide what is read.
__device__ __forceinline__ int64_t sum_up(int64_t v, int64_t (&waves)[kWaves], int64_t &total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t u = __shfl_up(v, o);
    if (lane >= o) v += u;
  }
  __syncthreads();  // what was read from `waves` before
  if (lane == 63) waves[wave] = v;
  __syncthreads();
  total = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) v += waves[w];
    total += waves[w];
  }
  return v;
}

__global__ __launch_bounds__(kThreads) void pages_kernel(const PagesParams P) {
  __shared__ int64_t s_waves[kWaves];
  __shared__ int s_taken, s_refused;
  const int tid = threadIdx.x, lane = tid & 63;
  if (tid == 0) s_taken = s_refused = 0;
  int64_t top = clamp(*P.n_free, 0, P.n_pages);
  if (P.release) {
    for (int s0 = 0; s0 < P.n_seqs; s0 += kThreads) {
      const int s = s0 + tid;
      int back = 0;
      if (s < P.n_seqs && P.release[s] != 0) back = pages_of(P, clamp(P.kv_len[s], 0, P.most));
      int64_t total;
      const int64_t at = top + sum_up(back, s_waves, total) - back;
      for (uint64_t left = __ballot(back > 0); left; left &= left - 1) {
        const int l = __builtin_ctzll(left), n = __shfl(back, l);
        const int64_t to = __shfl(at, l);
        const int32_t *row = P.table + (s - lane + l) * P.table_stride;
        for (int i = lane; i < n && to + i < P.n_pages; i += 64) P.free_pages[to + i] = row[i];
      }
      top += total;
    }
    top = min(top, int64_t(P.n_pages));
  }
  __syncthreads();  // the stack is read from here on, and tables written
  int64_t asked = 0;
  for (int s0 = 0; s0 < P.n_seqs; s0 += kThreads) {
    const int s = s0 + tid;
    int first = 0, count = 0, start = 0, have = 0, need = 0, page = -1;
    bool room = true;
    if (s < P.n_seqs) {
      const bool ended = P.release && P.release[s] != 0;
      first = clamp(P.q_begin[s], 0, P.n_tokens);
      count = clamp(P.q_begin[s + 1], first, P.n_tokens) - first;
      start = ended ? 0 : clamp(P.kv_len[s], 0, P.most);
      have = pages_of(P, start);
      room = count <= P.most - start;
      need = room ? pages_of(P, start + count) - have : 0;
      // the page of the first token, where the sequence holds it already
      if (count > 0 && start < have * int64_t(P.page_size))
        page = P.table[s * P.table_stride + have - 1];
    }
    int64_t total;
    const int64_t upto = asked + sum_up(need, s_waves, total);
    const bool fits = room && (need == 0 || upto <= top);
    const int take = fits ? need : 0;
    int32_t *row = P.table + s * P.table_stride;
    int next = -1;  // the first page taken
    if (take > 0) {
      next = P.free_pages[top - 1 - (upto - need)];
      row[have] = next;
      atomicMax(&s_taken, static_cast<int>(upto));
    }
    for (uint64_t left = __ballot(take > 1); left; left &= left - 1) {
      const int l = __builtin_ctzll(left), n = __shfl(take, l);
      const int64_t from = top - 1 - (__shfl(upto, l) - n);
      int32_t *to = P.table + (s - lane + l) * P.table_stride + __shfl(have, l);
      for (int i = lane + 1; i < n; i += 64) to[i] = P.free_pages[from - i];
    }
    const uint64_t no = __ballot(!fits);
    if (lane == 0 && no) atomicAdd(&s_refused, __popcll(no));
    if (s < P.n_seqs) {
      P.kv_len_out[s] = fits ? start + count : start;
      if (P.start) P.start[s] = fits ? start : -1;
      else if (count == 1)
        put(P, first, fits ? row_of(P, take > 0 ? next : page, start) : -1, start);
    }
    if (!P.start) {
      for (uint64_t left = __ballot(count > 1); left; left &= left - 1) {
        const int l = __builtin_ctzll(left), n = __shfl(count, l), begin = __shfl(start, l);
        const int t = __shfl(first, l), old = __shfl(page, l), held = __shfl(have, l);
        const bool in = __shfl(static_cast<int>(fits), l) != 0;
        const int64_t from = top - 1 - (__shfl(upto, l) - __shfl(need, l));
        for (int i = lane; i < n; i += 64) {
          const int at = static_cast<int>(static_cast<uint32_t>(begin + i) / P.page_size);
          const int p = !in ? -1 : at < held ? old : P.free_pages[from - (at - held)];
          put(P, t + i, row_of(P, p, begin + i), begin + i);
        }
      }
    }
    asked += total;
  }
  if (!P.start) {  // tokens that belong to nobody
    const int lo = P.n_seqs > 0 ? clamp(P.q_begin[0], 0, P.n_tokens) : 0;
    const int hi = P.n_seqs > 0 ? clamp(P.q_begin[P.n_seqs], 0, P.n_tokens) : 0;
    for (int t = tid; t < lo; t += kThreads) put(P, t, -1, 0);
    for (int t = max(lo, hi) + tid; t < P.n_tokens; t += kThreads) put(P, t, -1, 0);
  }
  __syncthreads();
  if (tid == 0) {
    *P.n_free_out = static_cast<int>(top) - s_taken;
    *P.refused = s_refused;
  }
}

constexpr int kSlotThreads = 256, kEach = 4;  // tokens of a thread
constexpr int kListed = 4096;                 // entries of q_begin kept in LDS

__global__ __launch_bounds__(kSlotThreads) void slots_kernel(const PagesParams P) {
  __shared__ int s_begin[kListed];
  const bool listed = P.n_seqs < kListed;
  if (listed) {
    for (int i = threadIdx.x; i <= P.n_seqs; i += kSlotThreads) s_begin[i] = P.q_begin[i];
    __syncthreads();
  }
  const int64_t t0 = (int64_t(workgroup()) * kSlotThreads + threadIdx.x) * kEach;
  const auto begin = [&](int s) { return listed ? s_begin[s] : P.q_begin[s]; };
  int s = -1;  // the last sequence that begins at or before the token
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    if (t0 + i >= P.n_tokens) return;
    const int t = static_cast<int>(t0) + i;
    if (i == 0) {
      int lo = -1, hi = P.n_seqs;  // begin(lo) <= t < begin(hi)
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (begin(mid) <= t) lo = mid;
        else hi = mid;
      }
      s = lo;
    } else {
      while (s + 1 < P.n_seqs && begin(s + 1) <= t) ++s;
    }
    int64_t slot = -1;
    int place = 0;
    if (s >= 0 && t < begin(s + 1)) {
      const int start = P.start[s], past = t - clamp(begin(s), 0, P.n_tokens);
      if (start >= 0 && past >= 0 && past < P.most - start) {
        place = start + past;
        const int at = static_cast<int>(static_cast<uint32_t>(place) / P.page_size);
        slot = row_of(P, P.table[s * P.table_stride + at], place);
      }
    }
    put(P, t, slot, place);
  }
}

}  // namespace

extern "C" size_t tg_pages_workspace_bytes(int32_t n_seqs, int32_t n_tokens) {
  if (n_seqs <= 0 || n_seqs > TG_PAGES_MAX_SEQS || n_tokens <= kFewTokens) return 0;
  return (static_cast<size_t>(n_seqs) * sizeof(int32_t) + 15) / 16 * 16;
}

extern "C" int tg_pages(const tg_pages_args *a, void *stream) {
  if (!a || a->n_seqs < 0 || a->n_seqs > TG_PAGES_MAX_SEQS || a->n_tokens < 0 || a->n_pages < 0 ||
      a->page_size < 1 || a->max_pages < 1 || a->table_stride < a->max_pages ||
      int64_t(a->n_pages) * a->page_size > INT32_MAX)
    return TG_E_INVAL;
  if (a->n_seqs == 0 && a->n_tokens == 0) return TG_OK;
  if (a->n_seqs > 0 && (!a->q_begin || !a->kv_len || !a->kv_len_out || !a->table))
    return TG_E_INVAL;
  if ((a->n_pages > 0 && !a->free_pages) || (a->n_tokens > 0 && !a->slot) || !a->n_free ||
      !a->n_free_out || !a->refused)
    return TG_E_INVAL;
  const size_t need = tg_pages_workspace_bytes(a->n_seqs, a->n_tokens);
  if (need > 0 && (!a->workspace || a->workspace_bytes < need || !aligned16(a->workspace)))
    return TG_E_WORKSPACE;
  PagesParams P = {};
  P.q_begin = a->q_begin;
  P.kv_len = a->kv_len;
  P.release = a->release;
  P.n_free = a->n_free;
  P.kv_len_out = a->kv_len_out;
  P.table = a->table;
  P.free_pages = a->free_pages;
  P.n_free_out = a->n_free_out;
  P.pos = a->pos;
  P.refused = a->refused;
  P.table_stride = a->table_stride;
  P.slot = a->slot;
  P.start = need > 0 ? static_cast<int32_t *>(a->workspace) : nullptr;
  P.n_seqs = a->n_seqs;
  P.n_tokens = a->n_tokens;
  P.n_pages = a->n_pages;
  P.page_size = a->page_size;
  P.most = static_cast<int32_t>(
      std::min<int64_t>(int64_t(a->max_pages) * a->page_size, INT32_MAX));
  hipStream_t s = static_cast<hipStream_t>(stream);
  hipLaunchKernelGGL(pages_kernel, dim3(1), dim3(kThreads), 0, s, P);
  if (P.start) {
    const int64_t blocks = (int64_t(P.n_tokens) + kSlotThreads * kEach - 1) / (kSlotThreads * kEach);
    hipLaunchKernelGGL(slots_kernel, grid_of(blocks, kSlotThreads), dim3(kSlotThreads), 0, s, P);
  }
  return hipGetLastError() == hipSuccess ? TG_OK : TG_E_HIP;
}
