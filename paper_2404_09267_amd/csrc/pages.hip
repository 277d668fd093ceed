// tg_pages: the pages of a cache given back and taken, page tables, and a cache row for every new
// token of a step, from lengths that stay on the device.
//
// What each sequence gets depends on what all before it have asked for, so one workgroup goes over
// the sequences, kThreads at a time, with a prefix sum of pages each: first of those that go back,
// which are pushed on the stack, then of those that are asked for, which come off its top. No
// sequence waits for another's write: a page that is taken is read from the stack by whoever needs
// it. Pages, and the tokens of prompts, are dealt out one a thread, so that a sequence of many is
// not one wave's (512 sequences, 51 that end and 77 with prompts of up to 4,096 tokens, pages of
// 64: 17.9 -> 14.1 us; four at a time are no faster). The rows of new tokens come with it where
// they are few; many are a second kernel's (the same: 11.9). There is next to nothing to read, so a
// chain of loads bounds it (lengths, stack, then the stores). Entries that are no page must not go
// back, or somebody else is given them: the pages that do are looked at on their way, and only
// where one is none is it all done again, by a sum over valid ones (the look alone: 11.9 -> 12.0, 28
// -> 30 where 164 of 512 sequences give back 48,000).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <cstdint>

#include "tg.h"
#include "token_math.h"

namespace {

using namespace tok;

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kMaxPages = 1 << 20;  // of a sequence, so that their sums hold in 32 bits
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

// Sum of `v` over the workgroup's threads up to and with this one; `total` over all. What is added
// are pages of a sequence, 2^20 at most each.
__device__ __forceinline__ int sum_up(int v, int (&waves)[kWaves], int &total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);  // the lanes 1, 2, 4 and 8 before
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);  // in a row of 16
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);  // the last of the row before
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);  // the last of the half before
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

// A sequence as the caller left it, clamped.
struct Seq {
  int first, count;  // its tokens
  int held;          // rows
  bool ended;
};

__device__ __forceinline__ Seq sequence(const PagesParams &P, int s) {
  Seq q = {0, 0, 0, false};
  if (s >= P.n_seqs) return q;
  const int begin = P.q_begin[s], end = P.q_begin[s + 1], held = P.kv_len[s];
  q.ended = P.release && P.release[s] != 0;
  q.first = clamp(begin, 0, P.n_tokens);
  q.count = clamp(end, q.first, P.n_tokens) - q.first;
  q.held = clamp(held, 0, P.most);
  return q;
}

// What is dealt out: the sequences of the turn that have any, one after the other, and where their
// items end; INT_MAX behind the last.
struct Dealt {
  int ends[kThreads], who[kThreads];
};

// Lists them (`mine` items of this thread's, which end at `upto`); the caller has set all ends to
// INT_MAX and waits.
__device__ __forceinline__ void list(Dealt &d, int mine, int upto, int (&waves)[kWaves]) {
  int all;
  const int at = sum_up(mine > 0, waves, all) - 1;
  if (mine <= 0) return;
  d.ends[at] = upto;
  d.who[at] = threadIdx.x;
}

// Which of them has item `i`. A wave's items follow each other, so that few sequences have them:
// that of its first is looked for by all lanes, and each lane goes on from there.
__device__ __forceinline__ int owner_of(const Dealt &d, int i) {
  constexpr int kEach = kThreads / 64;
  const int lane = threadIdx.x & 63, least = __builtin_amdgcn_readfirstlane(i);
  const int group = __builtin_ctzll(__ballot(d.ends[lane * kEach + kEach - 1] > least));
  int o = group * kEach +
          __builtin_ctzll(__ballot(d.ends[group * kEach + (lane & (kEach - 1))] > least));
  while (d.ends[o] <= i) ++o;
  return o;
}

// Pushes the pages of all sequences that have ended on the stack, whose `top` it moves; `q`: this
// thread's sequence of the first turn. True in some threads if an entry is no page. kSift: those
// are left out, which takes a prefix sum for every kThreads entries.
template <bool kSift>
__device__ __forceinline__ bool give_back(const PagesParams &P, Seq q, int64_t &top, Dealt &dealt,
                                          int (&waves)[kWaves]) {
  const int tid = threadIdx.x, lane = tid & 63;
  uint32_t most = 0;  // of the entries; as such, negative ones are large
  for (int s0 = 0; s0 < P.n_seqs; s0 += kThreads) {
    if (s0 > 0) q = sequence(P, s0 + tid);
    int total;
    const int back = q.ended ? pages_of(P, q.held) : 0;
    const int upto = sum_up(back, waves, total);
    dealt.ends[tid] = INT_MAX;
    list(dealt, back, upto, waves);
    __syncthreads();
    const auto entry = [&](int i) {
      const int o = owner_of(dealt, i), at = i - (o > 0 ? dealt.ends[o - 1] : 0);
      return P.table[static_cast<uint32_t>(s0 + dealt.who[o]) * P.table_stride + at];
    };
    if constexpr (kSift) {
      for (int i0 = 0; i0 < total && top < P.n_pages; i0 += kThreads) {
        const int page = entry(min(i0 + tid, total - 1));
        const bool one = i0 + tid < total && page >= 0 && page < P.n_pages;
        int all;
        const int64_t to = top + sum_up(one, waves, all) - 1;
        if (one && to < P.n_pages) P.free_pages[to] = page;
        top += all;
      }
    } else {
      const int n = static_cast<int>(min(int64_t(total), P.n_pages - min(top, int64_t(P.n_pages))));
      for (int i0 = tid - lane; i0 < n; i0 += kThreads) {
        const int i = min(i0 + lane, n - 1), page = entry(i);
        if (i0 + lane < n) P.free_pages[top + i] = page;
        most = max(most, static_cast<uint32_t>(page));
      }
      top += total;
    }
  }
  top = min(top, int64_t(P.n_pages));
  return most > 0 && most >= static_cast<uint32_t>(P.n_pages);
}

__global__ __launch_bounds__(kThreads) void pages_kernel(const PagesParams P) {
  __shared__ int s_waves[kWaves];
  __shared__ Dealt s_dealt;
  __shared__ int s_upto[kThreads], s_first[kThreads], s_start[kThreads], s_have[kThreads],
      s_page[kThreads];
  __shared__ int s_taken, s_refused, s_most, s_none;
  const int tid = threadIdx.x, lane = tid & 63;
  if (tid == 0) s_taken = s_refused = s_none = 0;  // s_none: entries that are no page go back
  int64_t top = clamp(*P.n_free, 0, P.n_pages);
  Seq q = sequence(P, tid);  // the first turn's, which is all of them most of the time
  if (P.release) {
    const int64_t before = top;
    if (give_back<false>(P, q, top, s_dealt, s_waves)) s_none = 1;
    __syncthreads();
    if (s_none) {
      top = before;
      give_back<true>(P, sequence(P, tid), top, s_dealt, s_waves);
    }
    if (P.n_seqs > kThreads) q = sequence(P, tid);
  }
  __syncthreads();  // the stack is read from here on, and tables written
  int64_t asked = 0;
  for (int s0 = 0; s0 < P.n_seqs; s0 += kThreads) {
    const int s = s0 + tid;
    if (s0 > 0) q = sequence(P, s);
    const int first = q.first, count = q.count, start = q.ended ? 0 : q.held;
    const int have = pages_of(P, start);
    const bool room = count <= P.most - start;
    const int need = room ? pages_of(P, start + count) - have : 0;
    // the page of the first token, where the sequence holds it already
    int page = -1;
    if (count > 0 && start < have * int64_t(P.page_size))
      page = P.table[s * P.table_stride + have - 1];
    if (tid == 0) s_most = 0;
    int total;
    const int upto = sum_up(need, s_waves, total);
    const bool fits = room && (need == 0 || asked + upto <= top);
    const int take = fits ? need : 0;
    int next = -1;  // the first page taken
    if (take > 0) {
      next = P.free_pages[top - 1 - (asked + upto - need)];
      P.table[s * P.table_stride + have] = next;
      atomicMax(&s_taken, static_cast<int>(asked + upto));
    }
    const uint64_t no = __ballot(!fits), many = __ballot(take > 1 || count > 1);
    if (lane == 0 && no) atomicAdd(&s_refused, __popcll(no));
    if (lane == 0 && many) s_most = 1;
    if (s < P.n_seqs) {
      P.kv_len_out[s] = fits ? start + count : start;
      if (P.start) P.start[s] = fits ? start : -1;
      else if (count == 1)
        put(P, first, fits ? row_of(P, take > 0 ? next : page, start) : -1, start);
    }
    __syncthreads();
    if (s_most) {  // more than a page or a token of one sequence: all of them over all threads
      s_dealt.ends[tid] = INT_MAX;
      list(s_dealt, need, upto, s_waves);
      s_upto[tid] = upto;
      s_start[tid] = fits ? start : -1;
      s_have[tid] = have;
      s_page[tid] = page;
      s_first[tid] = s < P.n_seqs ? first : P.n_tokens;
      __syncthreads();
      const int64_t under = top - 1 - asked;  // the first page on the stack for these sequences
      const int n = static_cast<int>(min(int64_t(total), max(top - asked, int64_t(0))));
      for (int64_t i0 = tid - lane; i0 < n; i0 += kThreads) {
        const int i = static_cast<int>(min(i0 + lane, int64_t(n - 1)));
        const int o = owner_of(s_dealt, i), at = i - (o > 0 ? s_dealt.ends[o - 1] : 0);
        const int who = s_dealt.who[o], taken = P.free_pages[under - i];
        if (i0 + lane < n && s_start[who] >= 0)
          P.table[(s0 + who) * P.table_stride + s_have[who] + at] = taken;
      }
      if (!P.start) {
        const int last = min(s0 + kThreads, P.n_seqs);
        const int end = clamp(P.q_begin[last], 0, P.n_tokens);
        for (int t = s_first[0] + tid; t < end; t += kThreads) {
          int lo = 0, hi = last - s0;  // the last sequence that begins at or before the token
          while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (s_first[mid] <= t) lo = mid;
            else hi = mid;
          }
          const int begin = s_start[lo], i = t - s_first[lo], place = begin + i;
          int64_t slot = -1;
          if (begin >= 0 && i >= 0 && i < P.most - begin) {
            const int at = static_cast<int>(static_cast<uint32_t>(place) / P.page_size);
            const int taken = at - s_have[lo];
            const int64_t from = under - (lo > 0 ? s_upto[lo - 1] : 0) - taken;
            if (taken < 0) slot = row_of(P, s_page[lo], place);
            else if (from >= 0 && from < P.n_pages) slot = row_of(P, P.free_pages[from], place);
          }
          put(P, t, slot, place);
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

// A token a thread, so that a wave's stores follow each other (four a thread: 14.1 us for 11.9 in
// the example above).
constexpr int kSlotThreads = 1024;
constexpr int kListed = 4096;  // entries of q_begin kept in LDS

__global__ __launch_bounds__(kSlotThreads) void slots_kernel(const PagesParams P) {
  __shared__ int s_begin[kListed];
  const bool listed = P.n_seqs < kListed;
  if (listed) {
    for (int i = threadIdx.x; i <= P.n_seqs; i += kSlotThreads) s_begin[i] = P.q_begin[i];
    __syncthreads();
  }
  const auto begin = [&](int s) { return listed ? s_begin[s] : P.q_begin[s]; };
  const int64_t token = int64_t(workgroup()) * kSlotThreads + threadIdx.x;
  if (token >= P.n_tokens) return;
  const int t = static_cast<int>(token);
  int lo = -1, hi = P.n_seqs;  // begin(lo) <= t < begin(hi)
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (begin(mid) <= t) lo = mid;
    else hi = mid;
  }
  int64_t slot = -1;
  int place = 0;
  if (lo >= 0 && t < begin(lo + 1)) {
    const int start = P.start[lo], past = t - clamp(begin(lo), 0, P.n_tokens);
    if (start >= 0 && past >= 0 && past < P.most - start) {
      place = start + past;
      const int at = static_cast<int>(static_cast<uint32_t>(place) / P.page_size);
      slot = row_of(P, P.table[lo * P.table_stride + at], place);
    }
  }
  put(P, t, slot, place);
}

}  // namespace

extern "C" size_t tg_pages_workspace_bytes(int32_t n_seqs, int32_t n_tokens) {
  if (n_seqs <= 0 || n_seqs > TG_PAGES_MAX_SEQS || n_tokens <= kFewTokens) return 0;
  return (static_cast<size_t>(n_seqs) * sizeof(int32_t) + 15) / 16 * 16;
}

extern "C" int tg_pages(const tg_pages_args *a, void *stream) {
  if (!a || a->n_seqs < 0 || a->n_seqs > TG_PAGES_MAX_SEQS || a->n_tokens < 0 || a->n_pages < 0 ||
      a->page_size < 1 || a->max_pages < 1 || a->max_pages > kMaxPages ||
      a->table_stride < a->max_pages ||
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
    const int64_t blocks = (int64_t(P.n_tokens) + kSlotThreads - 1) / kSlotThreads;
    hipLaunchKernelGGL(slots_kernel, grid_of(blocks, kSlotThreads), dim3(kSlotThreads), 0, s, P);
  }
  return hipGetLastError() == hipSuccess ? TG_OK : TG_E_HIP;
}
