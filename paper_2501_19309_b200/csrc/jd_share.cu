// Which sequences of a batch hold the same pages in front (jd_cache_share): the plan of an attention that reads those once.
//
// Entries with the same number (the caller's, or else the same first page) follow the first of them as far as their pages are its pages; a
// group's prefix is what all its members follow, in whole tiles of context. One launch: a block for each entry finds its leader and compares the two
// page tables, and the last block done, a thread for each entry, puts the groups together in the entries' order, so that the same tables always
// give the same plan. A handful of dependent loads, once a step for all layers: 32 sequences that share 512 pages take 6 us.
#include "jd_cache.h"

namespace jd {
namespace {

constexpr int kThreads = kMaxSharedBatch;         // the last block: one for each entry
constexpr int64_t kMostUnits = (int64_t)1 << 30;  // of all groups' prefix segments, whatever kernel takes them: their sums are 32 bits

// Inclusive sums over the block's threads.
__device__ __forceinline__ unsigned long long scan(unsigned long long v, unsigned long long* buf) {
  const int t = threadIdx.x;
  buf[t] = v;
  __syncthreads();
  for (int o = 1; o < kThreads; o <<= 1) {
    const unsigned long long x = t >= o ? buf[t - o] : 0;
    __syncthreads();
    buf[t] += x;
    __syncthreads();
  }
  v = buf[t];
  __syncthreads();
  return v;
}

struct Entry {
  int slot, pages, key;                           // pages: full ones; key < 0: shares nothing
};
__device__ __forceinline__ Entry entry_at(const CacheView& c, const int32_t* slots, const int32_t* groups, int b) {
  Entry e;
  e.slot = slots ? __ldcg(slots + b) : b;
  e.pages = 0;
  e.key = -1;
  if (e.slot < 0 || e.slot >= c.max_seqs) { e.slot = -1; return e; }
  int len, held;
  slot_state(c, e.slot, len, held);
  e.pages = len >> c.page_shift;
  if (e.pages > 0) e.key = groups ? __ldcg(groups + b) : __ldcg(c.table + (int64_t)e.slot * c.max_pages);
  return e;
}

__global__ void __launch_bounds__(kThreads) share_kernel(CacheView c, SharedView s, int B, int rows, const int32_t* slots, const int32_t* groups) {
  __shared__ int s_lead, s_same, s_last;
  __shared__ int of[kThreads], least[kThreads], members[kThreads], number[kThreads], start[kThreads];
  __shared__ unsigned long long buf[kThreads];
  pdl_wait();
  pdl_trigger();
  const int b = blockIdx.x, t = threadIdx.x;
  const Entry e = entry_at(c, slots, groups, b);
  if (t == 0) {
    slot_of(c, slots, b);                         // reports an entry that is out of range
    s_lead = b;
    s_same = e.pages;
  }
  __syncthreads();
  if (e.key >= 0)
    for (int i = t; i < b; i += kThreads)
      if (entry_at(c, slots, groups, i).key == e.key) atomicMin(&s_lead, i);
  __syncthreads();
  const int lead = s_lead;
  if (e.key >= 0 && lead != b) {
    const Entry l = entry_at(c, slots, groups, lead);
    const int32_t *mine = c.table + (int64_t)e.slot * c.max_pages, *its = c.table + (int64_t)l.slot * c.max_pages;
    if (t == 0) atomicMin(&s_same, l.pages);
    for (int i = t; i < min(e.pages, l.pages); i += kThreads)
      if (__ldcg(mine + i) != __ldcg(its + i)) { atomicMin(&s_same, i); break; }
  }
  __syncthreads();
  if (t == 0) {
    s.leader[b] = e.key >= 0 ? lead : -1;
    s.same[b] = s_same << c.page_shift;
    s.entry_slot[b] = e.slot;
    __threadfence();
    s_last = atomicAdd(s.count, 1) == (int)gridDim.x - 1;
  }
  __syncthreads();
  if (!s_last) return;
  __threadfence();
  // ---- the groups
  const int mine = t < B ? __ldcg(s.leader + t) : -1;
  of[t] = mine;
  least[t] = 0x7FFFFFFF;
  members[t] = 0;
  __syncthreads();
  if (mine >= 0) {
    atomicMin(&least[mine], __ldcg(s.same + t));
    atomicAdd(&members[mine], 1);
  }
  __syncthreads();
  const int n = members[t], tokens = mine == t ? least[t] & ~(kPrefixTokens - 1) : 0;
  bool whole = mine == t && n > 1 && (int64_t)(tokens / kPrefixTokens) * (n - 1) >= kPrefixWorth;
  const int64_t units = whole ? (((int64_t)n * rows + kSimtRows - 1) / kSimtRows) * ((tokens >> kSimtTileShift) + 8) : 0;
  const int64_t units_upto = (int64_t)scan((unsigned long long)units, buf);   // by every thread: it holds barriers
  whole = whole && units_upto <= kMostUnits;
  const unsigned long long upto = scan(whole ? ((unsigned long long)1 << 32) + n : 0, buf);
  number[t] = whole ? (int)(upto >> 32) - 1 : -1;
  start[t] = whole ? (int)(upto & 0xFFFFFFFFu) - n : 0;
  if (whole) {
    const int g = number[t];
    s.group_start[g] = start[t];
    s.group_start[g + 1] = start[t] + n;          // the next group's, if there is one, writes the same
    s.group_tokens[g] = tokens;
    s.group_slot[g] = __ldcg(s.entry_slot + t);
  }
  if (t == kThreads - 1) {
    *s.count = 0;
    s_last = (int)(upto >> 32);                   // groups
  }
  __syncthreads();
  if (t >= s_last && t < B / 2) s.group_tokens[t] = 0;
  if (t < B) {
    const int g = mine >= 0 ? number[mine] : -1;
    int place = 0;
    if (g >= 0) {
      for (int i = mine; i < t; ++i) place += of[i] == mine;
      s.member[start[mine] + place] = t;
    }
    s.entry_group[t] = g;
    s.entry_place[t] = place;
    s.entry_lead[t] = g >= 0 ? __ldcg(s.entry_slot + mine) : -1;
    s.entry_tokens[t] = g >= 0 ? least[mine] & ~(kPrefixTokens - 1) : 0;
  }
}

}  // namespace

cudaError_t run_share(const CacheView& c, const SharedView& s, int B, int rows, const int32_t* slots, const int32_t* groups, cudaStream_t st) {
  return launch_chained(share_kernel, dim3((unsigned)B), dim3(kThreads), 0, st, c, s, B, rows, slots, groups);
}

}  // namespace jd
