// Which sequences of a batch hold the same pages in front (jd_cache_share): the plan of an attention that reads those once.
//
// Entries with the same number (the caller's, or else the same first page) follow the first of them as far as their pages are its pages; a
// group's prefix is what all its members follow, in whole tiles of context. One launch: a block for each entry finds its leader and compares the two
// page tables, and the last block done, a thread for each entry, puts the groups together in the entries' order, so that the same tables always
// give the same plan, and weighs whether the call would gain by them. A handful of dependent loads, once a step for all layers: 16 sequences that share 118 pages
// take 8 us, 32 that share 512 pages 10 us.
#include "jd_cache.h"

namespace jd {
namespace {

constexpr int kThreads = kMaxSharedBatch;         // the last block: one for each entry

// Inclusive sums over the block's threads; buf [kThreads / 32].
__device__ __forceinline__ unsigned long long scan(unsigned long long v, unsigned long long* buf) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned long long x = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += x;
  }
  if (lane == 31) buf[warp] = v;
  __syncthreads();
  for (int w = 0; w < warp; ++w) v += buf[w];
  __syncthreads();
  return v;
}

// What a call takes in ns: fixed, an SM for its share of the segments (a block of rows of a group or a sequence) and of their tiles of 128 tokens, and the
// call for every 1000 elements of its output; with groups, then without. Least squares over 1860 random calls of 2 to 96 sequences, prefixes of 100
// to 32768 tokens and 1 to 64 nodes, each in every form and without a plan (B200; half of the calls are met within 5 %, nine of ten within 15 %). Shared whenever
// they can be, such calls take 1.15 times as long as without a plan; by cost 1.04 times, for most have too little in common, and those that share 0.55 to 0.9 times.
struct FormCost { float fixed, segment, tile, out; };
__device__ __forceinline__ FormCost form_cost(bool shared, int rows, int D) {
  const bool wide = D > 64;
  const float d = (float)D;
  switch (shared ? rows : -rows) {
    case 32: return wide ? FormCost{17040, 4360, 1310, 7} : FormCost{15950, 4510, 760, 7};
    case 64: return wide ? FormCost{16470, 4350, 1620, 11} : FormCost{14920, 5360, 990, 10};
    case 128: return wide ? FormCost{19680, 6170, 1990, 10} : FormCost{17850, 6320, 1300, 15};
    case 256: return wide ? FormCost{22570, 7500, 2560, 14} : FormCost{19060, 7550, 2370, 20};
    case 4: return FormCost{12570, 1170 + 4 * d, 1590 + 23 * d, 0};
    case 16: return FormCost{17310, 960 + 22 * d, 2550 + 40 * d, 2};
    case -32: return wide ? FormCost{12120, 1120, 970, 18} : FormCost{11280, 730, 660, 22};
    case -64: return wide ? FormCost{14590, 0, 1220, 6} : FormCost{12630, 2020, 900, 4};
    case -128: return wide ? FormCost{14890, 0, 1540, 4} : FormCost{13740, 1070, 1110, 6};
    case -256: return wide ? FormCost{19590, 0, 2170, 3} : FormCost{17320, 0, 1930, 5};
    case -4: return FormCost{9140, 7 * d, 1210 + 25 * d, 33};
    default: return FormCost{13820, 7 * d, 1970 + 41 * d, 4};
  }
}
__device__ __forceinline__ float cost_of(const FormCost& x, float segments, float tiles, float sms, float outs) {
  return x.fixed + (x.segment * segments + x.tile * tiles) / sms + x.out * outs / 1000.f;
}

struct Entry {
  int slot, len, pages, key;                      // pages: full ones; key < 0: shares nothing
};
__device__ __forceinline__ Entry entry_at(const CacheView& c, const int32_t* slots, const int32_t* groups, int b) {
  Entry e;
  e.slot = slots ? __ldcg(slots + b) : b;
  e.len = e.pages = 0;
  e.key = -1;
  if (e.slot < 0 || e.slot >= c.max_seqs) { e.slot = -1; return e; }
  int len, held;
  slot_state(c, e.slot, len, held);
  e.len = len;
  e.pages = len >> c.page_shift;
  if (e.pages > 0) e.key = groups ? __ldcg(groups + b) : __ldcg(c.table + (int64_t)e.slot * c.max_pages);
  return e;
}

__global__ void __launch_bounds__(kThreads) share_kernel(CacheView c, SharedView s, int B, int nodes, int q_heads, Forms forms, bool always, int num_sms,
                                                         const int32_t* slots, const int32_t* groups) {
  __shared__ int s_lead, s_same, s_last, s_form;
  __shared__ int s_entries, s_all, s_own, s_blocks[2], s_tiles[2];   // what the call has to take; of the groups in either form
  __shared__ int of[kThreads], least[kThreads], members[kThreads], number[kThreads], start[kThreads];
  __shared__ unsigned long long buf[kThreads / 32];
  pdl_wait();
  pdl_trigger();
  const int b = blockIdx.x, t = threadIdx.x, rows = nodes * (q_heads / c.kv_heads);
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
    s.first[b] = e.len;                           // scratch until the call
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
  const int64_t units = whole ? (((int64_t)n * rows + 3) / 4) * ((tokens >> kSimtTileShift) + 8) : 0;
  const int64_t units_upto = (int64_t)scan((unsigned long long)units, buf);   // by every thread: it holds barriers
  whole = whole && units_upto <= kMostUnits;
  // What the call costs, an entry's own part and a leader's group from each thread.
  start[t] = whole ? tokens : 0;
  if (t == 0) s_entries = s_all = s_own = s_blocks[0] = s_blocks[1] = s_tiles[0] = s_tiles[1] = 0;
  __syncthreads();
  const int slot = t < B ? __ldcg(s.entry_slot + t) : -1;
  const int len = slot >= 0 ? __ldcg(s.first + t) + nodes : 0;
  constexpr int kMost = 1 << 21;                  // tiles that are counted: the sums are 32 bits, and beyond them everything is shared anyway
  auto tiles_of = [](int n) { return min((n + kPrefixTokens - 1) / kPrefixTokens, kMost); };
  const unsigned entries = __reduce_add_sync(0xffffffffu, (unsigned)(slot >= 0));
  const unsigned with = __reduce_add_sync(0xffffffffu, (unsigned)tiles_of(len));
  const unsigned without = __reduce_add_sync(0xffffffffu, (unsigned)tiles_of(len - (mine >= 0 ? start[mine] : 0)));
  if ((t & 31) == 0) {
    atomicAdd(&s_entries, (int)entries);
    atomicAdd(&s_all, (int)with);
    atomicAdd(&s_own, (int)without);
  }
  if (whole)
    for (int i = 0; i < 2; ++i) {
      const int form = i ? forms.second : forms.first, blocks = (n * rows + form - 1) / form;
      atomicAdd(&s_blocks[i], blocks);
      atomicAdd(&s_tiles[i], (int)min((int64_t)blocks * (tokens / kPrefixTokens), (int64_t)kMost));
    }
  __syncthreads();
  if (t == 0) {
    const float sms = (float)num_sms / c.kv_heads, outs = (float)B * nodes * q_heads * c.head_dim;
    const float alone_blocks = (float)((rows + forms.first - 1) / forms.first);
    float least_cost = 0.97f * cost_of(form_cost(false, forms.first, c.head_dim), alone_blocks * s_entries, alone_blocks * s_all, sms, outs);   // 3 % have to come of it
    if (always) least_cost = INFINITY;
    s_form = 0;
    for (int i = 0; i < 2; ++i) {
      const int form = i ? forms.second : forms.first;
      const float blocks = (float)((rows + form - 1) / form);
      const float v = cost_of(form_cost(true, form, c.head_dim), blocks * s_entries + s_blocks[i], blocks * s_own + s_tiles[i], sms, outs);
      if (v < least_cost) { least_cost = v; s_form = form; }
    }
    s_last = s_form != 0;                         // something is shared
  }
  __syncthreads();
  whole = whole && s_last;
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
    s.form[0] = s_form;                           // a call that takes the other kernel has the forms of that: the larger, if it shares
    s.form[1] = s_form >= 32 ? kSimtRows : s_form;
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

cudaError_t run_share(const CacheView& c, const SharedView& s, const jd_shared_t& plan, int q_heads, bool tensor, int num_sms, const int32_t* slots, const int32_t* groups,
                      cudaStream_t st) {
  const Forms forms = shared_forms(tensor, c.head_dim, plan.rows, plan.B, plan.nodes * (q_heads / c.kv_heads));
  return launch_chained(share_kernel, dim3((unsigned)plan.B), dim3(kThreads), 0, st, c, s, plan.B, plan.nodes, q_heads, forms, plan.rows != 0, num_sms, slots, groups);
}

}  // namespace jd
