// The paged cache: handle, argument checks, and the kernels that keep its pages.
//
// The tables are small and every call is a handful of dependent loads, so these kernels are bound by latency: one
// launch each (a compaction: three), no host round trip, no lists that grow. The pool's state is a count of
// owners per page and a bitmap of the free ones. Releasing a page is one atomic on its count and, for the last owner,
// one on its bit: the result does not depend on the order. Handing out pages is one block's scan of the bitmap, lowest
// pages first, so that the same calls always give the same page numbers.
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>

#include "jd_cache.h"
#include "jd_path.h"

using namespace jd;

namespace {

constexpr int kBookThreads = 1024;

__device__ __forceinline__ int pages_for(const CacheView& c, int64_t tokens) {
  return (int)((tokens + c.page_size - 1) >> c.page_shift);
}

// Whether an earlier entry of the call names the same slot; the whole block takes part.
__device__ __forceinline__ bool named_before(const int32_t* slots, int b, int slot, int* flag) {
  if (threadIdx.x == 0) *flag = 0;
  __syncthreads();
  if (slots)
    for (int i = threadIdx.x; i < b; i += blockDim.x)
      if (__ldcg(slots + i) == slot) *flag = 1;
  __syncthreads();
  return *flag != 0;
}

// Free pages of word w of the bitmap; bits behind the last page count for nothing, whatever they are.
__device__ __forceinline__ uint32_t free_word(const CacheView& c, int w) {
  const int left = c.pages - 32 * w;
  return c.free_bits[w] & (left >= 32 ? 0xFFFFFFFFu : (1u << left) - 1u);
}

// One owner less for a page; its last one frees it.
__device__ __forceinline__ void release_page(const CacheView& c, int page) {
  if (page < 0 || page >= c.pages) { set_status(c.status, JD_ERR_BAD_INDEX); return; }
  const int before = atomicSub(c.refs + page, 1);
  if (before == 1) atomicOr(c.free_bits + (page >> 5), 1u << (page & 31));
  else if (before <= 0) { atomicAdd(c.refs + page, 1); set_status(c.status, JD_ERR_BAD_INDEX); }
}

// Cuts a slot to new_len tokens in `keep` pages; by the whole block, which holds len and held already.
__device__ __forceinline__ void cut_slot(const CacheView& c, int slot, int held, int keep, int new_len) {
  int32_t* table = c.table + (int64_t)slot * c.max_pages;
  for (int i = keep + threadIdx.x; i < held; i += blockDim.x) {
    release_page(c, table[i]);
    table[i] = -1;
  }
  if (threadIdx.x == 0) {
    c.seq_len[slot] = new_len;
    c.held[slot] = min(held, keep);
  }
}

__global__ void __launch_bounds__(256) truncate_kernel(CacheView c, const int32_t* slots, const int32_t* length) {
  __shared__ int flag;
  pdl_wait();
  pdl_trigger();
  const int b = blockIdx.x, slot = slot_of(c, slots, b);
  if (slot < 0) return;
  if (named_before(slots, b, slot, &flag)) { if (threadIdx.x == 0) set_status(c.status, JD_ERR_BAD_INDEX); return; }
  int len, held;
  slot_state(c, slot, len, held);
  const int to = length ? __ldcg(length + b) : 0;
  if (to < 0 || to > len) { if (threadIdx.x == 0) set_status(c.status, JD_ERR_BAD_INDEX); return; }
  __syncthreads();   // everybody has read the slot's state
  cut_slot(c, slot, held, pages_for(c, to), to);
}

__global__ void __launch_bounds__(256) fork_kernel(CacheView c, int n, const int32_t* src, const int32_t* dst) {
  __shared__ int flag;
  pdl_wait();
  pdl_trigger();
  const int i = blockIdx.x;
  const int s = __ldcg(src + i), d = __ldcg(dst + i);
  if (s == -1 || d == -1) return;
  if (threadIdx.x == 0) flag = s < 0 || s >= c.max_seqs || d < 0 || d >= c.max_seqs;
  __syncthreads();
  if (!flag)
    for (int j = threadIdx.x; j < n; j += blockDim.x) {
      const int sj = __ldcg(src + j), dj = __ldcg(dst + j);
      if (sj != -1 && dj != -1 && (sj == d || (j < i && dj == d))) flag = 1;   // padding entries name nothing
    }
  __syncthreads();
  if (!flag && threadIdx.x == 0 && (c.held[d] != 0 || c.seq_len[d] != 0)) flag = 1;
  __syncthreads();
  if (flag) { if (threadIdx.x == 0) set_status(c.status, JD_ERR_BAD_INDEX); return; }
  int len, held;
  slot_state(c, s, len, held);
  const int keep = pages_for(c, len);
  const int32_t* from = c.table + (int64_t)s * c.max_pages;
  int32_t* to = c.table + (int64_t)d * c.max_pages;
  for (int k = threadIdx.x; k < keep; k += blockDim.x) {
    const int page = from[k];
    to[k] = page;
    if (page >= 0 && page < c.pages) atomicAdd(c.refs + page, 1);
    else set_status(c.status, JD_ERR_BAD_INDEX);
  }
  if (threadIdx.x == 0) { c.seq_len[d] = len; c.held[d] = keep; }
}

// Exclusive prefix sum of one number per thread over a block of kBookThreads; total in *all.
__device__ __forceinline__ uint32_t block_exclusive(uint32_t v, uint32_t* warp_sums, uint32_t* all) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 31) warp_sums[warp] = x;
  __syncthreads();
  if (warp == 0) {
    uint32_t w = warp_sums[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t y = __shfl_up_sync(0xffffffffu, w, o);
      if (lane >= o) w += y;
    }
    warp_sums[lane] = w;
  }
  __syncthreads();
  *all = warp_sums[31];
  return x - v + (warp > 0 ? warp_sums[warp - 1] : 0);
}

// Copies n rows of page `from` to page `to` in one plane (layer, K or V, head); by kCopyThreads threads of which this is number t.
constexpr int kCopyThreads = 256;
__device__ __forceinline__ void copy_rows_of_page(const CacheView& c, int from, int to, int n, int plane, int t) {
  const int units = n * (c.row_bytes / 16), head = plane % c.kv_heads, lk = plane / c.kv_heads;
  char* base = (lk & 1) ? c.v : c.k;
  const uint4* s = reinterpret_cast<const uint4*>(base + page_row(c, lk >> 1, from, head, 0) * c.row_bytes);
  uint4* d = reinterpret_cast<uint4*>(base + page_row(c, lk >> 1, to, head, 0) * c.row_bytes);
  for (int u0 = t; u0 < units; u0 += 4 * kCopyThreads) {   // four loads in flight
    uint4 x[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (u0 + k * kCopyThreads < units) x[k] = s[u0 + k * kCopyThreads];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (u0 + k * kCopyThreads < units) d[u0 + k * kCopyThreads] = x[k];
  }
}

// Hands out pages and copies those that are about to be written and have other owners, in one launch without a block waiting for
// another: every block works out the whole plan from the state as it stands (thread b for sequence b, then all threads over
// the bitmap's words), copies its share of the rows, and counts itself done; the last one done writes the new state, which
// nobody reads any more. page_list[k] = the k-th page handed out; all blocks write the same.
__global__ void __launch_bounds__(kBookThreads) reserve_kernel(CacheView c, int B, const int32_t* slots, int n, int* page_list, int* blocks_done) {
  __shared__ int s_slot[kMaxCacheBatch], s_last[kMaxCacheBatch], s_off[kMaxCacheBatch], s_first[kMaxCacheBatch];
  __shared__ int s_rows[kMaxCacheBatch];   // rows to copy, 0: none
  __shared__ uint32_t warp_sums[32];
  __shared__ int fail, last_one;
  pdl_wait();
  pdl_trigger();
  const int b = threadIdx.x;
  if (b == 0) fail = 0;
  s_slot[b] = b < B ? slot_of(c, slots, b) : -1;
  s_last[b] = -1;
  __syncthreads();
  int slot = s_slot[b], len = 0, held = 0, want = 0, last = 0, rows = 0;
  if (slot >= 0 && slots) {
    bool named = false;
#pragma unroll 8
    for (int j = 0; j < b; ++j) named |= s_slot[j] == slot;
    if (named) { set_status(c.status, JD_ERR_BAD_INDEX); slot = -1; }
  }
  if (slot >= 0) {
    slot_state(c, slot, len, held);
    const int64_t end = (int64_t)len + n;
    if (end > ((int64_t)c.max_pages << c.page_shift)) fail = 1;
    else want = max(pages_for(c, end), held);
    last = len >> c.page_shift;
    rows = len & (c.page_size - 1);
    if (rows > 0) {   // a page in use: len <= held pages, so it has a table entry
      const int page = c.table[(int64_t)slot * c.max_pages + last];
      if (page >= 0 && page < c.pages) s_last[b] = page;
      else { fail = 1; set_status(c.status, JD_ERR_BAD_INDEX); }
    }
  }
  __syncthreads();
  bool copy = false;
  if (slot >= 0 && s_last[b] >= 0) {
    int owners = c.refs[s_last[b]];
    if (owners > 1)
#pragma unroll 8
      for (int j = 0; j < b; ++j) owners -= s_last[j] == s_last[b];
    copy = owners > 1;
  }
  const int need = slot >= 0 ? (want - held) + (copy ? 1 : 0) : 0;
  uint32_t all_pages, available;   // 1024 sequences may ask for 2^21 + 1 pages each, which 32 bits hold and 31 do not
  const int off = block_exclusive(need, warp_sums, &all_pages);
  const int words = (c.pages + 31) >> 5, per = (words + kBookThreads - 1) / kBookThreads;
  const int w0 = min(b * per, words), w1 = min(w0 + per, words);
  int mine = 0;
  for (int w = w0; w < w1; ++w) mine += __popc(free_word(c, w));
  const int first = block_exclusive(mine, warp_sums, &available);
  const bool ok = !fail && all_pages <= available;   // else nothing changes
  const int total = ok ? (int)all_pages : 0;
  if (!ok && b == 0) set_status(c.status, JD_ERR_PAGES);
  if (ok) {
    int rank = first;
    for (int w = w0; w < w1 && rank < total; ++w)
      for (uint32_t bits = free_word(c, w); bits && rank < total; bits &= bits - 1) page_list[rank++] = 32 * w + __ffs(bits) - 1;
  }
  s_off[b] = off;
  s_first[b] = held - (copy ? 1 : 0);
  s_rows[b] = ok && copy ? rows : 0;
  if (__syncthreads_or(s_rows[b] > 0)) {
    const int planes = c.layers * 2 * c.kv_heads;
    constexpr int kGroups = kBookThreads / kCopyThreads;
    for (int j = 0; j < B; ++j)
      if (s_rows[j] > 0)
        for (int plane = blockIdx.x * kGroups + b / kCopyThreads; plane < planes; plane += gridDim.x * kGroups)
          copy_rows_of_page(c, s_last[j], page_list[s_off[j]], s_rows[j], plane, b % kCopyThreads);
  }
  __syncthreads();
  if (b == 0) {
    __threadfence();
    last_one = atomicAdd(blocks_done, 1) == (int)gridDim.x - 1;
    if (last_one) *blocks_done = 0;
  }
  __syncthreads();
  if (!last_one || !ok) return;
  int rank = first;
  for (int w = w0; w < w1 && rank < total; ++w) {
    uint32_t bits = free_word(c, w), taken = 0;
    for (; bits && rank < total; bits &= bits - 1, ++rank) {
      const int i = __ffs(bits) - 1;
      taken |= 1u << i;
      c.refs[32 * w + i] = 1;
    }
    if (taken) c.free_bits[w] &= ~taken;
  }
  if (s_rows[b] > 0) {
    c.table[(int64_t)slot * c.max_pages + last] = page_list[off];
    atomicSub(c.refs + s_last[b], 1);
  }
  if (slot >= 0 && want > held) c.held[slot] = want;
  // table entries of the new pages, dealt out over the block: page k is of the last sequence whose pages start at or before k
  for (int k = b; k < total; k += kBookThreads) {
    int lo = 0, hi = kMaxCacheBatch - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (s_off[mid] <= k) lo = mid; else hi = mid - 1;
    }
    if (k > s_off[lo] || s_rows[lo] == 0) c.table[(int64_t)s_slot[lo] * c.max_pages + s_first[lo] + (k - s_off[lo])] = page_list[k];
  }
}

// Moves pages of a compaction: blockIdx.y strides over the moves, blockIdx.x over (layer, K or V, head).
__global__ void __launch_bounds__(kCopyThreads) move_pages_kernel(CacheView c, const int* src, const int* dst, const int* count) {
  pdl_wait();
  pdl_trigger();
  for (int i = blockIdx.y; i < *count; i += gridDim.y)
    for (int plane = blockIdx.x; plane < c.layers * 2 * c.kv_heads; plane += gridDim.x)
      copy_rows_of_page(c, src[i], dst[i], c.page_size, plane, threadIdx.x);
}

// Commit: blocks (x, b) move 16-byte columns of sequence b's kept rows, every thread its own column through all rows in
// rising order: a row's target is never behind its source, so nothing is overwritten before it has been read. The last
// block of a sequence to finish (a counter that it sets back to zero) then advances the length and releases pages.
constexpr int kMoveThreads = 256;
constexpr int kMoveBatch = 8;
__global__ void __launch_bounds__(kMoveThreads) commit_kernel(CacheView c, const int32_t* slots, const int32_t* accept_len, int num_paths,
                                                              int path_len, const int32_t* paths, int max_nodes, int32_t* chosen,
                                                              int* commit_cnt) {
  __shared__ int64_t s_from[kMaxNodes], s_to[kMaxNodes];
  __shared__ int s_node[kMaxNodes];
  __shared__ int flag, s_cut, s_moves, s_last;
  pdl_wait();
  pdl_trigger();
  const int b = blockIdx.y, slot = slot_of(c, slots, b);
  if (slot < 0) return;
  if (named_before(slots, b, slot, &flag)) { if (threadIdx.x == 0) set_status(c.status, JD_ERR_BAD_INDEX); return; }
  int len, held;
  slot_state(c, slot, len, held);
  int pick = 0, a = __ldcg(accept_len + (int64_t)b * num_paths);
#pragma unroll 4
  for (int i = 1; i < num_paths; ++i) {
    const int x = __ldcg(accept_len + (int64_t)b * num_paths + i);
    if (x > a) { a = x; pick = i; }
  }
  a = min(max(a, 0), path_len);
  // check the path and find its rows
  const int32_t* table = c.table + (int64_t)slot * c.max_pages;
  const int limit = held << c.page_shift;          // tokens that the sequence holds
  // Rows of a page that has other owners are not the sequence's to take or to write (a reserve that found no pages leaves it
  // at that). Owners of such a page hold tokens in it, so no block of this call releases it: every block sees the same count.
  if (threadIdx.x == 0) { s_cut = a; s_moves = 0; }
  if (threadIdx.x < a) s_node[threadIdx.x] = paths ? __ldcg(paths + ((int64_t)b * num_paths + pick) * path_len + threadIdx.x) : (int)threadIdx.x + 1;
  __syncthreads();
  if (threadIdx.x < a) {
    const int i = threadIdx.x, node = s_node[i], before = i ? s_node[i - 1] : 0;
    int from, to;
    bool ok = path_entries(len, limit, i, node, before, max_nodes, c.page_shift, &from, &to);
    if (ok) {
      const int fp = table[from], tp = table[to];
      ok = fp >= 0 && fp < c.pages && tp >= 0 && tp < c.pages;
      if (ok) ok = (c.refs[fp] <= 1) & (c.refs[tp] <= 1);
      const int mask = c.page_size - 1;
      s_from[i] = (((int64_t)fp * c.kv_heads) << c.page_shift) + ((len + node) & mask);
      s_to[i] = (((int64_t)tp * c.kv_heads) << c.page_shift) + ((len + 1 + i) & mask);
      if (ok && node != i + 1) s_moves = 1;
    }
    if (!ok) atomicMin(&s_cut, i);
  }
  if (threadIdx.x == kMaxNodes) {                  // node 0, by a thread that has no node to check
    bool ok = len < limit;
    if (ok) {
      const int page = table[len >> c.page_shift];
      ok = page >= 0 && page < c.pages && c.refs[page] <= 1;
    }
    if (!ok) atomicMin(&s_cut, -1);
  }
  __syncthreads();
  const int kept = s_cut;
  if (threadIdx.x == 0 && blockIdx.x == 0 && kept < a) set_status(c.status, JD_ERR_BAD_INDEX);
  if (s_moves && kept > 0) {
    int skip = 0;
    while (skip < kept && s_node[skip] == skip + 1) ++skip;
    const int chunks = c.row_bytes / 16;
    const uint32_t columns = (uint32_t)c.layers * 2 * c.kv_heads * chunks;   // at most 4096 x 2 x 1024 x 64
    for (uint32_t u = blockIdx.x * kMoveThreads + threadIdx.x; u < columns; u += gridDim.x * kMoveThreads) {
      const uint32_t plane = u / chunks;
      const int chunk = (int)(u - plane * chunks), lk = (int)(plane / c.kv_heads), head = (int)plane - lk * c.kv_heads;
      char* base = ((lk & 1) ? c.v : c.k) + page_row(c, lk >> 1, 0, head, 0) * c.row_bytes + chunk * 16;
      for (int i0 = skip; i0 < kept; i0 += kMoveBatch) {
        uint4 x[kMoveBatch];
#pragma unroll
        for (int i = 0; i < kMoveBatch; ++i)
          if (i0 + i < kept) x[i] = *reinterpret_cast<const uint4*>(base + s_from[i0 + i] * c.row_bytes);
#pragma unroll
        for (int i = 0; i < kMoveBatch; ++i)
          if (i0 + i < kept) *reinterpret_cast<uint4*>(base + s_to[i0 + i] * c.row_bytes) = x[i];
      }
    }
  }
  // every block of the sequence has read its state by now; the last one changes it
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    s_last = gridDim.x == 1 || atomicAdd(commit_cnt + b, 1) == (int)gridDim.x - 1;
  }
  __syncthreads();
  if (!s_last) return;
  if (threadIdx.x == 0) {
    if (gridDim.x > 1) commit_cnt[b] = 0;
    if (chosen) chosen[b] = pick;
  }
  const int new_len = len + kept + 1;
  cut_slot(c, slot, held, pages_for(c, new_len), new_len);
}

// Compaction, step 1 (one block): the k-th page in use above the number of pages in use moves into the k-th free one below it.
// The owner counts and the bitmap follow; map[p] = new number of page p.
__global__ void __launch_bounds__(kBookThreads) compact_plan_kernel(CacheView c, int* map, int* move_src, int* move_dst, int* move_cnt,
                                                                    int32_t* used_out) {
  __shared__ uint32_t warp_sums[32];
  pdl_wait();
  pdl_trigger();
  const int t = threadIdx.x, words = (c.pages + 31) >> 5, per = (words + kBookThreads - 1) / kBookThreads;
  const int w0 = min(t * per, words), w1 = min(w0 + per, words);
  auto used_bits = [&](int w) {
    const int left = c.pages - 32 * w;
    return ~c.free_bits[w] & (left >= 32 ? 0xFFFFFFFFu : (1u << left) - 1u);
  };
  uint32_t mine = 0, all_used, all_holes, all_movers;
  for (int w = w0; w < w1; ++w) mine += __popc(used_bits(w));
  block_exclusive(mine, warp_sums, &all_used);
  const int used = (int)all_used;
  int holes = 0, movers = 0;
  for (int w = w0; w < w1; ++w) {
    const uint32_t u = used_bits(w);
    const int below = min(max(used - 32 * w, 0), 32);          // pages of this word with numbers < used
    const uint32_t low = below >= 32 ? 0xFFFFFFFFu : (1u << below) - 1u;
    holes += below - __popc(u & low);
    movers += __popc(u & ~low);
  }
  int hole = block_exclusive(holes, warp_sums, &all_holes), mover = block_exclusive(movers, warp_sums, &all_movers);
  for (int w = w0; w < w1; ++w) {
    const uint32_t u = used_bits(w);
    for (int i = 0; i < 32 && 32 * w + i < c.pages; ++i) {
      const int p = 32 * w + i;
      const bool in_use = (u >> i) & 1u;
      map[p] = p;
      if (p < used && !in_use) move_dst[hole++] = p;
      if (p >= used && in_use) move_src[mover++] = p;
    }
  }
  __syncthreads();
  for (int k = t; k < (int)all_movers; k += kBookThreads) {
    const int s = move_src[k], d = move_dst[k];
    map[s] = d;
    c.refs[d] = c.refs[s];
    c.refs[s] = 0;
  }
  for (int w = w0; w < w1; ++w) {
    const int below = min(max(used - 32 * w, 0), 32), left = min(c.pages - 32 * w, 32);
    const uint32_t low = below >= 32 ? 0xFFFFFFFFu : (1u << below) - 1u, real = left >= 32 ? 0xFFFFFFFFu : (1u << left) - 1u;
    c.free_bits[w] = real & ~low;
  }
  if (t == 0) {
    *move_cnt = all_movers;
    if (used_out) *used_out = used;
  }
}

// Step 2: the tables' page numbers. Runs behind the plan and beside or behind the copies.
__global__ void __launch_bounds__(256) remap_kernel(CacheView c, const int* map) {
  pdl_wait();
  pdl_trigger();
  const int slot = blockIdx.x;
  int len, held;
  slot_state(c, slot, len, held);
  int32_t* table = c.table + (int64_t)slot * c.max_pages;
  for (int i = threadIdx.x; i < held; i += 256) {
    const int p = table[i];
    if (p >= 0 && p < c.pages) table[i] = map[p];
  }
}

// ------------------------------------------------------------------------------------------ host side

bool cache_config_ok(const jd_cache_config_t* g) {
  if (!g) return false;
  if (g->num_layers < 1 || g->num_pages < 1 || g->max_seqs < 1 || g->max_pages < 1 || g->kv_heads < 1 || g->q_heads < 1) return false;
  if (g->page_size < 8 || g->page_size > 1024 || (g->page_size & (g->page_size - 1))) return false;
  if (g->head_dim < 8 || g->head_dim > 256 || g->head_dim % 8) return false;
  if (g->q_heads % g->kv_heads || g->q_heads > 1024) return false;
  if (g->max_nodes < 1 || g->max_nodes > kMaxNodes) return false;
  if (g->dtype != JD_DTYPE_F32 && g->dtype != JD_DTYPE_BF16) return false;
  if ((int64_t)g->max_pages * g->page_size > (1 << 24)) return false;
  if (g->num_pages > (1 << 24) || g->num_layers > 4096 || g->max_seqs > (1 << 20)) return false;
  // rows of the K matrix are coordinates of its tensor map
  if ((int64_t)g->num_layers * g->num_pages * g->kv_heads > (int64_t)0x7FFFFFFF / g->page_size) return false;
  return true;
}

bool on_tensor_cores(const jd_cache_config_t& g) { return g.dtype == JD_DTYPE_BF16 && (g.head_dim == 64 || g.head_dim == 128); }
int rows_of(const jd_cache_config_t& g) { return g.max_nodes * (g.q_heads / g.kv_heads); }

size_t carve_cache(const jd_cache_config_t& g, char* base, jd_cache_s* c) {
  size_t off = 0;
  auto take = [&](size_t bytes) {
    char* p = base ? base + off : nullptr;
    off += (bytes + 255) / 256 * 256;
    return p;
  };
  unsigned* status = (unsigned*)take(256);
  int* cnt = (int*)take(kMaxCacheBatch * 4);
  int* rc = (int*)take(256);
  int* pl = (int*)take((size_t)g.num_pages * 4);
  int* ms = (int*)take((size_t)g.num_pages * 4);
  int* md = (int*)take((size_t)g.num_pages * 4);
  int* mc = (int*)take(256);
  int4* sp = (int4*)take((size_t)2 * kMaxCtas * sizeof(int4));
  // two partial results for each CTA of an attention call: up to 256 rows each on the tensor cores (one CTA per SM), where
  // they take the cache, kSimtRows on CUDA cores (two per SM)
  const size_t rows = std::max<size_t>(on_tensor_cores(g) ? std::min(rows_of(g), 256) : 0, 2 * kSimtRows);
  float* part = (float*)take((size_t)kMaxCtas * 2 * rows * (g.head_dim + kPartPad) * 4);
  if (c) {
    c->status = status; c->commit_cnt = cnt; c->reserve_cnt = rc;
    c->page_list = pl; c->move_src = ms; c->move_dst = md; c->move_cnt = mc; c->split = sp; c->part = part;
  }
  return off;
}

CacheView view_of(jd_cache_t c) {
  CacheView v;
  const jd_cache_config_t& g = c->cfg;
  v.layers = g.num_layers; v.pages = g.num_pages; v.page_size = g.page_size; v.page_shift = c->page_shift;
  v.kv_heads = g.kv_heads; v.head_dim = g.head_dim; v.max_seqs = g.max_seqs; v.max_pages = g.max_pages;
  v.row_bytes = g.head_dim * (g.dtype == JD_DTYPE_F32 ? 4 : 2);
  v.k = (char*)c->buf.k_pages; v.v = (char*)c->buf.v_pages;
  v.table = c->buf.page_table; v.seq_len = c->buf.seq_len; v.held = c->buf.held; v.refs = c->buf.refs;
  v.free_bits = c->buf.free_bits;
  v.status = c->status;
  return v;
}

bool on16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool on4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// The cache's device for the length of a call; the caller's comes back.
class OnDevice {
 public:
  explicit OnDevice(int device) {
    ok_ = cudaGetDevice(&before_) == cudaSuccess;
    if (ok_ && before_ != device) { ok_ = cudaSetDevice(device) == cudaSuccess; moved_ = ok_; }
  }
  ~OnDevice() { if (moved_) cudaSetDevice(before_); }
  bool ok() const { return ok_; }

 private:
  int before_ = 0;
  bool ok_ = false, moved_ = false;
};

bool batch_ok(jd_cache_t c, int B, const int32_t* slots) {
  return B >= 1 && B <= kMaxCacheBatch && (slots ? on4(slots) : B <= c->cfg.max_seqs);
}

// stride in elements: dense, or at least that and whole 16-byte units
bool stride_ok(int64_t stride, int64_t dense, int elem) {
  return stride == 0 || (stride >= dense && stride <= ((int64_t)1 << 40) && stride * elem % 16 == 0);
}

bool tree_ok(jd_cache_t c, const jd_tree_t& t) {
  return t.nodes >= 1 && t.nodes <= c->cfg.max_nodes && (t.per_seq == 0 || t.per_seq == 1) && on4(t.mask) && on4(t.depth) && on4(t.num_nodes);
}

bool append_ok(jd_cache_t c, const jd_append_args_t* a) {
  if (!c || !a || !batch_ok(c, a->B, a->slots) || !tree_ok(c, a->tree)) return false;
  const jd_cache_config_t& g = c->cfg;
  const int e = g.dtype == JD_DTYPE_F32 ? 4 : 2;
  if (a->layer < 0 || a->layer >= g.num_layers || !a->k || !a->v || !on16(a->k) || !on16(a->v)) return false;
  const int64_t kd = (int64_t)g.kv_heads * g.head_dim, qd = (int64_t)g.q_heads * g.head_dim;
  if (!stride_ok(a->k_stride, kd, e) || !stride_ok(a->v_stride, kd, e)) return false;
  if (a->q) {
    if (!a->q_out || !on16(a->q) || !on16(a->q_out) || !stride_ok(a->q_stride, qd, e) || !stride_ok(a->q_out_stride, qd, e)) return false;
    if (a->q == a->q_out && (a->q_stride ? a->q_stride : qd) != (a->q_out_stride ? a->q_out_stride : qd)) return false;
  }
  return !a->rope || rope_valid(*a->rope, g.head_dim);
}

bool attend_ok(jd_cache_t c, const jd_attend_args_t* a) {
  if (!c || !a || !batch_ok(c, a->B, a->slots) || !tree_ok(c, a->tree)) return false;
  const jd_cache_config_t& g = c->cfg;
  const int e = g.dtype == JD_DTYPE_F32 ? 4 : 2;
  if (a->layer < 0 || a->layer >= g.num_layers || !a->q || !a->out || a->q == a->out || !on16(a->q) || !on16(a->out) || !on4(a->lse)) return false;
  const int64_t qd = (int64_t)g.q_heads * g.head_dim;
  if (!stride_ok(a->q_stride, qd, e) || !stride_ok(a->out_stride, qd, e) || !(a->scale > 0.f && std::isfinite(a->scale))) return false;
  return a->variant >= JD_ATTEND_AUTO && a->variant <= JD_ATTEND_TENSOR;
}

AttendParams attend_params(jd_cache_t c, const jd_attend_args_t& a, bool tensor) {
  const jd_cache_config_t& g = c->cfg;
  const int e = g.dtype == JD_DTYPE_F32 ? 4 : 2;
  const int64_t qd = (int64_t)g.q_heads * g.head_dim;
  AttendParams p = {};
  p.c = view_of(c);
  p.B = a.B; p.layer = a.layer; p.T = a.tree.nodes; p.W = (a.tree.nodes + 31) / 32;
  p.q_heads = g.q_heads; p.group = g.q_heads / g.kv_heads;
  p.rows = p.T * p.group;
  p.slots = a.slots;
  p.mask = a.tree.mask;
  p.mask_stride = a.tree.per_seq ? (int64_t)p.T * p.W : 0;
  p.num_nodes = a.tree.num_nodes;
  p.q = (const char*)a.q; p.out = (char*)a.out;
  p.q_stride = (a.q_stride ? a.q_stride : qd) * e; p.out_stride = (a.out_stride ? a.out_stride : qd) * e;
  p.lse = a.lse;
  p.scale_log2 = a.scale * 1.4426950408889634f;
  p.part = c->part;
  p.split = c->split;
  if (tensor) {
    p.tile_shift = kTensorTileShift;
    p.seg_cost = tensor_seg_cost(g.head_dim, p.rows);
    p.rows_per_block = p.rows > 128 ? 256 : 128;
  } else {
    p.tile_shift = kSimtTileShift;
    p.seg_cost = kSimtSegCost;
    p.rows_per_block = p.rows <= 4 ? 4 : kSimtRows;   // one token's few rows leave the others' registers and products out
  }
  p.part_rows = std::min(p.rows, p.rows_per_block);
  p.row_blocks = (p.rows + p.rows_per_block - 1) / p.rows_per_block;
  p.groups = std::max(1, (tensor ? c->num_sms : 2 * c->num_sms) / p.row_blocks);
  return p;
}

// The parts of a plan's buffer; its size.
size_t carve_shared(jd_cache_t c, int B, int nodes, char* base, SharedView* s) {
  size_t off = 0;
  auto take = [&](size_t bytes) {
    char* p = base ? base + off : nullptr;
    off += (bytes + 255) / 256 * 256;
    return p;
  };
  const jd_cache_config_t& g = c->cfg;
  SharedView v;
  v.count = (int32_t*)take(256);
  for (int32_t** x : {&v.leader, &v.same, &v.group_start, &v.group_tokens, &v.group_slot, &v.member, &v.entry_group, &v.entry_place, &v.entry_slot,
                      &v.entry_lead, &v.entry_tokens, &v.first})
    *x = (int32_t*)take((size_t)(B + 1) * 4);
  v.units = (int32_t*)take((size_t)(B / 2 + B + 1) * 4);
  v.form = (int32_t*)take(8);
  const size_t row = (size_t)(g.head_dim + kPartPad) * 4, rows = (size_t)B * nodes * (g.q_heads / g.kv_heads);
  v.rec_group = (float*)take(rows * g.kv_heads * row);
  v.rec_own = (float*)take(rows * g.kv_heads * row);
  // two parts for each CTA, as in carve_cache
  const size_t most = std::max<size_t>(c->tm_ok ? std::min<size_t>(rows, 256) : 0, 2 * std::min<size_t>(rows, kSimtRows));
  v.part = (float*)take((size_t)c->num_sms * 2 * most * row);
  if (s) *s = v;
  return off;
}
bool form_ok(int rows) {
  for (int m = 0; m < kSharedForms; ++m)
    if (rows == form_rows(m)) return true;
  return false;
}
bool shared_ok(jd_cache_t c, const jd_shared_t* plan, SharedView* s) {
  if (!c || !plan || plan->B < 1 || plan->B > kMaxSharedBatch || plan->nodes < 1 || plan->nodes > c->cfg.max_nodes) return false;
  if (!plan->buffer || (reinterpret_cast<uintptr_t>(plan->buffer) & 255u) || plan->bytes < carve_shared(c, plan->B, plan->nodes, nullptr, nullptr)) return false;
  if (plan->rows != 0 && !form_ok(plan->rows)) return false;
  carve_shared(c, plan->B, plan->nodes, (char*)plan->buffer, s);
  return true;
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// [rows, head_dim] bf16, box 64 columns (128 bytes, 128-byte swizzle) x box_rows; rows out of range read as zero
bool encode_rows(CUtensorMap* tm, void* base, uint64_t rows, uint64_t d, uint32_t box_rows) {
  void* p = nullptr;
  cudaDriverEntryPointQueryResult q;
  if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess)
    return false;
  const cuuint64_t dims[2] = {d, rows};
  const cuuint64_t strides[1] = {d * 2};
  const cuuint32_t box[2] = {64, box_rows}, estr[2] = {1, 1};
  return ((EncodeTiledFn)p)(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, base, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

jd_status_t finish(jd_cache_t c, cudaError_t err, cudaStream_t st) {
  if (err != cudaSuccess) { cudaGetLastError(); return JD_ERR_CUDA; }
  c->last_stream = st;
  return JD_OK;
}

}  // namespace

extern "C" {

size_t jd_cache_workspace_bytes(const jd_cache_config_t* cfg) {
  return cache_config_ok(cfg) ? carve_cache(*cfg, nullptr, nullptr) : 0;
}

jd_status_t jd_cache_create(jd_cache_t* out, const jd_cache_config_t* cfg, const jd_cache_buffers_t* b) {
  if (!out || !cache_config_ok(cfg) || !b) return JD_ERR_INVALID_ARG;
  if (!b->k_pages || !b->v_pages || !b->page_table || !b->seq_len || !b->held || !b->refs || !b->free_bits || !b->workspace)
    return JD_ERR_INVALID_ARG;
  if (!on16(b->k_pages) || !on16(b->v_pages) || !on4(b->page_table) || !on4(b->seq_len) || !on4(b->held) || !on4(b->refs) ||
      !on4(b->free_bits) || (reinterpret_cast<uintptr_t>(b->workspace) & 255u))
    return JD_ERR_INVALID_ARG;
  if (b->workspace_bytes < carve_cache(*cfg, nullptr, nullptr)) return JD_ERR_INVALID_ARG;
  int ndev = 0, major = 0, sms = 0;
  if (cudaGetDeviceCount(&ndev) != cudaSuccess || cfg->device < 0 || cfg->device >= ndev) { cudaGetLastError(); return JD_ERR_CUDA; }
  if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, cfg->device) != cudaSuccess ||
      cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, cfg->device) != cudaSuccess)
    return JD_ERR_CUDA;
  if (major != 10) return JD_ERR_ARCH;
  OnDevice dev(cfg->device);
  if (!dev.ok() || !attend_configure()) { cudaGetLastError(); return JD_ERR_CUDA; }
  jd_cache_s* c = new (std::nothrow) jd_cache_s();
  if (!c) return JD_ERR_ALLOC;
  c->cfg = *cfg;
  c->buf = *b;
  c->num_sms = std::min(sms, kMaxCtas);
  c->page_shift = 0;
  while ((1 << c->page_shift) < cfg->page_size) ++c->page_shift;
  c->last_stream = nullptr;
  carve_cache(*cfg, (char*)b->workspace, c);
  c->tm_ok = false;
  if (on_tensor_cores(*cfg)) {
    const uint64_t rows = (uint64_t)cfg->num_layers * cfg->num_pages * cfg->kv_heads * cfg->page_size;
    const uint32_t box = (uint32_t)std::min(cfg->page_size, 1 << kTensorTileShift);
    c->tm_ok = encode_rows(&c->tm_k, b->k_pages, rows, (uint64_t)cfg->head_dim, box) &&
               encode_rows(&c->tm_v, b->v_pages, rows, (uint64_t)cfg->head_dim, box);
  }
  *out = c;
  return JD_OK;
}

jd_status_t jd_cache_destroy(jd_cache_t c) {
  delete c;
  return JD_OK;
}

jd_status_t jd_cache_reserve(jd_cache_t c, int32_t B, const int32_t* slots, int32_t n, void* cuda_stream) {
  if (!c || !batch_ok(c, B, slots) || n < 1) return JD_ERR_INVALID_ARG;
  OnDevice dev(c->cfg.device);
  if (!dev.ok()) return JD_ERR_CUDA;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  const CacheView v = view_of(c);
  // One block is enough unless pages are copied, which the host does not know: a group of
  // 256 threads for each plane, up to what is resident at once.
  const int blocks = (v.layers * 2 * v.kv_heads + kBookThreads / kCopyThreads - 1) / (kBookThreads / kCopyThreads);
  return finish(c, launch_chained(reserve_kernel, dim3((unsigned)std::min(blocks, 2 * c->num_sms)), dim3(kBookThreads), 0, st, v, B, slots, n,
                                  c->page_list, c->reserve_cnt), st);
}

jd_status_t jd_cache_append(jd_cache_t c, const jd_append_args_t* a, void* cuda_stream) {
  if (!append_ok(c, a)) return JD_ERR_INVALID_ARG;
  OnDevice dev(c->cfg.device);
  if (!dev.ok()) return JD_ERR_CUDA;
  return finish(c, run_append(view_of(c), *a, c->cfg.q_heads, c->cfg.dtype, (cudaStream_t)cuda_stream), (cudaStream_t)cuda_stream);
}

jd_status_t jd_cache_append_heads(jd_cache_t c, const jd_append_args_t* a, const jd_append_heads_t* x, void* cuda_stream) {
  if (!append_ok(c, a) || !x || !append_heads_valid(x->norm, x->axes, a->rope) || !on4(x->positions)) return JD_ERR_INVALID_ARG;
  OnDevice dev(c->cfg.device);
  if (!dev.ok()) return JD_ERR_CUDA;
  return finish(c, run_append_heads(view_of(c), *a, *x, c->cfg.q_heads, c->cfg.dtype, (cudaStream_t)cuda_stream), (cudaStream_t)cuda_stream);
}

jd_status_t jd_cache_attend(jd_cache_t c, const jd_attend_args_t* a, void* cuda_stream) {
  if (!attend_ok(c, a)) return JD_ERR_INVALID_ARG;
  if (a->variant == JD_ATTEND_TENSOR && !c->tm_ok) return JD_ERR_UNSUPPORTED;
  const bool tensor = a->variant != JD_ATTEND_SIMT && c->tm_ok;
  OnDevice dev(c->cfg.device);
  if (!dev.ok()) return JD_ERR_CUDA;
  const AttendParams p = attend_params(c, *a, tensor);
  cudaStream_t st = (cudaStream_t)cuda_stream;
  cudaError_t err = tensor ? run_attend_tensor(p, c->tm_k, c->tm_v, st) : run_attend_simt(p, c->cfg.dtype, st);
  // one group alone splits nothing
  if (err == cudaSuccess && p.groups > 1) err = run_attend_join(p, c->cfg.dtype, st);
  return finish(c, err, st);
}

size_t jd_cache_shared_bytes(jd_cache_t c, int32_t B, int32_t nodes) {
  return c && B >= 1 && B <= kMaxSharedBatch && nodes >= 1 && nodes <= c->cfg.max_nodes ? carve_shared(c, B, nodes, nullptr, nullptr) : 0;
}

jd_status_t jd_cache_share(jd_cache_t c, const jd_shared_t* plan, const int32_t* slots, const int32_t* groups, void* cuda_stream) {
  SharedView s;
  if (!shared_ok(c, plan, &s) || !batch_ok(c, plan->B, slots) || !on4(groups)) return JD_ERR_INVALID_ARG;
  if (plan->rows >= form_rows(0) && !c->tm_ok) return JD_ERR_UNSUPPORTED;
  OnDevice dev(c->cfg.device);
  if (!dev.ok()) return JD_ERR_CUDA;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  return finish(c, run_share(view_of(c), s, *plan, c->cfg.q_heads, c->tm_ok, c->num_sms, slots, groups, st), st);
}

jd_status_t jd_cache_attend_shared(jd_cache_t c, const jd_attend_args_t* a, const jd_shared_t* plan, void* cuda_stream) {
  SharedView s;
  if (!attend_ok(c, a) || !shared_ok(c, plan, &s) || plan->B != a->B || a->tree.nodes > plan->nodes) return JD_ERR_INVALID_ARG;
  if (a->B == 1) return jd_cache_attend(c, a, cuda_stream);   // nobody to share with
  if (a->variant == JD_ATTEND_TENSOR && !c->tm_ok) return JD_ERR_UNSUPPORTED;
  const bool tensor = a->variant != JD_ATTEND_SIMT && c->tm_ok;
  OnDevice dev(c->cfg.device);
  if (!dev.ok()) return JD_ERR_CUDA;
  AttendParams p = attend_params(c, *a, tensor);
  const Forms forms = shared_forms(tensor, c->cfg.head_dim, plan->rows, plan->B, plan->nodes * p.group);
  // the division's sums are 32 bits: the plan bounds the groups' part, and a batch whose own could pass the rest goes by itself
  const int64_t tiles = ((int64_t)c->cfg.max_pages * c->cfg.page_size >> p.tile_shift) + 8;
  if (a->B * ((p.rows + forms.first - 1) / forms.first) * tiles > kMostUnits) return jd_cache_attend(c, a, cuda_stream);
  p.sh = s;
  p.max_groups = a->B / 2;
  p.rows_per_block = forms.first;
  p.second_rows = forms.second;
  p.part_rows = std::min(a->B * p.rows, p.rows_per_block);
  if (tensor) p.seg_cost = tensor_seg_cost(c->cfg.head_dim, p.rows_per_block);
  p.row_blocks = 1;
  p.groups = tensor ? c->num_sms : 2 * c->num_sms;
  p.part = s.part;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  cudaError_t err = tensor ? run_attend_shared_tensor(p, c->tm_k, c->tm_v, st) : run_attend_shared_simt(p, c->cfg.dtype, st);
  if (err == cudaSuccess) err = run_attend_shared_join(p, c->cfg.dtype, st);
  return finish(c, err, st);
}

jd_status_t jd_cache_commit(jd_cache_t c, const jd_commit_args_t* a, void* cuda_stream) {
  if (!c || !a || !batch_ok(c, a->B, a->slots)) return JD_ERR_INVALID_ARG;
  if (!a->accept_len || !on4(a->accept_len) || a->num_paths < 1 || a->num_paths > 65536 || a->path_len < 0 || a->path_len >= c->cfg.max_nodes ||
      !on4(a->paths) || !on4(a->chosen))
    return JD_ERR_INVALID_ARG;
  OnDevice dev(c->cfg.device);
  if (!dev.ok()) return JD_ERR_CUDA;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  const CacheView v = view_of(c);
  const int64_t columns = (int64_t)v.layers * 2 * v.kv_heads * (v.row_bytes / 16);
  int blocks = a->paths && a->path_len > 0 ? (int)std::min<int64_t>((columns + kMoveThreads - 1) / kMoveThreads, 65535) : 1;
  // Finding a sequence's rows takes a block longer than a turn of moving them: three blocks on an SM in all, in even turns. 64 trees of 26
  // nodes in 32 layers of 8 heads of 128, with the truncation and the reserve in front of it: 45 us, a block for each turn 51.
  const int most = std::max(1, 3 * c->num_sms / a->B);
  if (blocks > most) {
    const int turns = (blocks + most - 1) / most;
    blocks = (blocks + turns - 1) / turns;
  }
  return finish(c, launch_chained(commit_kernel, dim3((unsigned)blocks, (unsigned)a->B), dim3(kMoveThreads), 0, st, v, a->slots, a->accept_len,
                                  a->num_paths, a->path_len, a->paths, c->cfg.max_nodes, a->chosen, c->commit_cnt), st);
}

jd_status_t jd_cache_fork(jd_cache_t c, int32_t n, const int32_t* src, const int32_t* dst, void* cuda_stream) {
  if (!c || n < 1 || n > kMaxCacheBatch || !src || !dst || !on4(src) || !on4(dst)) return JD_ERR_INVALID_ARG;
  OnDevice dev(c->cfg.device);
  if (!dev.ok()) return JD_ERR_CUDA;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  return finish(c, launch_chained(fork_kernel, dim3((unsigned)n), dim3(256), 0, st, view_of(c), n, src, dst), st);
}

jd_status_t jd_cache_truncate(jd_cache_t c, int32_t B, const int32_t* slots, const int32_t* length, void* cuda_stream) {
  if (!c || !batch_ok(c, B, slots) || !on4(length)) return JD_ERR_INVALID_ARG;
  OnDevice dev(c->cfg.device);
  if (!dev.ok()) return JD_ERR_CUDA;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  return finish(c, launch_chained(truncate_kernel, dim3((unsigned)B), dim3(256), 0, st, view_of(c), slots, length), st);
}

jd_status_t jd_cache_compact(jd_cache_t c, int32_t* used, void* cuda_stream) {
  if (!c || !on4(used)) return JD_ERR_INVALID_ARG;
  OnDevice dev(c->cfg.device);
  if (!dev.ok()) return JD_ERR_CUDA;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  const CacheView v = view_of(c);
  cudaError_t err = launch_chained(compact_plan_kernel, dim3(1), dim3(kBookThreads), 0, st, v, c->page_list, c->move_src, c->move_dst, c->move_cnt, used);
  if (err == cudaSuccess) err = launch_chained(remap_kernel, dim3((unsigned)v.max_seqs), dim3(256), 0, st, v, (const int*)c->page_list);
  if (err == cudaSuccess)
    err = launch_chained(move_pages_kernel, dim3((unsigned)std::min(v.layers * 2 * v.kv_heads, 16), (unsigned)std::min(v.pages, 64)), dim3(256), 0, st, v,
                         (const int*)c->move_src, (const int*)c->move_dst, (const int*)c->move_cnt);
  return finish(c, err, st);
}

jd_status_t jd_cache_last_status(jd_cache_t c, int* out) {
  if (!c || !out) return JD_ERR_INVALID_ARG;
  OnDevice dev(c->cfg.device);
  if (!dev.ok()) return JD_ERR_CUDA;
  unsigned word = 0;
  if (cudaStreamSynchronize(c->last_stream) != cudaSuccess ||
      cudaMemcpyAsync(&word, c->status, sizeof(word), cudaMemcpyDeviceToHost, c->last_stream) != cudaSuccess ||
      cudaMemsetAsync(c->status, 0, sizeof(word), c->last_stream) != cudaSuccess || cudaStreamSynchronize(c->last_stream) != cudaSuccess)
    return JD_ERR_CUDA;
  *out = (int)word;
  return JD_OK;
}

}  // extern "C"
