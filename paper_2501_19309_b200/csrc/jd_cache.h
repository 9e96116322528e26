// Internal interface of the paged cache: the handle, the parameters its kernels share and the
// division of an attention call's work among CTAs.
#pragma once

#include <cuda.h>

#include <type_traits>

#include "jd_common.cuh"

struct jd_cache_s {
  jd_cache_config_t cfg;
  jd_cache_buffers_t buf;
  int num_sms;
  int page_shift;
  CUtensorMap tm_k, tm_v;     // K and V as [rows, head_dim] matrices, box 64 columns x box_rows
  bool tm_ok;                 // the tensor-core attention covers this cache
  cudaStream_t last_stream;
  // regions of the workspace
  unsigned* status;
  int* commit_cnt;            // [1024] blocks of the sequence that have finished moving (self-resetting)
  int* reserve_cnt;           // [1] blocks of a reserve that are done (self-resetting)
  int* page_list;             // [num_pages] pages handed out by a reserve; page map of a compaction
  int* move_src;              // [num_pages] compaction: pages to move, and where to
  int* move_dst;
  int* move_cnt;              // [1]
  int4* split;                // [2 kMaxCtas] the segment that a group of an attention call begins and others go on with
  float* part;                // partial attention results of split sequences
};

namespace jd {

constexpr int kMaxCacheBatch = 1024;   // sequences of one call
constexpr int kMaxNodes = 128;

// What every cache kernel needs to know, by value.
struct CacheView {
  int layers, pages, page_size, page_shift, kv_heads, head_dim, max_seqs, max_pages;
  int row_bytes;             // head_dim x element size
  char* k;
  char* v;
  int32_t* table;
  int32_t* seq_len;
  int32_t* held;
  int32_t* refs;
  uint32_t* free_bits;
  unsigned* status;
};

// Row r of page p, layer l, kv head h, as a row number of the [rows, head_dim] matrix: 64 bits, a long cache
// passes 2^31 bytes many times over.
__device__ __forceinline__ int64_t page_row(const CacheView& c, int layer, int page, int head, int row) {
  return ((((int64_t)layer * c.pages + page) * c.kv_heads + head) << c.page_shift) + row;
}

// Slot of entry b: -1 for padding and for entries out of range (reported).
__device__ __forceinline__ int slot_of(const CacheView& c, const int32_t* slots, int b) {
  if (!slots) return b;
  const int s = __ldcg(slots + b);
  if (s >= 0 && s < c.max_seqs) return s;
  if (s != -1) set_status(c.status, JD_ERR_BAD_INDEX);
  return -1;
}

// Held pages and committed tokens of a slot, clamped to what the tables can mean.
__device__ __forceinline__ void slot_state(const CacheView& c, int slot, int& len, int& held) {
  held = min(max(c.held[slot], 0), c.max_pages);
  len = min(max(c.seq_len[slot], 0), held << c.page_shift);
}

// ---------------------------------------------------------------------------------------
// Attention: the call's rows and their division.
//
// A (sequence, kv head) pair is a segment of ceil(kv_end / tile) tiles of the cache, at least one. Work is counted in units: a
// segment has seg_cost units for what it costs to begin and end it, and one for each tile. All units of all segments,
// sequence-major, are cut into `groups` runs of equal length, one for each group of `row_blocks` CTAs; the CTAs of a group
// take the same tiles for different blocks of query rows, so that all but one find them in L2.
// A run that covers only a part of a segment's tiles leaves a partial result (numerator, running maximum, sum): in slot 1
// of its group if the part begins the segment, else in slot 0, so two slots are enough.
// The cut depends on nothing but the lengths and the SM count: results repeat bit for bit.
// ---------------------------------------------------------------------------------------
// Sequences that share a prefix (jd_cache_share). The call's items are then the groups, each with the tiles of its prefix and the rows of all its
// members one behind another, and the sequences with the tiles behind their prefix; an item's rows are cut into blocks of rows_per_block, and its
// segments are the kv heads and the blocks within. All lie in one division: the groups' long segments and the sequences' short ones fill the SMs
// together. A piece of a group, or of a sequence with a prefix, leaves numerators, maximum and sum: of a whole segment in a record of the row's
// own, of a part in its run's slot; a join adds them up.
enum Share { kAlone = 0, kShared = 1 };
template <int kShare> using ShareOf = std::integral_constant<int, kShare>;

constexpr int kMaxSharedBatch = 512; // sequences of a plan: groups and sequences are at most 1.5 times as many items
constexpr int kPrefixTokens = 128;   // prefixes are cut to whole tiles of the tensor-core kernel, which are whole tiles of the other
// units of all groups' prefix segments, whatever kernel takes them, and of all sequences' own ones: the sums of both are 32 bits
constexpr int64_t kMostUnits = (int64_t)1 << 30;
// tiles of kPrefixTokens that a group has to save to be one; whether the call shares anything at all goes by its cost (form_cost)
constexpr int kPrefixWorth = 2;

constexpr int kSimtRows = 16, kSimtTileShift = 6, kSimtSegCost = 1;
constexpr int kTensorTileShift = 7;
// what beginning and ending a segment costs, in tiles: some 8,000 cycles, against 1,400 (64 columns) or 2,800 (128) for a tile at
// HBM rate. A batch of 16 chains up to 6,000 tokens long: 40 us at 3, 36 at 6, 38 at 10 (64 columns). More than 128 rows: a pair of row
// tiles takes longer a tile, and its parts are large, so that cutting a segment less often pays too (16 trees of 208 rows on 200 to
// 4,000 tokens: 101 us at 1, 70 at 4, 66 at 5, 68 at 6).
__host__ __device__ constexpr int tensor_seg_cost(int head_dim, int rows) { return head_dim == 64 ? 6 : (rows > 128 ? 5 : 4); }

// Rows of a block that a shared call may have: those of the tensor-core kernel's forms, or of the other's.
constexpr int kTensorForms = 4, kSharedForms = 6;
__host__ __device__ constexpr int form_rows(int form) { return form < kTensorForms ? 32 << form : (form == kTensorForms ? 4 : 16); }
// The forms that a plan chooses from. A block of few rows costs a sequence's own few tokens least, one of many saves a group passes over its prefix: the
// smallest form that takes a sequence's rows, and, where the batch has the rows for long work, twice that in the same kernel, of which the plan picks by cost.
// A second form costs every call some 4 us (the code no longer stays in the instruction cache, and registers are spilled: 436 bytes of blocks of 128 and 256 rows of
// 128 columns, 68 of the latter alone; 15.1 us alone, 19.2 with another beside it), a
// wrong one up to twice the time. Of random calls with 33 to 64 rows of 128 columns the sum of times falls by 8 % with the rule, with 65 to 128 rows by 10 %. On
// CUDA cores, whose code is short, up to 4 rows of a sequence go in blocks of 4 or of 16; with more than 128 columns the latter would take the former's
// second block off the SM.
constexpr int kSecondForm = 1024;
struct Forms { int first, second; };
__host__ __device__ inline Forms shared_forms(bool tensor, int head_dim, int want, int B, int rows) {
  if (want && tensor == (want >= form_rows(0))) return Forms{want, want};
  if (!tensor) return rows > 4 ? Forms{kSimtRows, kSimtRows} : Forms{4, head_dim > 128 ? 4 : kSimtRows};
  const int first = rows <= 32 ? 32 : (rows <= 64 ? 64 : (rows <= 128 ? 128 : 256));
  return Forms{first, first < 256 && B * rows >= kSecondForm ? 2 * first : first};
}

// How a call's rows are cut: for sequences by themselves by the host, with a plan by its form.
struct Division {
  int rows_per_block, part_rows, seg_cost;
};

struct SharedView {                  // arrays of a plan of B sequences, all on the device
  int32_t* count;                    // [1] blocks of jd_cache_share that are done (self-resetting)
  int32_t* leader;                   // [B] the first entry with the same beginning, and the tokens that both have in the same pages: scratch
  int32_t* same;
  int32_t* group_start;              // [B / 2 + 1] first of the group's members
  int32_t* group_tokens;             // [B / 2] 0: no group
  int32_t* group_slot;               // [B / 2] slot whose pages are read
  int32_t* member;                   // [B] entries by group
  int32_t* entry_group;              // [B] -1: none
  int32_t* entry_place;              // [B] number within the group
  int32_t* entry_slot;               // [B] slot when the plan was made
  int32_t* entry_lead;               // [B] the group's slot
  int32_t* entry_tokens;             // [B] its prefix, 0: none
  int32_t* first;                    // [B] tokens that the call takes off the sequence, as the tables stand: written by it for its join
  int32_t* units;                    // [B / 2 + B + 1] the call's division (unit_prefix), likewise
  int32_t* form;                     // [2] rows of a block of the calls on the tensor cores and of the others
  float* rec_group;                  // [B x T x group][kv_heads][head_dim + kPartPad] rows by group member; by entry
  float* rec_own;
  float* part;                       // parts of the call
};

struct AttendParams {
  CacheView c;
  int B, layer, T, W;              // W: mask words of a row
  int q_heads, group;              // group: query heads of a kv head
  int rows;                        // T * group, query rows of a (sequence, kv head)
  int row_blocks, rows_per_block;  // CTAs of a group, and the rows that each takes
  int groups;
  int part_rows;                   // rows of a partial result: min(rows, rows_per_block)
  int tile_shift;
  int seg_cost;
  const int32_t* slots;
  const uint32_t* mask;
  int64_t mask_stride;             // words between sequences, 0: shared
  const int32_t* num_nodes;
  const char* q;
  char* out;
  int64_t q_stride, out_stride;    // bytes between tokens
  float* lse;
  float scale_log2;                // scale x log2(e)
  SharedView sh;                   // kShared
  int max_groups;                  // items in front of the sequences; 0 for kAlone
  int second_rows;                 // the other rows_per_block that the plan may name
  int4* split;                     // [groups] sequence, kv head and last group of the segment that the group leaves unfinished; x < 0: none
  float* part;                     // [groups * row_blocks][2][part_rows][head_dim + kPartPad]
};

constexpr int kPartPad = 4;        // a part's row is head_dim numerators, m, l and two unused words (16-byte rows)

struct SeqExtent {
  int slot, ctx, nodes, kv_end;
};
// With shared prefixes: of a sequence its first tile behind the prefix; of a group its first member, and its rows in place of nodes.
struct SharedExtent : SeqExtent {
  int more;
};
template <int kShare> struct ExtentOf { using type = SharedExtent; };
template <> struct ExtentOf<kAlone> { using type = SeqExtent; };
template <int kShare> using Extent = typename ExtentOf<kShare>::type;

// a group's first member
__device__ __forceinline__ int64_t member0_of(const SeqExtent&) { return 0; }
__device__ __forceinline__ int64_t member0_of(const SharedExtent& e) { return e.more; }

__device__ __forceinline__ SeqExtent seq_extent(const AttendParams& p, int b) {
  SeqExtent e;
  e.slot = slot_of(p.c, p.slots, b);
  e.ctx = e.nodes = e.kv_end = 0;
  if (e.slot < 0) return e;
  int held;
  slot_state(p.c, e.slot, e.ctx, held);
  e.nodes = p.num_nodes ? min(max(__ldcg(p.num_nodes + b), 0), p.T) : p.T;
  e.kv_end = min(e.ctx + e.nodes, held << p.c.page_shift);
  return e;
}
__device__ __forceinline__ int extent_units(const AttendParams& p, const Division& d, const SeqExtent& e) {
  if (e.slot < 0 || e.nodes == 0) return 0;
  return d.seg_cost + max(1, (e.kv_end + (1 << p.tile_shift) - 1) >> p.tile_shift);
}

// Tokens that sequence b leaves to its group: those of the plan if slot still has them in the group's pages, else none, so that a plan which the tables
// have left behind costs time alone. Calls change tables from their ends or as a whole, and a page has the same place in all tables that hold it, so lengths and the
// prefix's last page tell; so that the
// loads are under way together, none waits for another's outcome.
__device__ __forceinline__ int prefix_of(const AttendParams& p, int b, int slot, int ctx) {
  const int tokens = __ldcg(p.sh.entry_tokens + b), was = __ldcg(p.sh.entry_slot + b), lead = __ldcg(p.sh.entry_lead + b);
  if (tokens < 1 || slot < 0 || slot != was || lead < 0 || lead >= p.c.max_seqs || (tokens - 1) >> p.c.page_shift >= p.c.max_pages) return 0;
  const int at = (tokens - 1) >> p.c.page_shift;
  const int mine = __ldcg(p.c.table + (int64_t)slot * p.c.max_pages + at), its = __ldcg(p.c.table + (int64_t)lead * p.c.max_pages + at);
  int len, held;
  slot_state(p.c, lead, len, held);
  return mine == its && tokens <= ctx && tokens <= len ? tokens : 0;
}

// Item i of the call: a group if i < p.max_groups, else a sequence.
template <int kShare> __device__ __forceinline__ Extent<kShare> extent_at(const AttendParams& p, int i) {
  if constexpr (kShare == kAlone) {
    return seq_extent(p, i);
  } else {
    SharedExtent e;
    if (i >= p.max_groups) {
      const int b = i - p.max_groups;
      static_cast<SeqExtent&>(e) = seq_extent(p, b);
      e.more = prefix_of(p, b, e.slot, e.ctx) >> p.tile_shift;
      return e;
    }
    e.slot = -1;
    e.ctx = e.nodes = e.kv_end = e.more = 0;
    const int start = __ldcg(p.sh.group_start + i), end = __ldcg(p.sh.group_start + i + 1), tokens = __ldcg(p.sh.group_tokens + i);
    const int lead = __ldcg(p.sh.group_slot + i);
    if (tokens < 1 || lead < 0 || lead >= p.c.max_seqs) return e;
    int len, held;
    slot_state(p.c, lead, len, held);
    if (tokens > len) return e;
    e.slot = lead;
    e.ctx = e.kv_end = tokens;
    e.more = start;
    e.nodes = (end - start) * p.rows;
    return e;
  }
}
__device__ __forceinline__ int row_blocks_of(const Division& d, int rows) { return (int)((uint32_t)(rows + d.rows_per_block - 1) / (uint32_t)d.rows_per_block); }
__device__ __forceinline__ Division own_division(const AttendParams& p) { return Division{p.rows_per_block, p.part_rows, p.seg_cost}; }
template <int kShare> __device__ __forceinline__ int item_blocks(const AttendParams& p, const Division& d, int i, const Extent<kShare>& e) {
  return kShare == kAlone ? 1 : row_blocks_of(d, i < p.max_groups ? e.nodes : p.rows);
}
template <int kShare> __device__ __forceinline__ int units_at(const AttendParams& p, const Division& d, int i, const Extent<kShare>& e) {
  const int n = extent_units(p, d, e);
  if constexpr (kShare == kAlone) return n;
  else return n == 0 ? 0 : item_blocks<kShare>(p, d, i, e) * (i < p.max_groups ? n : max(n - e.more, d.seg_cost + 1));
}
template <int kShare> __device__ __forceinline__ int items_of(const AttendParams& p) { return kShare == kAlone ? p.B : p.max_groups + p.B; }

// prefix[b] = units of one kv head in the items before b, prefix[items] = all; extents (optional): what extent_at says of each
// item. By the whole block.
template <int kShare>
__device__ __forceinline__ void unit_prefix(ShareOf<kShare>, const AttendParams& p, const Division& d, int* prefix, int* warp_sums, Extent<kShare>* extents = nullptr) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, nthreads = blockDim.x, nwarps = nthreads >> 5, items = items_of<kShare>(p);
  int carry = 0;
  for (int b0 = 0; b0 < items; b0 += nthreads) {
    const int b = b0 + tid;
    int n = 0;
    if (b < items) {
      const Extent<kShare> e = extent_at<kShare>(p, b);
      if (extents) extents[b] = e;
      n = units_at<kShare>(p, d, b, e);
      if constexpr (kShare == kShared)
        if (blockIdx.x == 0 && b >= p.max_groups) p.sh.first[b - p.max_groups] = e.more << p.tile_shift;
    }
    int x = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    if (lane == 31) warp_sums[warp] = x;
    __syncthreads();
    int before = carry, all = 0;
    for (int w = 0; w < nwarps; ++w) {
      if (w < warp) before += warp_sums[w];
      all += warp_sums[w];
    }
    if (b < items) prefix[b] = before + x - n;
    carry += all;
    __syncthreads();
  }
  if (tid == 0) prefix[items] = carry;
  __syncthreads();
  if constexpr (kShare == kShared) {
    if (blockIdx.x == 0)
      for (int i = tid; i <= items; i += nthreads) p.sh.units[i] = prefix[i];
  }
}

// First unit of run g, and the run that holds unit u; 32-bit divisions where they are enough (64-bit ones take ten times as long).
// With fewer units than groups the first `units` groups take one each: a run between two others is never empty, so that every group
// between a segment's first and its last has left a part.
__device__ __forceinline__ int64_t run_start(int64_t units, int groups, int g) {
  if (units <= groups) return min((int64_t)g, units);
  const int64_t n = units * g;
  return units < (1 << 22) ? (int64_t)((uint32_t)n / (uint32_t)groups) : n / groups;
}
__device__ __forceinline__ int run_of(int64_t units, int groups, int64_t u) {
  if (units <= groups) return (int)u;
  const int64_t n = (u + 1) * groups - 1;
  return units < (1 << 22) ? (int)((uint32_t)n / (uint32_t)units) : (int)(n / units);
}

// One stretch of a run inside a segment. tiles may be 0: the run holds only units that stand for the segment's fixed cost.
struct Piece {
  int b, head, tile0, tiles, all;   // b: item; all: tiles of the whole segment
  int64_t next;                     // first unit behind it
  int first;                        // the segment's first tile in the sequence; 0 unless a prefix is taken off
  int row0;                         // the segment's first row; 0 where CTAs share a sequence's rows
};
template <int kShare = kAlone>
__device__ __forceinline__ Piece piece_at(const AttendParams& p, const Division& d, const int* prefix, int64_t u, int64_t run1, const Extent<kShare>* extents = nullptr) {
  Piece x;
  x.first = x.row0 = 0;
  int lo = 0, hi = items_of<kShare>(p) - 1;   // the last item with units whose first is at or before u
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if ((int64_t)prefix[mid] * p.c.kv_heads <= u) lo = mid; else hi = mid - 1;
  }
  x.b = lo;
  const int64_t first = (int64_t)prefix[lo] * p.c.kv_heads;
  int n = prefix[lo + 1] - prefix[lo], segment;
  if constexpr (kShare == kShared) {
    const Extent<kShare> e = extents ? extents[lo] : extent_at<kShare>(p, lo);
    const int blocks = item_blocks<kShare>(p, d, lo, e);
    if (lo >= p.max_groups) x.first = e.more;
    n = (int)((uint32_t)n / (uint32_t)blocks);
    const int64_t in_item = u - first;
    segment = in_item < 0x7FFFFFFF ? (int)((uint32_t)in_item / (uint32_t)n) : (int)(in_item / n);
    x.head = (int)((uint32_t)segment / (uint32_t)blocks);
    x.row0 = (segment - x.head * blocks) * d.rows_per_block;
  } else {
    const int in_seq = (int)(u - first);
    x.head = segment = (int)((uint32_t)in_seq / (uint32_t)n);
  }
  const int at = (int)(u - first - (int64_t)segment * n);
  const int64_t seg_end = first + (int64_t)(segment + 1) * n;
  x.next = min(seg_end, run1);
  x.all = n - d.seg_cost;
  x.tile0 = max(0, at - d.seg_cost);
  x.tiles = max(0, at + (int)(x.next - u) - d.seg_cost) - x.tile0;
  return x;
}

// Mask word of node t for nodes 32 w .. 32 w + 31, nodes behind the sequence's last one hidden.
__device__ __forceinline__ uint32_t node_word(const AttendParams& p, int b, int t, int w, int nodes) {
  const int left = nodes - 32 * w;
  if (left <= 0) return 0u;
  uint32_t m;
  if (p.mask) m = __ldcg(p.mask + (int64_t)b * p.mask_stride + (int64_t)t * p.W + w);
  else { const int own = t + 1 - 32 * w; m = own >= 32 ? 0xFFFFFFFFu : (own <= 0 ? 0u : (1u << own) - 1u); }
  return left >= 32 ? m : m & ((1u << left) - 1u);
}

// What the join goes by: group g begins this segment and run `last` ends it. By one thread of the group's first CTA: none() as the kernel
// starts, set() where a piece begins a segment that it does not end.
__device__ __forceinline__ void split_none(const AttendParams& p, int g) { p.split[g] = make_int4(-1, 0, 0, 0); }
__device__ __forceinline__ void split_set(const AttendParams& p, int g, int64_t units, const Piece& x) {
  p.split[g] = make_int4(x.b, x.head, run_of(units, p.groups, x.next + (x.all - x.tiles) - 1), 0);
}

__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void pdl_trigger() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// How a call with a plan cuts its rows, once the kernel that may have made the plan is done.
template <bool kTensor> __device__ __forceinline__ Division plan_division(const AttendParams& p) {
  Division d = own_division(p);
  if (p.second_rows == p.rows_per_block) return d;
  pdl_wait();
  if (__ldcg(p.sh.form + (kTensor ? 0 : 1)) == p.second_rows) {
    d.rows_per_block = p.second_rows;
    d.part_rows = min(p.B * p.rows, p.second_rows);
    if (kTensor) d.seg_cost = tensor_seg_cost(p.c.head_dim, p.second_rows);
  }
  return d;
}

// A kernel that starts early runs while the one in front of it still writes, so nothing it reads is read-only for its whole life: the
// kernels here use no non-coherent loads (__ldg, const __restrict__), and take what other kernels write from L2 (__ldcg) or by plain
// loads behind pdl_wait().
// Launches a kernel that may start before the one in front of it on the stream has ended; it calls pdl_wait() before it reads or
// writes anything that another kernel touches. (In front of a kernel that triggers nothing itself this saves the launch's latency alone.)
template <typename... Params, typename... Args>
inline cudaError_t launch_chained(void (*kernel)(Params...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<Params>(args)...);
}

cudaError_t run_attend_simt(const AttendParams& p, int dtype, cudaStream_t st);
cudaError_t run_attend_tensor(const AttendParams& p, const CUtensorMap& tm_k, const CUtensorMap& tm_v, cudaStream_t st);
cudaError_t run_attend_join(const AttendParams& p, int dtype, cudaStream_t st);
// Attention with a plan, and what adds its results up.
cudaError_t run_attend_shared_simt(const AttendParams& p, int dtype, cudaStream_t st);
cudaError_t run_attend_shared_tensor(const AttendParams& p, const CUtensorMap& tm_k, const CUtensorMap& tm_v, cudaStream_t st);
cudaError_t run_attend_shared_join(const AttendParams& p, int dtype, cudaStream_t st);
bool simt_attend_configure();
bool attend_configure();   // dynamic shared-memory limits on the current device, once per device

cudaError_t run_share(const CacheView& c, const SharedView& s, const jd_shared_t& plan, int q_heads, bool tensor, int num_sms, const int32_t* slots, const int32_t* groups, cudaStream_t st);
bool rope_valid(const jd_rope_t& r, int head_dim);
cudaError_t run_append(const CacheView& c, const jd_append_args_t& a, int q_heads, int dtype, cudaStream_t st);
bool append_heads_valid(const jd_head_norm_t* n, const jd_rope_axes_t* a, const jd_rope_t* r);
cudaError_t run_append_heads(const CacheView& c, const jd_append_args_t& a, const jd_append_heads_t& x, int q_heads, int dtype, cudaStream_t st);

}  // namespace jd
