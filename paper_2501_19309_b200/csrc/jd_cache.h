// Internal interface of the paged cache: the handle, the parameters its kernels share and the
// division of an attention call's work among CTAs.
#pragma once

#include <cuda.h>

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
  int4* split;                     // [groups] sequence, kv head and last group of the segment that the group leaves unfinished; x < 0: none
  float* part;                     // [groups * row_blocks][2][part_rows][head_dim + kPartPad]
};

constexpr int kPartPad = 4;        // a part's row is head_dim numerators, m, l and two unused words (16-byte rows)

struct SeqExtent {
  int slot, ctx, nodes, kv_end;
};
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
__device__ __forceinline__ int extent_units(const AttendParams& p, const SeqExtent& e) {
  if (e.slot < 0 || e.nodes == 0) return 0;
  return p.seg_cost + max(1, (e.kv_end + (1 << p.tile_shift) - 1) >> p.tile_shift);
}

// prefix[b] = units of one kv head in the sequences before b, prefix[B] = all; extents (optional): what seq_extent says of each
// sequence. By the whole block.
__device__ __forceinline__ void unit_prefix(const AttendParams& p, int* prefix, int* warp_sums, SeqExtent* extents = nullptr) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, nthreads = blockDim.x, nwarps = nthreads >> 5;
  int carry = 0;
  for (int b0 = 0; b0 < p.B; b0 += nthreads) {
    const int b = b0 + tid;
    int n = 0;
    if (b < p.B) {
      const SeqExtent e = seq_extent(p, b);
      if (extents) extents[b] = e;
      n = extent_units(p, e);
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
    if (b < p.B) prefix[b] = before + x - n;
    carry += all;
    __syncthreads();
  }
  if (tid == 0) prefix[p.B] = carry;
  __syncthreads();
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
  int b, head, tile0, tiles, all;   // all: tiles of the whole segment
  int64_t next;                     // first unit behind it
};
__device__ __forceinline__ Piece piece_at(const AttendParams& p, const int* prefix, int64_t u, int64_t run1) {
  Piece x;
  int lo = 0, hi = p.B - 1;         // the last sequence with units whose first is at or before u
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if ((int64_t)prefix[mid] * p.c.kv_heads <= u) lo = mid; else hi = mid - 1;
  }
  x.b = lo;
  const int n = prefix[lo + 1] - prefix[lo];
  const int64_t first = (int64_t)prefix[lo] * p.c.kv_heads;
  const int in_seq = (int)(u - first);
  x.head = (int)((uint32_t)in_seq / (uint32_t)n);
  const int at = in_seq - x.head * n;
  const int64_t seg_end = first + (int64_t)(x.head + 1) * n;
  x.next = min(seg_end, run1);
  x.all = n - p.seg_cost;
  x.tile0 = max(0, at - p.seg_cost);
  x.tiles = max(0, at + (int)(x.next - u) - p.seg_cost) - x.tile0;
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
bool simt_attend_configure();
bool attend_configure();   // dynamic shared-memory limits on the current device, once per device
constexpr int kSimtRows = 16, kSimtTileShift = 6, kSimtSegCost = 1;
constexpr int kTensorTileShift = 7;
// what beginning and ending a segment costs, in tiles: some 8,000 cycles, against 1,400 (64 columns) or 2,800 (128) for a tile at
// HBM rate. A batch of 16 chains up to 6,000 tokens long: 40 us at 3, 36 at 6, 38 at 10 (64 columns). More than 128 rows: a pair of row
// tiles takes longer a tile, and its parts are large, so that cutting a segment less often pays too (16 trees of 208 rows on 200 to
// 4,000 tokens: 101 us at 1, 70 at 4, 66 at 5, 68 at 6).
constexpr int tensor_seg_cost(int head_dim, int rows) { return head_dim == 64 ? 6 : (rows > 128 ? 5 : 4); }

bool rope_valid(const jd_rope_t& r, int head_dim);
cudaError_t run_append(const CacheView& c, const jd_append_args_t& a, int q_heads, int dtype, cudaStream_t st);

}  // namespace jd
