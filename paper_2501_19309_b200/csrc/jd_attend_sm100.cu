// Attention of a drafted block over the paged cache on the tensor cores (bf16, head width 64 or 128).
//
// Rows of a (sequence, kv head) are its nodes times the query heads that share the kv head; a CTA takes up to 128 or 256
// of them through its run of tiles of 128 cached tokens (jd_cache.h says how runs are cut). Per tile and 128 rows:
//
//   S = Q K^T            tcgen05.mma, Q and K tiles in shared memory, S (128 x 128 fp32) in tensor memory
//   P = 2^(S c - m)      a thread per row reads its row of S, keeps the running maximum m and sum l in registers and
//                        writes P as bf16 over S
//   O = O + P V          tcgen05.mma with P from tensor memory, V as it lies in its pages (tokens x columns: the
//                        transposed operand form), O (128 x head width fp32) in tensor memory
//
// P is rounded to bf16, by 2^-8 of each weight at most, because the product takes no wider type at this rate; l is the sum of the
// weights before they are rounded, so that the logarithm of the sum keeps float32. O is rescaled only when a row's
// maximum has grown by more than 2^8 since it was last (the weights stay below 2^8 until then), which after the first
// tiles is rare.
//
// Two chains S -> softmax -> P V keep the pipe busy while each waits for itself, a warpgroup for each one's softmax. With up to 128
// rows they take alternate tiles, each with its own O, m and l that meet when the segment ends; with more rows each takes 128
// rows of every tile, and K and V are fetched once for both. Two warps follow the page table and fetch K and V tiles by
// TMA, a box per page and 64 columns, through a ring; one or two more issue the MMAs.
//
// What bounds it (B200, 148 SMs):
//   up to 128 rows   long contexts: HBM. 16 sequences of 40,000 tokens, 8 kv heads of 128, one token each: 391 us, 6.7 TB/s; heads of 64: 204 us,
//                    6.4 TB/s. Ragged batches: beginning and ending segments (16 chains of 9 on 90 to 6,000 tokens, heads of 64: 36 us, 44 %
//                    of the HBM rate)
//   129 rows and up  the chains' own latency: a pair of row tiles takes about 3,450 cycles a tile, of which its products are 2,200 (S: 75
//                    cycles a step of 16 columns, as Q comes from shared memory again every time; P V: 64), its exponentials
//                    2,050 on each SM partition and the rest the hand-overs between them; 416 rows over 131,046 tokens: 252 us, 885 TFLOP/s,
//                    in short bursts; back to back the power limit holds the clock near 1.5 GHz: 298 us, 750 TFLOP/s. 4 sequences of
//                    208 rows on 9,000 to 40,000 tokens: heads of 128 114 us, of 64 102 us
//   short contexts   about 8,000 cycles to begin and end a segment
// Tried and slower: a second pair of softmax warpgroups, half the columns each (275 against 260 us on that case); a quarter of the
// exponentials as polynomials on the FMA pipe (274); S in halves of 64 tokens with a buffer each, so that the next is ready when
// one is done (282: a product of 64 columns costs what one of 128 does); weighing against the maximum so far while the
// tile's own is found (265).
#include <algorithm>
#include <type_traits>

#include "jd_cache.h"
#include "jd_sm100_ptx.cuh"

namespace jd {
namespace {

constexpr int kTile = 1 << kTensorTileShift;   // cached tokens of a tile
constexpr int kThreads = 384;                  // warps 0-3, 4-7: softmax; 8, 10: TMA; 9, 11: MMA
constexpr int kSoftmaxRegs = 216, kOtherRegs = 72;   // 2 x 128 x 216 + 128 x 72 = 384 x 168, what the block is launched with
constexpr float kLazy = 8.f;                   // log2 of how far a maximum may grow before O is rescaled

// 2^(s c - base) with base = m c rounded is off by 2^(2^-24 base) in all weights of a row alike, which the sum divides out again as long as
// float32 holds it. From this base on neighbouring float32 scores are 16 and more apart, so that a weight is 1 or next to nothing, any
// factor not below c tells which, and with the next power of two base is exact.
constexpr float kFar = 0x1p28f;

// How a CTA's rows lie in the 128 rows of an MMA. kPairMode: up to 256 rows, two MMAs, every tile for both chains. Else up to 128 / kMode rows,
// kMode times over: the copies weigh a kMode-th of a tile's columns each and have zeroes for the rest of P, so that few rows
// keep all four SM partitions' exponential units busy instead of one; their O, m and l are parts that meet at the end.
constexpr int kPairMode = 0;
template <int D, int kMode> struct Shape {
  static constexpr bool kPair = kMode == kPairMode;
  static constexpr int kCopies = kPair ? 1 : kMode;
  static constexpr int kCopyRows = 128 / kCopies;              // rows of a copy
  static constexpr int kCols = kTile / kCopies;                // columns of S that a thread weighs
  static constexpr int kChunks = D / 64;                       // 128-byte column groups
  static constexpr int kChunkBytes = kTile * 128;
  static constexpr int kTileBytes = kChunks * kChunkBytes;     // one K, V or Q tile
  // A multiple of 4, so that K and V keep to slots of their own and, with alternate tiles, so do the two chains: a slot's barrier is then
  // only ever waited on by those that used up its previous content, and two phases cannot be taken for one another.
  static constexpr int kStages = D == 128 ? 4 : 8;
  static constexpr int kQTiles = kPair ? 2 : 1;
  static constexpr int kStageCols = D / 4;                     // columns of O that the copies' sums go through shared memory by
  static constexpr int kStageBytes = kCopies > 1 ? 2 * 128 * kStageCols * 4 : 0;
  // Q of the next piece is fetched while this one ends, where the registers are there for it: 256 rows of 128 columns are 64 a thread.
  static constexpr bool kFetchAhead = !kPair || D == 64;
  // What is kept of a piece (Shared::PerPiece): this one's and the next's. With every tile for both chains and Q fetched ahead a warpgroup
  // can be through with a short piece while the other still writes the one before it out, and hands over the one behind: three.
  static constexpr int kPieces = kPair && kFetchAhead ? 3 : 2;
};

template <int kPieces> struct Shared {
  uint64_t full[8], empty[8];
  uint64_t s_full[2], p_ready[2][2], o_done[2], q_ready[2];   // p_ready: first and second 64 columns of P
  uint32_t tmem_base;
  int abort_flag;
  int warp_sums[kThreads / 32];
  struct PerPiece {                      // of a piece, and of the next ones, which begin while this one is written out
    uint32_t node_mask[kMaxNodes][kMaxNodes / 32];
    float ml[2][kTile][2];               // m and l of the two chains
    float inv[2][kTile / 2];             // 1 / l of a row, for the threads that put its copies together
    int odd_values;                      // nodes hold values that are not finite
  } piece[kPieces];
  int prefix[kMaxCacheBatch + 1];
  SeqExtent extents[kMaxCacheBatch];
};

template <int D, int kMode>
constexpr size_t attend_smem() {
  using S = Shape<D, kMode>;
  return 1024 + (sizeof(Shared<S::kPieces>) + 1023) / 1024 * 1024 + (size_t)(S::kStages + S::kQTiles) * S::kTileBytes + S::kStageBytes;
}

// Bounded wait that gives up as soon as another role has.
__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
  for (unsigned it = 0; it < kSpinLimit; ++it) {
    if (mbar_try_wait(bar, parity)) return true;
    if (*abort_flag) return false;
    if (it > 128) __nanosleep(64);
  }
  *abort_flag = 1;
  return false;
}

__device__ __forceinline__ void fence_async_proxy() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void softmax_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

__device__ __forceinline__ uint64_t policy_evict_normal() {
  uint64_t p;
  asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(p));
  return p;
}

// V tile as the MMA's B operand [tokens x columns], columns contiguous: 128-byte swizzle, 64-column groups kChunkBytes apart,
// groups of 8 tokens 1024 bytes apart.
__device__ __forceinline__ uint64_t make_v_desc(uint32_t saddr, uint32_t chunk_bytes) {
  uint64_t d = 0;
  d |= (uint64_t)((saddr & 0x3FFFFu) >> 4);
  d |= (uint64_t)(chunk_bytes >> 4) << 16;
  d |= (uint64_t)(1024u >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}
constexpr uint32_t kTransposeB = 1u << 16;

// A from tensor memory: lane = row, two bf16 per column
__device__ __forceinline__ void umma_bf16_ta(uint32_t tmem_d, uint32_t tmem_a, uint64_t db, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(tmem_d), "r"(tmem_a), "l"(db), "r"(idesc), "r"(acc) : "memory");
}

__device__ __forceinline__ void ld32_issue(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
        "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
        "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void pin16(uint32_t* r) {
#pragma unroll
  for (int i = 0; i < 16; i += 8)
    asm volatile("" : "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3]), "+r"(r[i + 4]), "+r"(r[i + 5]), "+r"(r[i + 6]), "+r"(r[i + 7])
                 :: "memory");
}
// keeps what reads the registers behind the wait in front of it (the statement itself is empty)
__device__ __forceinline__ void pin32(uint32_t* r) {
#pragma unroll
  for (int i = 0; i < 32; i += 8)
    asm volatile("" : "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3]), "+r"(r[i + 4]), "+r"(r[i + 5]), "+r"(r[i + 6]), "+r"(r[i + 7])
                 :: "memory");
}
__device__ __forceinline__ void st16(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void st32(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
      "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]),
        "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]),
        "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// one lane of the converged warp
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n\t.reg .pred q;\n\telect.sync _|q, 0xFFFFFFFF;\n\tselp.b32 %0, 1, 0, q;\n\t}" : "=r"(p));
  return p != 0;
}
__device__ __forceinline__ int64_t uniform64(int64_t x) {
  const uint32_t lo = __shfl_sync(0xffffffffu, (uint32_t)x, 0), hi = __shfl_sync(0xffffffffu, (uint32_t)((uint64_t)x >> 32), 0);
  return (int64_t)(((uint64_t)hi << 32) | lo);
}

// two float32 at once: one issue slot for two lanes' worth of the FMA pipe
__device__ __forceinline__ uint64_t pack2(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// Sums of the values of cached tokens begin .. end - 1 that are not finite, in four columns from c; begin is a multiple of 8. A call of its own,
// since it is hardly ever made, with 32 loads under way at once, since other roles' waits have a limit (some 1.8 s; 65 ns a token and call,
// up to eight calls a thread and piece: some 3 million tokens of a piece, with infinities in all columns and no NaN).
template <int D>
__device__ __noinline__ float4 spoilt_by_context(const AttendParams& p, int slot, int head, int begin, int end, int c) {
  constexpr int kGroups = 4, kGroup = 8;               // no page is smaller than a group
  float sum[4] = {};
  for (int kv0 = begin; kv0 < end; kv0 += kGroups * kGroup) {
    uint2 y[kGroups * kGroup];
    int page[kGroups];
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      const int kv = kv0 + g * kGroup;
      page[g] = kv < end ? __ldcg(p.c.table + (int64_t)slot * p.c.max_pages + (kv >> p.c.page_shift)) : -1;
    }
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      const int kv = kv0 + g * kGroup;
      const bool there = page[g] >= 0 && page[g] < p.c.pages;
      const uint2* v = reinterpret_cast<const uint2*>(reinterpret_cast<const __nv_bfloat16*>(p.c.v) +
                                                      page_row(p.c, p.layer, there ? page[g] : 0, head, kv & (p.c.page_size - 1)) * D + c);
#pragma unroll
      for (int k = 0; k < kGroup; ++k) {
        const uint2 x = __ldcg(v + k * (D / 4));       // rows of the page behind the last token are there, whatever they hold
        y[g * kGroup + k] = there && kv + k < end ? x : make_uint2(0u, 0u);
      }
    }
#pragma unroll
    for (int k = 0; k < kGroups * kGroup; ++k) {
      const float e[4] = {__uint_as_float(y[k].x << 16), __uint_as_float(y[k].x & 0xFFFF0000u), __uint_as_float(y[k].y << 16), __uint_as_float(y[k].y & 0xFFFF0000u)};
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (!isfinite(e[i])) sum[i] += e[i];
    }
    if (isnan(sum[0]) && isnan(sum[1]) && isnan(sum[2]) && isnan(sum[3])) break;
  }
  return make_float4(sum[0], sum[1], sum[2], sum[3]);
}

template <int D, int kMode>
__global__ void __launch_bounds__(kThreads, 1)
attend_sm100_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ AttendParams p) {
  using Sh = Shape<D, kMode>;
  constexpr bool kPair = Sh::kPair;
  constexpr int kCopies = Sh::kCopies, kCopyRows = Sh::kCopyRows, kCols = Sh::kCols;
  constexpr int kStages = Sh::kStages, kChunks = Sh::kChunks, kChunkBytes = Sh::kChunkBytes, kTileBytes = Sh::kTileBytes;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  using Shm = Shared<Sh::kPieces>;
  Shm& sh = *reinterpret_cast<Shm*>(smem);
  uint8_t* q_smem = smem + (sizeof(Shm) + 1023) / 1024 * 1024;
  uint8_t* ring = q_smem + Sh::kQTiles * kTileBytes;
  uint8_t* stage_smem = ring + kStages * kTileBytes;
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  volatile int* abort_flag = &sh.abort_flag;
  const int g = blockIdx.x / p.row_blocks, rb = blockIdx.x - g * p.row_blocks;

  if (tid == 0) {
    for (int i = 0; i < kStages; ++i) { mbar_init(smem_u32(&sh.full[i]), 1); mbar_init(smem_u32(&sh.empty[i]), 1); }
    for (int w = 0; w < 2; ++w) {
      mbar_init(smem_u32(&sh.s_full[w]), 1);
      mbar_init(smem_u32(&sh.p_ready[w][0]), 4);
      mbar_init(smem_u32(&sh.p_ready[w][1]), 4);
      mbar_init(smem_u32(&sh.o_done[w]), 1);
      mbar_init(smem_u32(&sh.q_ready[w]), 8);
    }
    sh.abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  pdl_wait();      // so far nothing was touched that another kernel knows of
  // Tensor memory is taken behind the wait and held before the next kernel may start: a block that holds it while it waits for a kernel in
  // front, whose blocks on the same SM have yet to take theirs, would wait for good, and so would this one for a block behind it.
  if (warp == 9) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem_base)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  if (rb == 0 && tid == 0) split_none(p, g);
  unit_prefix(p, sh.prefix, sh.warp_sums, sh.extents);   // ends with a barrier
  pdl_trigger();
  tc_fence_after();
  const int64_t units = (int64_t)sh.prefix[p.B] * p.c.kv_heads;
  const int64_t run0 = run_start(units, p.groups, g), run1 = run_start(units, p.groups, g + 1);
  const uint32_t tmem = __shfl_sync(0xffffffffu, sh.tmem_base, 0);
  const uint32_t ring_addr = smem_u32(ring), q_addr = smem_u32(q_smem);

  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
    if (warp == 8 || warp == 10) {
      // ------------------------------------------------------------------ producers: warp 8 fetches K tiles, warp 10 V tiles
      // Ring items are K and V of the run's tiles in turn. A box costs the issuing warp about 100 cycles, whatever its size, which with
      // small pages is most of a tile's time: hence a warp each. Page numbers are fetched two tiles ahead.
      const bool is_v = warp == 10;
      const CUtensorMap* tm = is_v ? &tm_v : &tm_k;
      const uint64_t policy = p.row_blocks == 1 ? policy_evict_first() : policy_evict_normal();
      const int shift = p.c.page_shift, box_shift = min(shift, kTensorTileShift), boxes_per_tile = kTile >> box_shift;
      const int no_row = (int)page_row(p.c, p.c.layers, 0, 0, 0);   // one behind the last: reads as zero
      int stage = is_v ? 1 : 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int64_t u = run0; u < run1 && ok;) {
        const Piece x = piece_at(p, sh.prefix, u, run1);
        u = x.next;
        if (x.tiles == 0) continue;
        const SeqExtent ex = sh.extents[x.b];
        const int32_t* table = p.c.table + (int64_t)ex.slot * p.c.max_pages;
        auto token_of = [&](int t) { return (x.tile0 + t) * kTile + (lane << box_shift); };   // this lane's box of tile t
        auto fetch = [&](int t) {
          const int at = token_of(t);
          return t < x.tiles && lane < boxes_per_tile && at < ex.kv_end ? __ldcg(table + (at >> shift)) : 0;
        };
        int page0 = fetch(0), page1 = fetch(1);
        for (int t = 0; t < x.tiles; ++t) {
          const int page = page0;
          page0 = page1;
          page1 = fetch(t + 2);
          const int at = token_of(t);
          const bool mine = lane < boxes_per_tile && at < ex.kv_end;
          int row = no_row;
          if (mine) {
            if (page >= 0 && page < p.c.pages) row = (int)page_row(p.c, p.layer, page, x.head, at & (p.c.page_size - 1));
            else set_status(p.c.status, JD_ERR_BAD_INDEX);
          }
          const int boxes = __popc(__ballot_sync(0xffffffffu, mine));
          const uint32_t bar = smem_u32(&sh.full[stage]);
          if (lane == 0) {
            ok = wait(smem_u32(&sh.empty[stage]), phase ^ 1u, abort_flag);
            if (ok) mbar_expect_tx(bar, (uint32_t)(boxes * kChunks) << (box_shift + 7));
          }
          ok = __shfl_sync(0xffffffffu, ok, 0);
          if (!ok) break;
          if (mine) {
            const uint32_t dst = ring_addr + stage * kTileBytes + ((uint32_t)lane << (box_shift + 7));
#pragma unroll
            for (int c = 0; c < kChunks; ++c) tma_load_2d(dst + c * kChunkBytes, tm, bar, c * 64, row, policy);
          }
          stage += 2;
          if (stage >= kStages) { stage -= kStages; phase ^= 1u; }
        }
      }
      if (!ok && lane == 0) set_status(p.c.status, JD_ERR_TIMEOUT);
    } else if (!kPair || warp == 9) {
      // ------------------------------------------------------------------ MMA issue
      // Alternate tiles: warp 9 for chain 0, warp 11 for chain 1, since S -> softmax -> P V -> S is what a chain waits for and each
      // wait and issue costs its warp some 150 cycles. Every tile for both chains: warp 9 alone, because its order (all of chain 0's
      // products, then chain 1's) is what keeps one chain's softmax beside the other's products; two warps' products
      // interleave, the chains fall into step, and the long-context call takes a third longer (342 against 258 us).
      // The whole warp walks the schedule and one elected lane issues: descriptors and addresses then live in uniform registers,
      // which is what the instruction takes. (Inside an `if (lane == 0)` every MMA moved its operands there first, and the
      // issue took longer than the products.)
      const uint32_t idesc_s = make_idesc(kTile), idesc_o = make_idesc(D) | kTransposeB;
      uint32_t p_phase[2] = {0, 0}, q_phase[2] = {0, 0};
      bool ok = true;                                  // after a wait that ran out nothing waits any more; what is issued reads stale tiles
      auto await = [&](uint64_t* bar, uint32_t phase) {
        ok = wait(smem_u32(bar), phase, abort_flag) && ok;
        __syncwarp();
        tc_fence_after();
      };
      auto slot = [](int item) { return item % kStages; };
      auto await_item = [&](int item) { await(&sh.full[slot(item)], (uint32_t)(item / kStages) & 1u); };
      auto issue_s = [&](int w, int item, bool release) {   // S = Q K^T; the last chain that reads K lets it go
        const uint64_t a = make_smem_desc(q_addr + (kPair ? w * kTileBytes : 0)), b = make_smem_desc(ring_addr + slot(item) * kTileBytes);
        if (elect_one()) {
#pragma unroll
          for (int k = 0; k < D / 16; ++k) {
            const uint32_t off = ((k >> 2) * kChunkBytes + (k & 3) * 32) >> 4;
            umma_bf16(tmem + w * 128, a + off, b + off, idesc_s, k == 0 ? 0u : 1u);
          }
          umma_commit(smem_u32(&sh.s_full[w]));
          if (release) umma_commit(smem_u32(&sh.empty[slot(item)]));
        }
        __syncwarp();
      };
      auto issue_o = [&](int w, int item, uint32_t acc, bool release) {   // O (+)= P V as the halves of P arrive
        const uint64_t b = make_v_desc(ring_addr + slot(item) * kTileBytes, kChunkBytes);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          await(&sh.p_ready[w][half], p_phase[w]);
          if (elect_one()) {
#pragma unroll
            for (int k = half * (kTile / 32); k < (half + 1) * (kTile / 32); ++k)
              umma_bf16_ta(tmem + 256 + w * 128, tmem + w * 128 + k * 8, b + (k * 2048 >> 4), idesc_o, k == 0 ? acc : 1u);
            if (half == 1) {
              umma_commit(smem_u32(&sh.o_done[w]));
              if (release) umma_commit(smem_u32(&sh.empty[slot(item)]));
            }
          }
          __syncwarp();
        }
        p_phase[w] ^= 1u;
      };
      int base = 0;                                    // ring items of the pieces in front
      for (int64_t u = uniform64(run0); u < uniform64(run1);) {
        const Piece x = piece_at(p, sh.prefix, u, run1);
        const int n = __shfl_sync(0xffffffffu, x.tiles, 0);
        u = uniform64(x.next);
        if (n == 0) continue;
        if constexpr (kPair) {
          await(&sh.q_ready[0], q_phase[0]);
          await(&sh.q_ready[1], q_phase[0]);
          q_phase[0] ^= 1u;
          await_item(base);
          issue_s(0, base, false);
          issue_s(1, base, true);
          for (int t = 0; t < n; ++t) {
            const int v = base + 2 * t + 1;
            const bool more = t + 1 < n;
            await_item(v);
            issue_o(0, v, t > 0, false);
            if (more) { await_item(v + 1); issue_s(0, v + 1, false); }
            issue_o(1, v, t > 0, true);
            if (more) issue_s(1, v + 1, true);
          }
        } else {
          const int w = warp == 11 ? 1 : 0;            // tiles w, w + 2, .. are this chain's
          if (w < n) {
            await(&sh.q_ready[w], q_phase[w]);
            q_phase[w] ^= 1u;
            await_item(base + 2 * w);
            issue_s(w, base + 2 * w, true);
          }
          for (int t = w; t < n; t += 2) {
            const int v = base + 2 * t + 1;
            const bool more = t + 2 < n;
            await_item(v);                             // ahead of P, so that nothing stands between P's arrival and the products
            if (more) await_item(v + 3);
            issue_o(w, v, t > w, true);
            if (more) issue_s(w, v + 3, true);
          }
        }
        base += 2 * n;
      }
      if (!ok && lane == 0) set_status(p.c.status, JD_ERR_TIMEOUT);
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
    // ------------------------------------------------------------------ softmax: thread = row
    const int w = warp >> 2, r = tid & 127;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t t_s = tmem + lanes + w * 128, t_o = tmem + lanes + 256 + w * 128;
    const int r0 = rb * p.rows_per_block;
    const int copy = r / kCopyRows, col0 = copy * kCols;            // the copy that this warp belongs to, and its columns
    const int my_row = r0 + r % kCopyRows + (kPair ? w * 128 : 0);
    const bool warp_live = my_row - lane < p.rows;
    const int t_node = my_row / p.group, gq = my_row - t_node * p.group;
    const float c2 = p.scale_log2;
    const float c2_far = __uint_as_float((__float_as_uint(c2) + 0x7FFFFFu) & 0xFF800000u);
    uint32_t s_phase = 0, o_phase = 0;
    int tile_count = 0;                              // tiles of the run in front of this piece
    // A piece's Q rows and mask words, fetched while the piece before it ends: a thread keeps its place within a row of Q
    constexpr int kVecs = D / 8, kQThreads = kPair ? 128 : 256, kQRows = kQThreads / kVecs, kQLoads = kCopyRows / kQRows;
    static_assert(kCopyRows % kQRows == 0, "whole steps");
    constexpr int kMaskLoads = kMaxNodes * (kMaxNodes / 32) / 256;
    const int q_first = kPair ? r : tid, q_c = q_first % kVecs, q_r = q_first / kVecs;
    const int q_row0 = r0 + (kPair ? w * 128 : 0) + q_r, q_t = q_row0 / p.group, q_h = q_row0 - q_t * p.group;
    const int step_t = kQRows / p.group, step_h = kQRows - step_t * p.group;
    uint4 q_regs[kQLoads];
    uint32_t mask_regs[kMaskLoads];
    int64_t u = run0;
    auto next_piece = [&]() {                        // tiles == 0: none left
      Piece y;
      y.tiles = 0;
      while (u < run1) {
        y = piece_at(p, sh.prefix, u, run1);
        u = y.next;
        if (y.tiles > 0) break;
      }
      return y;
    };
    auto fetch = [&](const Piece& y) {
      if (y.tiles == 0) return;
      const int nodes = sh.extents[y.b].nodes;
      const char* q_seq = p.q + (int64_t)y.b * p.T * p.q_stride + (int64_t)y.head * p.group * (D * 2) + q_c * 16;
      // every load is made, rows that are not there from the first one's place: no branch stands between a load and the next
      int t = q_t, h = q_h;
#pragma unroll
      for (int i = 0; i < kQLoads; ++i) {
        const bool there = t < min(nodes, p.T);
        const uint4 v = __ldcg(reinterpret_cast<const uint4*>(q_seq + (there ? t * p.q_stride + h * (D * 2) : 0)));
        q_regs[i] = make_uint4(there ? v.x : 0u, there ? v.y : 0u, there ? v.z : 0u, there ? v.w : 0u);
        t += step_t;
        h += step_h;
        if (h >= p.group) { h -= p.group; ++t; }
      }
#pragma unroll
      for (int i = 0; i < kMaskLoads; ++i) {
        const int at = tid + i * 256, t = at / p.W, k = at - t * p.W;
        mask_regs[i] = t < nodes ? node_word(p, y.b, t, k, nodes) : 0u;
      }
    };
    constexpr bool kFetchAhead = Sh::kFetchAhead;
    static_assert(!kFetchAhead || kQLoads <= 8, "registers");
    int now = 0;                                     // this piece's place in sh.piece, and the next one's
    auto behind = [&]() { return now + 1 == Sh::kPieces ? 0 : now + 1; };
    // the fetched piece's masks and Q to shared memory, and the word to the chains that have tiles in it: no other waits for it
    auto hand_over = [&](const Piece& y, typename Shm::PerPiece& to) {
#pragma unroll
      for (int i = 0; i < kMaskLoads; ++i) {
        const int at = tid + i * 256, t = at / p.W;
        if (t < p.T) to.node_mask[t][at - t * p.W] = mask_regs[i];
      }
      if (tid == 0) to.odd_values = 0;
      uint8_t* q_dst = q_smem + (kPair ? w * kTileBytes : 0) + (q_c >> 3) * kChunkBytes;
#pragma unroll
      for (int i = 0; i < kQLoads; ++i) {
        const int row = q_r + i * kQRows;            // and the same row of every copy: kCopyRows keeps row % 8
#pragma unroll
        for (int k = 0; k < kCopies; ++k)
          *reinterpret_cast<uint4*>(q_dst + (row + k * kCopyRows) * 128 + (((q_c & 7) ^ (row & 7)) << 4)) = q_regs[i];
      }
      fence_async_proxy();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(smem_u32(&sh.q_ready[0]));
        if (kPair || y.tiles > 1) mbar_arrive(smem_u32(&sh.q_ready[1]));
      }
    };
    Piece x = next_piece();
    if (x.tiles > 0) {
      fetch(x);
      hand_over(x, sh.piece[0]);
    }
    while (x.tiles > 0) {
      const SeqExtent ex = sh.extents[x.b];
      typename Shm::PerPiece& mine = sh.piece[now];
      float m = -INFINITY, l = 0.f;
      int done = 0;                                  // tiles of this piece that this warpgroup has taken
      for (int t = kPair ? 0 : w; t < x.tiles; t += kPair ? 1 : 2, ++done) {
        const int kv0 = (x.tile0 + t) * kTile;
        const bool tail = kv0 + kTile > ex.ctx;      // holds nodes, or ends behind the sequence
        wait(smem_u32(&sh.s_full[w]), s_phase, abort_flag);
        s_phase ^= 1u;
        // V rows that are no tokens may hold anything: 0 x NaN would reach every row. They become zeroes; and so do values of nodes
        // that are not finite, which the rows that see them get back at the end. (Chain 1's products of a tile are issued behind chain 0's.)
        // Behind the wait for S, because only then has the slot's last content been used up: waiting for V any earlier could take
        // that content's phase for this one's, and zeroes would go into a tile that is still to be multiplied.
        if (tail && (!kPair || w == 0)) {
          const int item = 2 * (tile_count + t) + 1;
          wait(smem_u32(&sh.full[item % kStages]), (uint32_t)(item / kStages) & 1u, abort_flag);
          uint8_t* v = ring + (item % kStages) * kTileBytes;
          const int first = max(0, ex.ctx - kv0), valid = min(kTile, max(0, ex.kv_end - kv0));
          for (int i = first * kVecs + r; i < kTile * kVecs; i += 128) {
            const int row = i / kVecs, c = i - row * kVecs;
            uint4* at = reinterpret_cast<uint4*>(v + (c >> 3) * kChunkBytes + row * 128 + (((c & 7) ^ (row & 7)) << 4));
            if (row >= valid) { *at = make_uint4(0u, 0u, 0u, 0u); continue; }
            uint4 y = *at;
            uint32_t* e = &y.x;
            bool odd = false;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              if ((e[k] & 0x7F80u) == 0x7F80u) { e[k] &= 0xFFFF0000u; odd = true; }
              if ((e[k] & 0x7F800000u) == 0x7F800000u) { e[k] &= 0xFFFFu; odd = true; }
            }
            if (odd) { *at = y; mine.odd_values = 1; }
          }
          fence_async_proxy();
        }
        if (warp_live) {
          tc_fence_after();
          uint32_t s[kCols];
#pragma unroll
          for (int k = 0; k < kCols; k += 32) ld32_issue(t_s + col0 + k, s + k);
          ld_wait();
#pragma unroll
          for (int k = 0; k < kCols; k += 32) pin32(s + k);
          if constexpr (kCopies > 1) {               // the other copies' columns of P
            const uint32_t zero[16] = {};
#pragma unroll
            for (int k = 0; k < (kTile - kCols) / 2; k += 16) st16(t_s + ((col0 / 2 + kCols / 2 + k) & (kTile / 2 - 1)), zero);
          }
          if (tail) {
#pragma unroll
            for (int k = 0; k < kCols; k += 32) {
              const int at = kv0 + col0 + k, off = at - ex.ctx, word = off >> 5, valid = ex.kv_end - at;
              auto bits_of = [&](int i) { return i < 0 ? 0xFFFFFFFFu : (i < p.W && t_node < p.T ? mine.node_mask[t_node][i] : 0u); };
              uint32_t see = __funnelshift_r(bits_of(word), bits_of(word + 1), off & 31);
              if (valid < 32) see &= valid <= 0 ? 0u : (1u << valid) - 1u;
#pragma unroll
              for (int i = 0; i < 32; ++i)
                if (!((see >> i) & 1u)) s[k + i] = 0xFF800000u;   // -inf
            }
          }
          float mx[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) mx[k] = __uint_as_float(s[k]);
#pragma unroll
          for (int i = 4; i < kCols - 4; i += 8)
#pragma unroll
            for (int k = 0; k < 4; ++k) mx[k] = max3(mx[k], __uint_as_float(s[i + k]), __uint_as_float(s[i + 4 + k]));
#pragma unroll
          for (int k = 0; k < 4; ++k) mx[k] = fmaxf(mx[k], __uint_as_float(s[kCols - 4 + k]));
          const float top = fmaxf(max3(mx[0], mx[1], mx[2]), mx[3]);
          // a row that has seen nothing yet has O = 0 and l = 0: its maximum may jump without a rescale
          const bool grow = top > m && (m == -INFINITY || (top - m) * c2 > kLazy);
          const float m_new = grow ? top : m;
          const bool rescale = grow && m != -INFINITY;
          if (__any_sync(0xffffffffu, rescale) && done > 0) {
            const float f = rescale ? fast_exp2((m - m_new) * c2) : 1.f;
            wait(smem_u32(&sh.o_done[w]), o_phase ^ 1u, abort_flag);   // the last product has been added
            tc_fence_after();
#pragma unroll 1
            for (int c = 0; c < D; c += 32) {
              uint32_t o[32];
              ld32_issue(t_o + c, o);
              ld_wait();
              pin32(o);
#pragma unroll
              for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
              st32(t_o + c, o);
            }
            l *= f;
          }
          m = m_new;
          float base = m == -INFINITY ? 0.f : m * c2;
          uint64_t c2_2 = pack2(c2, c2);
          const bool far = fabsf(base) >= kFar;
          if (__any_sync(0xffffffffu, far)) {
            const float c2_row = far ? c2_far : c2;
            base = m == -INFINITY ? 0.f : m * c2_row;
            c2_2 = pack2(c2_row, c2_row);
          }
          const uint64_t base_2 = pack2(-base, -base);
          uint64_t sum[2] = {0ull, 0ull};
#pragma unroll
          for (int k = 0; k < kCols / 32; ++k) {
            uint32_t pk[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              float a, b;
              unpack2(fma2(pack2(__uint_as_float(s[32 * k + 2 * i]), __uint_as_float(s[32 * k + 2 * i + 1])), c2_2, base_2), a, b);
              a = fast_exp2(a);
              b = fast_exp2(b);
              sum[i & 1] = add2(sum[i & 1], pack2(a, b));
              pk[i] = pack_bf16(a, b);
            }
            st16(t_s + col0 / 2 + k * 16, pk);
            if (kCopies == 1 && k == 1) {   // the first half may go
              st_wait();
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(smem_u32(&sh.p_ready[w][0]));
            }
          }
          float l0, l1;
          unpack2(add2(sum[0], sum[1]), l0, l1);
          l += l0 + l1;
          st_wait();
          tc_fence_before();
        }
        __syncwarp();
        if (lane == 0) {
          if (kCopies > 1 || !warp_live) mbar_arrive(smem_u32(&sh.p_ready[w][0]));
          mbar_arrive(smem_u32(&sh.p_ready[w][1]));
        }
        o_phase ^= 1u;
      }
      // ---------------------------------------------------------------- the piece's end
      const Piece next = next_piece();
      if (kFetchAhead) fetch(next);
      if (done > 0) wait(smem_u32(&sh.o_done[w]), o_phase ^ 1u, abort_flag);
      tc_fence_after();
      const bool whole = x.tiles == x.all;
      if (!whole && x.tile0 == 0 && rb == 0 && tid == 0) split_set(p, g, units, x);
      const bool live = my_row < p.rows && t_node < ex.nodes;
      float f0 = 1.f, f1 = 0.f;                      // factors on this lane's O_0 and O_1 (pair mode: on its own O)
      if constexpr (!kPair) {
        mine.ml[w][r][0] = m;
        mine.ml[w][r][1] = l;
      }
      // Every product of this piece has ended: the next one's Q takes its place, and its S runs while this one is written out. Its
      // P V waits for the softmax of these same warps, so O stays until they have read it. (With every tile for both chains a
      // warpgroup's Q and O are its own, and neither waits for the other; with alternate tiles both read both.)
      if constexpr (!kPair) {
        tc_fence_before();
        softmax_sync();
        tc_fence_after();
      }
      if (kFetchAhead && next.tiles > 0) hand_over(next, sh.piece[behind()]);
      if constexpr (!kPair) {
        const float m0 = mine.ml[0][r][0], m1 = mine.ml[1][r][0];
        m = -INFINITY;
#pragma unroll
        for (int i = 0; i < 2 * kCopies; ++i) m = fmaxf(m, mine.ml[i & 1][(i >> 1) * kCopyRows + r % kCopyRows][0]);
        const float base = m == -INFINITY ? 0.f : m;
        f0 = m0 == -INFINITY ? 0.f : fast_exp2((m0 - base) * c2);
        f1 = m1 == -INFINITY ? 0.f : fast_exp2((m1 - base) * c2);
        l = 0.f;
#pragma unroll
        for (int i = 0; i < 2 * kCopies; ++i) {
          const float* ml = mine.ml[i & 1][(i >> 1) * kCopyRows + r % kCopyRows];
          l += (ml[0] == -INFINITY ? 0.f : fast_exp2((ml[0] - base) * c2)) * ml[1];
        }
        if (kCopies > 1 && copy == 0) mine.inv[w][r] = l == 0.f ? 0.f : 1.f / l;   // each warpgroup its own
      }
      const bool two = !kPair && x.tiles > 1;
      const float inv = !whole ? 1.f : (l == 0.f ? 0.f : 1.f / l);
      const bool odd = *reinterpret_cast<volatile int*>(&mine.odd_values) != 0;
      float* part0 = p.part + (((int64_t)blockIdx.x * 2 + (x.tile0 == 0 ? 1 : 0)) * p.part_rows - r0) * (D + kPartPad);
      // kN elements of a query row from column c: back to a part, or out. With copies, an element that is no number while the row's
      // sum is one has met an infinity of V: one copy's weight makes it that infinity, the others' zeroes make it NaN.
      auto write = [&](auto count, int row, int c, float* o, float factor, bool sum_ok) {
        constexpr int kN = decltype(count)::value;
        const int t = row / p.group, h = x.head * p.group + row - t * p.group;
        if (row >= p.rows || t >= ex.nodes) return;
        bool lost = false;
        if constexpr (kCopies > 1) {
#pragma unroll
          for (int i = 0; i < kN; ++i) lost |= isnan(o[i]);
          lost &= sum_ok;
        }
        if (odd || lost) {
          // What is finite does not count beside what is not.
          float sum[kN] = {};
          if (odd) {                                 // values of this piece's nodes that are not finite, to the rows that see them
            for (int j = 0; j < ex.nodes; ++j) {
              const int kv = ex.ctx + j;
              if (kv < x.tile0 * kTile || kv >= (x.tile0 + x.tiles) * kTile || kv >= ex.kv_end || !((mine.node_mask[t][j >> 5] >> (j & 31)) & 1u)) continue;
              const int page = p.c.table[(int64_t)ex.slot * p.c.max_pages + (kv >> p.c.page_shift)];
              if (page < 0 || page >= p.c.pages) continue;
              const __nv_bfloat16* v = reinterpret_cast<const __nv_bfloat16*>(p.c.v) + page_row(p.c, p.layer, page, x.head, kv & (p.c.page_size - 1)) * D + c;
#pragma unroll
              for (int i = 0; i < kN; ++i) {
                const float y = __bfloat162float(v[i]);
                if (!isfinite(y)) sum[i] += y;
              }
            }
          }
          if constexpr (kCopies > 1) {
            if (lost) {
              const float4 y = spoilt_by_context<D>(p, ex.slot, x.head, x.tile0 * kTile, min((x.tile0 + x.tiles) * kTile, ex.ctx), c);
              const float of[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
              for (int i = 0; i < kN; ++i)
                if (isnan(o[i]) && of[i] != 0.f) o[i] = of[i];
            }
          }
#pragma unroll
          for (int i = 0; i < kN; ++i)
            if (sum[i] != 0.f) o[i] += sum[i];
        }
        if (whole) {
          uint2* out = reinterpret_cast<uint2*>(p.out + ((int64_t)x.b * p.T + t) * p.out_stride + ((int64_t)h * D + c) * 2);
#pragma unroll
          for (int i = 0; i < kN; i += 4) out[i / 4] = make_uint2(pack_bf16(o[i] * factor, o[i + 1] * factor), pack_bf16(o[i + 2] * factor, o[i + 3] * factor));
        } else {
          float4* part = reinterpret_cast<float4*>(part0 + (int64_t)row * (D + kPartPad) + c);
#pragma unroll
          for (int i = 0; i < kN; i += 4) part[i / 4] = make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]);
        }
      };
      // this lane's sum of the two chains, 16 columns
      auto read_o = [&](int c, float* o) {
        uint32_t a[16], b[16];
        tmem_ld16_issue((kPair ? t_o : tmem + lanes + 256) + c, a);
        if (two) tmem_ld16_issue(tmem + lanes + 384 + c, b);
        ld_wait();
        pin16(a);
        if (two) pin16(b);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          o[i] = kPair ? __uint_as_float(a[i]) : (f0 == 0.f ? 0.f : __uint_as_float(a[i]) * f0);
          if (two && f1 != 0.f) o[i] = fmaf(__uint_as_float(b[i]), f1, o[i]);
        }
      };
      if constexpr (kCopies == 1) {
        if (warp_live) {
          // alternate tiles: the two warpgroups write half of the columns each
          const int c_begin = kPair ? 0 : w * (D / 2), c_end = kPair ? D : c_begin + D / 2;
#pragma unroll 1
          for (int c = c_begin; c < c_end; c += 16) {
            float o[16];
            read_o(c, o);
            write(std::integral_constant<int, 16>(), my_row, c, o, inv, true);
          }
        }
      } else {
        // The copies' sums meet in shared memory: a quarter of the columns at a time, alternately
        // by warpgroup. A row's 16-byte places are turned by its number, so that neighbouring rows do not meet in a bank.
        constexpr int kStageCols = Sh::kStageCols, kPlaces = kStageCols / 4;
        float* stage = reinterpret_cast<float*>(stage_smem) + w * 128 * kStageCols;
        auto place = [&](int at, int k) { return reinterpret_cast<float4*>(stage + at * kStageCols) + ((k + at) & (kPlaces - 1)); };
#pragma unroll 1
        for (int c = kStageCols * w; c < D; c += 2 * kStageCols) {
          if (warp_live) {
#pragma unroll 1
            for (int k = 0; k < kStageCols; k += 16) {
              float o[16];
              read_o(c + k, o);
#pragma unroll
              for (int i = 0; i < 16; i += 4) *place(r, (k + i) / 4) = make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]);
            }
          }
          asm volatile("bar.sync %0, 128;" ::"r"(2 + w) : "memory");
          for (int i = r; i < kCopyRows * kPlaces; i += 128) {
            const int row = i / kPlaces, q = i % kPlaces;
            if (r0 + row >= p.rows) continue;
            float y[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < kCopies; ++k) {
              const float4 v = *place(k * kCopyRows + row, q);
              y[0] += v.x; y[1] += v.y; y[2] += v.z; y[3] += v.w;
            }
            const float by = mine.inv[w][row];
            write(std::integral_constant<int, 4>(), r0 + row, c + q * 4, y, whole ? by : 1.f, !isnan(by));
          }
          asm volatile("bar.sync %0, 128;" ::"r"(2 + w) : "memory");
        }
      }
      if (live && copy == 0 && (kPair || w == 0)) {
        const float m2 = m * c2;
        if (whole) {
          if (p.lse) p.lse[((int64_t)x.b * p.T + t_node) * p.q_heads + x.head * p.group + gq] = l == 0.f ? -INFINITY : (m2 + log2f(l)) * 0.69314718055994531f;
        } else {
          *reinterpret_cast<float2*>(part0 + (int64_t)my_row * (D + kPartPad) + D) = make_float2(m == -INFINITY ? -INFINITY : m2, l);
        }
      }
      tc_fence_before();
      if constexpr (!kPair) softmax_sync();          // both warpgroups have read both chains' O, which the next piece's first products overwrite
      if (!kFetchAhead && next.tiles > 0) {
        fetch(next);
        hand_over(next, sh.piece[behind()]);
      }
      tile_count += x.tiles;
      x = next;
      now = behind();
    }
  }

  __syncthreads();
  if (sh.abort_flag) {   // copies that are under way land before the block goes
    for (int i = 0; i < 64; ++i) __nanosleep(2000);
    __syncthreads();
  }
  if (warp == 9) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  }
}

template <int D, int kMode>
cudaError_t launch(const AttendParams& p, const CUtensorMap& tm_k, const CUtensorMap& tm_v, cudaStream_t st) {
  return launch_chained(attend_sm100_kernel<D, kMode>, dim3((unsigned)(p.groups * p.row_blocks)), dim3(kThreads), attend_smem<D, kMode>(), st, tm_k, tm_v, p);
}
template <int D>
cudaError_t launch_mode(const AttendParams& p, const CUtensorMap& tm_k, const CUtensorMap& tm_v, cudaStream_t st) {
  if (p.rows_per_block > 128) return launch<D, kPairMode>(p, tm_k, tm_v, st);
  if (p.rows > 64) return launch<D, 1>(p, tm_k, tm_v, st);
  return p.rows > 32 ? launch<D, 2>(p, tm_k, tm_v, st) : launch<D, 4>(p, tm_k, tm_v, st);
}
template <int D, int kMode>
bool configure() {
  static_assert(attend_smem<D, kMode>() <= 227 * 1024, "shared memory of an SM");
  return cudaFuncSetAttribute(attend_sm100_kernel<D, kMode>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)attend_smem<D, kMode>()) == cudaSuccess;
}
template <int D>
bool configure_modes() { return configure<D, kPairMode>() && configure<D, 1>() && configure<D, 2>() && configure<D, 4>(); }

}  // namespace

cudaError_t run_attend_tensor(const AttendParams& p, const CUtensorMap& tm_k, const CUtensorMap& tm_v, cudaStream_t st) {
  return p.c.head_dim == 64 ? launch_mode<64>(p, tm_k, tm_v, st) : launch_mode<128>(p, tm_k, tm_v, st);
}

bool attend_configure() { return simt_attend_configure() && configure_modes<64>() && configure_modes<128>(); }

}  // namespace jd
