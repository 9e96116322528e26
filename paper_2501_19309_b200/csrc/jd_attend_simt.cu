// Attention of a drafted block over the paged cache on CUDA cores: any type and head width, float32 throughout; and the
// kernel that joins the partial results of split sequences, which the tensor-core variant shares.
//
// A CTA takes 16 query rows (4 where there are no more) of a (sequence, kv head) - a row is a node and one of the query
// heads that share the kv head - and walks its run of tiles of 64 cached tokens (jd_cache.h says how runs are cut). Per tile: K and
// V to shared memory, the scores by 256 threads (two tokens, four rows and half of the columns each), running maximum and sum
// by a warp for a row, and the weighted sum of V with every warp taking an eighth of the tokens for all rows and up to 256 columns in
// registers, so that one shared-memory read of V serves all rows. The warps' sums meet once per piece of a segment.
// Two CTAs on an SM, so that one's loads run beside the other's products. float32, B200: 16 sequences of 8,000 tokens, 8 heads of
// 128, one token each: 260 us, 4.0 TB/s; 8 blocks of 26 nodes, 16 heads on 4 of 128 over 2,000 tokens: 200 us, 17 TFLOP/s, of which
// 58 % of the issue slots, 50 % of the shared-memory accesses and 36 % of the FMA pipe: what stays is shared memory's latency (the
// largest stall) and the barriers between a tile's four phases, with 16 warps on an SM.
// bf16 head widths that the tensor-core kernel does not take come here too, far from its rates: 16 sequences of 8,000 tokens, 8 heads, one
// token each, 32 query heads: 352 us for heads of 80, 397 of 96, 1,530 of 256 (one block on an SM), against 91 of 128 there.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "jd_cache.h"
#include "jd_sm100_ptx.cuh"

namespace jd {
namespace {

constexpr int kThreads = 256;
constexpr int kTile = 1 << kSimtTileShift;

template <typename T> __device__ __forceinline__ void load4(const T* p, float* v);
template <> __device__ __forceinline__ void load4<float>(const float* p, float* v) {
  const float4 a = *reinterpret_cast<const float4*>(p);
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
}
template <> __device__ __forceinline__ void load4<__nv_bfloat16>(const __nv_bfloat16* p, float* v) {
  const uint2 a = *reinterpret_cast<const uint2*>(p);
  v[0] = __uint_as_float(a.x << 16); v[1] = __uint_as_float(a.x & 0xFFFF0000u);
  v[2] = __uint_as_float(a.y << 16); v[3] = __uint_as_float(a.y & 0xFFFF0000u);
}
__device__ __forceinline__ void store4(float* p, const float* v) { *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]); }
__device__ __forceinline__ void store4(__nv_bfloat16* p, const float* v) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(v[0], v[1]), b = __floats2bfloat162_rn(v[2], v[3]);
  *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}

// 16 bytes from global to shared memory without a register in between; zeroes if !there (src is then not read, but has to be an address)
__device__ __forceinline__ void copy16_or_zero(float* dst, const void* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(there ? 16 : 0) : "memory");
}

__host__ __device__ constexpr int pitch_of(int head_dim) { return head_dim + 4; }   // floats; keeps 16-byte accesses off one bank group

// floats between tokens of the score buffer: the rows and padding, 16-byte aligned
__host__ __device__ constexpr int score_pad(int rows) { return rows == 4 ? 12 : rows + 4; }
size_t simt_smem(int head_dim, int rows) {
  return sizeof(float) * ((size_t)2 * kTile * pitch_of(head_dim) + rows * pitch_of(head_dim) + (rows == 4 ? 1 : 2) * kTile * score_pad(rows));
}

// kCols: groups of 128 columns that a lane's accumulators cover (head_dim <= 128 kCols)
// kRows: query rows of the block, 4 or 16
template <typename T, int kCols, int kRows, int kShare>
__device__ __forceinline__ void attend_simt(const AttendParams& p, const Division cut) {
  constexpr int kScorePad = score_pad(kRows);
  extern __shared__ __align__(16) float smem[];
  __shared__ int prefix[kMaxCacheBatch + 1], warp_sums[kThreads / 32];
  __shared__ int64_t s_row[kTile];   // elements in front of a token's row of K and V
  __shared__ float s_m[kRows], s_l[kRows], s_fac[kRows];
  __shared__ uint32_t s_mask[kRows][kMaxNodes / 32];
  const int D = p.c.head_dim, pitch = pitch_of(D);
  float* sK = smem;
  float* sV = sK + kTile * pitch;
  float* sQ = sV + kTile * pitch;
  float* sS = sQ + kRows * pitch;
  float* sS1 = sS + kTile * kScorePad;   // 16 rows: the other half of the columns' share
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int g = blockIdx.x / p.row_blocks, rb = blockIdx.x - g * p.row_blocks;
  int r0 = rb * kRows, nrows = min(kRows, p.rows - r0);   // with shared prefixes they move with the piece
  pdl_wait();
  pdl_trigger();
  if (kShare == kAlone && rb == 0 && tid == 0) split_none(p, g);
  unit_prefix(ShareOf<kShare>(), p, cut, prefix, warp_sums);
  const int64_t units = (int64_t)prefix[items_of<kShare>(p)] * p.c.kv_heads;
  if (units == 0) return;
  const int64_t run0 = run_start(units, p.groups, g), run1 = run_start(units, p.groups, g + 1);
  const T* kbase = reinterpret_cast<const T*>(p.c.k);
  const T* vbase = reinterpret_cast<const T*>(p.c.v);

  const int step = kCols == 1 && D <= 64 ? 2 : 1, col_lane = step == 2 ? lane & 15 : lane, my_token = step == 2 ? lane >> 4 : 0;
  for (int64_t u = run0; u < run1;) {
    const Piece x = piece_at<kShare>(p, cut, prefix, u, run1);
    u = x.next;
    if (x.tiles == 0) continue;
    const bool shared_rows = kShare == kShared && x.b < p.max_groups;
    const int b = x.b - (kShare == kShared ? p.max_groups : 0), head = x.head, tiles = x.all, tile0 = x.first + x.tile0, ntiles = x.tiles;
    const Extent<kShare> ex = extent_at<kShare>(p, x.b);
    if constexpr (kShare == kShared) {
      r0 = x.row0;
      nrows = min(kRows, (shared_rows ? ex.nodes : p.rows) - r0);
    }

    __syncthreads();   // the previous segment's buffers are free
    for (int i = tid; i < kRows * (D / 4); i += kThreads) {
      const int r = i / (D / 4), d = (i - r * (D / 4)) * 4;
      float v[4] = {0.f, 0.f, 0.f, 0.f};
      int from = b, row = r0 + r;
      bool there = r < nrows;
      if (shared_rows && there) {                    // whose row it is
        const int m = row / p.rows;
        from = __ldcg(p.sh.member + member0_of(ex) + m);
        row -= m * p.rows;
      }
      const int t = row / p.group, gq = row - t * p.group;
      if (shared_rows) there = there && (!p.num_nodes || t < __ldcg(p.num_nodes + from));
      else there = there && t < ex.nodes;
      if (there)
        load4<T>(reinterpret_cast<const T*>(p.q + ((int64_t)from * p.T + t) * p.q_stride) + (int64_t)(head * p.group + gq) * D + d, v);
#pragma unroll
      for (int k = 0; k < 4; ++k) sQ[r * pitch + d + k] = v[k];
    }
    if (tid < kRows) { s_m[tid] = -INFINITY; s_l[tid] = 0.f; }
    for (int i = tid; !shared_rows && i < kRows * p.W; i += kThreads) {
      const int r = i / p.W, w = i - r * p.W, t = (r0 + r) / p.group;
      s_mask[r][w] = r < nrows && t < ex.nodes ? node_word(p, b, t, w, ex.nodes) : 0u;
    }
    float acc[kRows][4 * kCols];
#pragma unroll
    for (int r = 0; r < kRows; ++r)
#pragma unroll
      for (int k = 0; k < 4 * kCols; ++k) acc[r][k] = 0.f;

    // page of this thread's token of a tile (rows behind the sequence: the last one's), fetched a tile ahead
    auto token_of = [&](int tile) { return tile * kTile + min(tid, max(min(kTile, ex.kv_end - tile * kTile) - 1, 0)); };
    auto page_of = [&](int tile) {
      const int kv = token_of(tile);
      return tid < kTile && kv < ex.kv_end ? __ldcg(p.c.table + (int64_t)ex.slot * p.c.max_pages + (kv >> p.c.page_shift)) : 0;
    };
    int page = page_of(tile0);
    for (int tile = tile0; tile < tile0 + ntiles; ++tile) {
      const int kv0 = tile * kTile, nkv = max(0, min(kTile, ex.kv_end - kv0));
      __syncthreads();   // the previous tile's buffers are free
      if (tid < kTile) {
        if (page < 0 || page >= p.c.pages) { set_status(p.c.status, JD_ERR_BAD_INDEX); page = 0; }
        s_row[tid] = page_row(p.c, p.layer, page, head, token_of(tile) & (p.c.page_size - 1)) * D;
        if (tile + 1 < tile0 + ntiles) page = page_of(tile + 1);
      }
      __syncthreads();
      const int vec = D / 4;
      // i / vec for i < 64 x 64: (2^20 / vec rounded up) x i is off by less than 4096 x 63 < 2^20
      const uint32_t per_vec = ((1u << 20) + vec - 1) / vec;
      if constexpr (sizeof(T) == 4) {              // straight to shared memory; rows behind the sequence may hold anything: zeroes
        for (int i = tid; i < kTile * vec; i += kThreads) {
          const int r = (int)((i * per_vec) >> 20), d = (i - r * vec) * 4;
          const int64_t off = s_row[r] + d;
          copy16_or_zero(sK + r * pitch + d, kbase + off, r < nkv);
          copy16_or_zero(sV + r * pitch + d, vbase + off, r < nkv);
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
      } else {
        constexpr int kAhead = 4;                  // pieces of K and of V whose loads are under way at once
        for (int i0 = tid; i0 < kTile * vec; i0 += kAhead * kThreads) {
          float kx[kAhead][4], vx[kAhead][4];
#pragma unroll
          for (int j = 0; j < kAhead; ++j) {
            const int i = i0 + j * kThreads, r = i / vec, d = (i - r * vec) * 4;
#pragma unroll
            for (int e = 0; e < 4; ++e) kx[j][e] = vx[j][e] = 0.f;
            if (r < nkv) {
              const int64_t off = s_row[r] + d;
              load4<T>(kbase + off, kx[j]);
              load4<T>(vbase + off, vx[j]);
            }
          }
#pragma unroll
          for (int j = 0; j < kAhead; ++j) {
            const int i = i0 + j * kThreads, r = i / vec, d = (i - r * vec) * 4;
            if (i < kTile * vec) {
              store4(sK + r * pitch + d, kx[j]);
              store4(sV + r * pitch + d, vx[j]);
            }
          }
        }
      }
      __syncthreads();
      auto score = [&](float s, int kv, int r) {   // scaled; -inf where row r must not see token kv of the tile
        const int node = kv0 + kv - ex.ctx;        // < 0: context
        return kv < nkv && (node < 0 || ((s_mask[r][node >> 5] >> (node & 31)) & 1u)) ? s * p.scale_log2 : -INFINITY;
      };
      if constexpr (kRows == 4) {   // scores: token tid % 64, row tid / 64
        const int kv = tid & (kTile - 1), r = tid >> kSimtTileShift;
        float s = 0.f;
#pragma unroll 4
        for (int d = 0; d < D; d += 4) {
          const float4 x = *reinterpret_cast<const float4*>(sK + kv * pitch + d);
          const float4 y = *reinterpret_cast<const float4*>(sQ + r * pitch + d);
          s = fmaf(x.x, y.x, fmaf(x.y, y.y, fmaf(x.z, y.z, fmaf(x.w, y.w, s))));
        }
        sS[kv * kScorePad + r] = score(s, kv, r);
      } else {
        // A warp takes 16 tokens, all rows and half of the columns; a lane two tokens and four rows: eight lanes read eight tokens and
        // four read four rows in one shared-memory access each, six of them for 32 products. (A token and four rows a lane read
        // 16 bytes of Q at a time for a whole warp, and the accesses took twice as long as the products.)
        const int t0 = (warp & 3) * 16 + (lane & 7), rl = lane >> 3, half = D / 2, d0 = (warp >> 2) * half;
        float s[2][4] = {};
#pragma unroll 2
        for (int d = d0; d < d0 + half; d += 4) {
          float4 x[2];
#pragma unroll
          for (int j = 0; j < 2; ++j) x[j] = *reinterpret_cast<const float4*>(sK + (t0 + 8 * j) * pitch + d);
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float4 y = *reinterpret_cast<const float4*>(sQ + (4 * r + rl) * pitch + d);
#pragma unroll
            for (int j = 0; j < 2; ++j) s[j][r] = fmaf(x[j].x, y.x, fmaf(x[j].y, y.y, fmaf(x[j].z, y.z, fmaf(x[j].w, y.w, s[j][r]))));
          }
        }
        float* to = warp >> 2 ? sS1 : sS;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r) to[(t0 + 8 * j) * kScorePad + 4 * r + rl] = s[j][r];
      }
      __syncthreads();
      for (int r = warp; r < kRows; r += kThreads / 32) {   // statistics: a row per warp and turn
        float* a = sS + lane * kScorePad + r;
        float* c = sS + (lane + 32) * kScorePad + r;
        float x = *a, y = *c;
        if constexpr (kRows != 4) {
          x = score(x + sS1[lane * kScorePad + r], lane, r);
          y = score(y + sS1[(lane + 32) * kScorePad + r], lane + 32, r);
        }
        float m = fmaxf(x, y);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        const float before = s_m[r], now = fmaxf(before, m);
        const float base = now == -INFINITY ? 0.f : now;   // nothing seen yet: every weight is exp2(-inf) = 0
        const float px = exp2f(x - base), py = exp2f(y - base);
        float l = px + py;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
        *a = px;
        *c = py;
        __syncwarp();
        if (lane == 0) {
          const float fac = exp2f(before - base);
          s_fac[r] = fac;
          s_l[r] = s_l[r] * fac + l;
          s_m[r] = now;
        }
      }
      __syncthreads();
      {   // weighted sum of V: this warp's tokens, all rows, columns 4 lane + 128 j (up to 64 columns: half a warp takes every other
          // token). A row that must not see a token
          // has weight 0 for it, but 0 x inf is not 0: where a token's values are not finite, such rows skip it.
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
          const float f = s_fac[r];
#pragma unroll
          for (int k = 0; k < 4 * kCols; ++k) acc[r][k] *= f;
        }
        auto add_token = [&](int kv, auto check) {
          float w[kRows];
#pragma unroll
          for (int r = 0; r < kRows; r += 4) {
            const float4 x = *reinterpret_cast<const float4*>(sS + kv * kScorePad + r);
            w[r] = x.x; w[r + 1] = x.y; w[r + 2] = x.z; w[r + 3] = x.w;
          }
          const int node = kv0 + kv - ex.ctx;
#pragma unroll
          for (int j = 0; j < kCols; ++j) {
            const int d = col_lane * 4 + 128 * j;
            if (d >= D) continue;
            const float4 x = *reinterpret_cast<const float4*>(sV + kv * pitch + d);
            const bool plain = !decltype(check)::value || node < 0 || (isfinite(x.x) && isfinite(x.y) && isfinite(x.z) && isfinite(x.w));
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
              if (plain || ((s_mask[r][node >> 5] >> (node & 31)) & 1u)) {
                acc[r][4 * j] = fmaf(w[r], x.x, acc[r][4 * j]);
                acc[r][4 * j + 1] = fmaf(w[r], x.y, acc[r][4 * j + 1]);
                acc[r][4 * j + 2] = fmaf(w[r], x.z, acc[r][4 * j + 2]);
                acc[r][4 * j + 3] = fmaf(w[r], x.w, acc[r][4 * j + 3]);
              }
            }
          }
        };
        const int first = warp * (kTile / 8);      // tokens behind the sequence have weight 0 and value 0
        if (kv0 + kTile <= ex.ctx) {               // context alone: every row sees every token
#pragma unroll 2
          for (int i = 0; i < kTile / 8; i += step) add_token(first + i + my_token, std::false_type());
        } else {
          for (int i = 0; i < min(kTile / 8, nkv - first); i += step) add_token(first + i + my_token, std::true_type());
        }
      }
    }

    // the warps' sums meet over the K and V buffers, which hold 8 x kRows x D floats: each its own place, then all added
    __syncthreads();
    if (step == 2) {
#pragma unroll
      for (int r = 0; r < kRows; ++r)
#pragma unroll
        for (int k = 0; k < 4; ++k) acc[r][k] += __shfl_xor_sync(0xffffffffu, acc[r][k], 16);
    }
#pragma unroll
    for (int r = 0; r < kRows; ++r)
#pragma unroll
      for (int j = 0; j < kCols; ++j) {
        const int d = col_lane * 4 + 128 * j;
        if (d < D && my_token == 0) store4(sK + (warp * kRows + r) * D + d, &acc[r][4 * j]);
      }
    __syncthreads();
    const bool whole = ntiles == tiles, begins = x.tile0 == 0;
    const bool direct = whole && (kShare == kAlone || (!shared_rows && x.first == 0));   // nothing to add
    if (kShare == kAlone && !whole && tile0 == 0 && rb == 0 && tid == 0) split_set(p, g, units, x);
    for (int i = tid; i < nrows * (D / 4); i += kThreads) {
      const int r = i / (D / 4), d = (i - r * (D / 4)) * 4;
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kThreads / 32; ++w) {
        const float4 y = *reinterpret_cast<const float4*>(sK + (w * kRows + r) * D + d);
        x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
      }
      if (direct) {
        const int t = (r0 + r) / p.group, gq = (r0 + r) - t * p.group;
        if (t >= ex.nodes) continue;
        const float l = s_l[r], inv = l == 0.f ? 0.f : 1.f / l;
        const float o[4] = {x.x * inv, x.y * inv, x.z * inv, x.w * inv};
        const int h = head * p.group + gq;
        store4(reinterpret_cast<T*>(p.out + ((int64_t)b * p.T + t) * p.out_stride) + (int64_t)h * D + d, o);
        if (d == 0 && p.lse) p.lse[((int64_t)b * p.T + t) * p.q_heads + h] = l == 0.f ? -INFINITY : (s_m[r] + log2f(l)) * 0.69314718055994531f;
      } else {
        float* part = p.part + (((int64_t)blockIdx.x * 2 + (begins ? 1 : 0)) * cut.part_rows + r) * (D + kPartPad);
        if (kShare != kAlone && whole)
          part = (shared_rows ? p.sh.rec_group : p.sh.rec_own) +
                 (((shared_rows ? member0_of(ex) : b) * p.rows + r0 + r) * p.c.kv_heads + head) * (D + kPartPad);
        *reinterpret_cast<float4*>(part + d) = x;
        if (d == 0) { part[D] = s_m[r]; part[D + 1] = s_l[r]; }
      }
    }
  }
}

template <typename T, int kCols, int kRows>
__global__ void __launch_bounds__(kThreads, kCols * kRows <= 16 ? 2 : 1) attend_simt_kernel(AttendParams p) {
  attend_simt<T, kCols, kRows, kAlone>(p, own_division(p));
}
// With a plan that names one of two forms.
template <typename T, int kCols, int kFirst, int kSecond>
__global__ void __launch_bounds__(kThreads, kCols * kSecond <= 16 ? 2 : 1) attend_simt_shared_kernel(const __grid_constant__ AttendParams p) {
  const Division d = plan_division<false>(p);
  if constexpr (kFirst == kSecond) attend_simt<T, kCols, kFirst, kShared>(p, d);
  else if (d.rows_per_block == kSecond) attend_simt<T, kCols, kSecond, kShared>(p, d);
  else attend_simt<T, kCols, kFirst, kShared>(p, d);
}

// Joins the partial results of split segments; rows of whole segments are written already.
// out = sum_i 2^(m_i - m) o_i / sum_i 2^(m_i - m) l_i over the parts in order.
// Block (k, j) takes a few rows of the j-th segment that a group left unfinished: with up to kJoinFewRows rows in all one
// row, whose parts its warps take in turn (what the join costs is their latency, and a row of one long sequence has a part
// from every SM); with more four rows, and a warp for each unless the parts are many. With fewer segments than half the groups there is
// a block for each segment and looks for it: blocks that find nothing to do cost the join more than its loads (16 us against 6 for
// 4 trees x 208 rows with a block for every group). With more there is a block for each group and knows its place (16 trees x 208
// rows: the whole call 73 us, 81 with blocks that look).
constexpr int kJoinWarps = 4, kJoinBatch = 8, kJoinFewRows = 32, kJoinFewParts = 32, kJoinAhead = 5;
__host__ __device__ constexpr int join_rows(int rows) { return rows <= kJoinFewRows ? 1 : kJoinWarps; }

template <int kCols> struct RowSum {   // kCols: groups of 128 columns
  float m, l, o[kCols][4];             // columns 4 lane .. of each group
};

// parts first, first + step, .. last of a row; at(g) is where part g stands
template <int kCols, typename At>
__device__ __forceinline__ RowSum<kCols> sum_parts(int first, int last, int step, int D, int lane, At at) {
  RowSum<kCols> s = {-INFINITY, 0.f, {}};
  const int d = lane * 4;
  for (int g0 = first; g0 <= last; g0 += step * kJoinBatch) {
    float2 ml[kJoinBatch];
    float4 x[kJoinBatch][kCols];
#pragma unroll
    for (int k = 0; k < kJoinBatch; ++k) {
      const int g = g0 + k * step;
      ml[k] = make_float2(-INFINITY, 0.f);
#pragma unroll
      for (int j = 0; j < kCols; ++j) x[k][j] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (g <= last) {
        const float* part = at(g);
        ml[k] = __ldcg(reinterpret_cast<const float2*>(part + D));
#pragma unroll
        for (int j = 0; j < kCols; ++j)
          if (d + 128 * j < D) x[k][j] = __ldcg(reinterpret_cast<const float4*>(part + d + 128 * j));
      }
    }
    float top = s.m;
#pragma unroll
    for (int k = 0; k < kJoinBatch; ++k) top = fmaxf(top, ml[k].x);
    const float base = top == -INFINITY ? 0.f : top, f0 = exp2f(s.m - base);
    s.l *= f0;
#pragma unroll
    for (int j = 0; j < kCols; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) s.o[j][e] *= f0;
#pragma unroll
    for (int k = 0; k < kJoinBatch; ++k) {
      const float f = exp2f(ml[k].x - base);
      s.l += f * ml[k].y;
      if (ml[k].x == -INFINITY) continue;   // a part that saw nothing has no say, whatever it holds
#pragma unroll
      for (int j = 0; j < kCols; ++j) {
        s.o[j][0] = fmaf(f, x[k][j].x, s.o[j][0]); s.o[j][1] = fmaf(f, x[k][j].y, s.o[j][1]);
        s.o[j][2] = fmaf(f, x[k][j].z, s.o[j][2]); s.o[j][3] = fmaf(f, x[k][j].w, s.o[j][3]);
      }
    }
    s.m = top;
  }
  return s;
}

// What a block's warps have summed up, columns 128 j + 4 lane ..
template <int kCols>
__device__ __forceinline__ void add_warps(const float4 (*s_o)[kCols][32], const float2* s_ml, int j, int lane, float* y, float& m, float& l) {
  m = -INFINITY;
#pragma unroll
  for (int w = 0; w < kJoinWarps; ++w) m = fmaxf(m, s_ml[w].x);
  const float base = m == -INFINITY ? 0.f : m;
  l = 0.f;
  y[0] = y[1] = y[2] = y[3] = 0.f;
#pragma unroll
  for (int w = 0; w < kJoinWarps; ++w) {
    const float f = exp2f(s_ml[w].x - base);
    const float4 x = s_o[w][j][lane];
    l += f * s_ml[w].y;
    if (s_ml[w].x == -INFINITY) continue;
    y[0] = fmaf(f, x.x, y[0]); y[1] = fmaf(f, x.y, y[1]); y[2] = fmaf(f, x.z, y[2]); y[3] = fmaf(f, x.w, y[3]);
  }
}

template <typename T, int kCols>
__global__ void __launch_bounds__(32 * kJoinWarps) attend_join_kernel(AttendParams p) {
  __shared__ float4 s_o[kJoinWarps][kCols][32];
  __shared__ float2 s_ml[kJoinWarps];
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int D = p.c.head_dim, pitch = D + kPartPad;
  const int block_rows = join_rows(p.rows), first_row = blockIdx.x * block_rows;
  // this block's segment: the one that group blockIdx.y left unfinished, or number blockIdx.y of all those (there are no more than blocks)
  int b = -1, head = 0, g0 = 0, g1 = 0;
  if ((int)gridDim.y == p.groups) {
    const int4 x = __ldcg(p.split + blockIdx.y);
    b = x.x; head = x.y; g0 = blockIdx.y; g1 = x.z;
  } else for (int base_g = 0, seen = 0; base_g < p.groups && b < 0; base_g += 32 * kJoinAhead) {
    int4 mine[kJoinAhead];
#pragma unroll
    for (int k = 0; k < kJoinAhead; ++k) {
      const int g = base_g + 32 * k + lane;
      mine[k] = g < p.groups ? __ldcg(p.split + g) : make_int4(-1, 0, 0, 0);
    }
#pragma unroll
    for (int k = 0; k < kJoinAhead; ++k) {
      const unsigned left = __ballot_sync(0xffffffffu, mine[k].x >= 0);
      const unsigned hit = __ballot_sync(0xffffffffu, mine[k].x >= 0 && seen + __popc(left & ((1u << lane) - 1u)) == (int)blockIdx.y);
      seen += __popc(left);
      if (hit) {
        const int from = __ffs(hit) - 1;
        b = __shfl_sync(0xffffffffu, mine[k].x, from);
        head = __shfl_sync(0xffffffffu, mine[k].y, from);
        g0 = base_g + 32 * k + from;
        g1 = __shfl_sync(0xffffffffu, mine[k].z, from);
      }
    }
  }
  if (b < 0) return;
  const int nodes = p.num_nodes ? min(max(__ldcg(p.num_nodes + b), 0), p.T) : p.T;
  const int rows = min(p.rows, nodes * p.group);
  auto write = [&](int row, int d, const float* o, float m, float l) {   // columns d .. d + 3
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const float y[4] = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
    const int t = row / p.group, h = head * p.group + row - t * p.group;
    if (d < D) store4(reinterpret_cast<T*>(p.out + ((int64_t)b * p.T + t) * p.out_stride) + (int64_t)h * D + d, y);
    if (d == 0 && p.lse) p.lse[((int64_t)b * p.T + t) * p.q_heads + h] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
  };
  auto place = [&](int row) {
    const int rb = row / p.rows_per_block, r = row - rb * p.rows_per_block;
    const float* base = p.part + ((int64_t)rb * 2 * p.part_rows + r) * pitch;
    return [=](int g) { return base + ((int64_t)g * p.row_blocks * 2 + (g == g0 ? 1 : 0)) * p.part_rows * pitch; };
  };
  if (block_rows > 1 && g1 - g0 < kJoinFewParts) {
    const int row = first_row + warp;
    if (row >= rows) return;
    const RowSum<kCols> s = sum_parts<kCols>(g0, g1, 1, D, lane, place(row));
#pragma unroll
    for (int j = 0; j < kCols; ++j) write(row, 128 * j + lane * 4, s.o[j], s.m, s.l);
    return;
  }
  for (int row = first_row; row < min(rows, first_row + block_rows); ++row) {
    const RowSum<kCols> s = sum_parts<kCols>(g0 + warp, g1, kJoinWarps, D, lane, place(row));
    __syncthreads();   // the last row's sums have been read
#pragma unroll
    for (int j = 0; j < kCols; ++j) s_o[warp][j][lane] = make_float4(s.o[j][0], s.o[j][1], s.o[j][2], s.o[j][3]);
    if (lane == 0) s_ml[warp] = make_float2(s.m, s.l);
    __syncthreads();
    if (warp < kCols) {   // columns 128 warp ..
      float y[4], top, sum;
      add_warps<kCols>(s_o, s_ml, warp, lane, y, top, sum);
      write(row, 128 * warp + lane * 4, y, top, sum);
    }
  }
}

// Adds up what a row's group and the row's sequence have left, parts and records alike. A warp for a row, or, with few rows, whose
// parts from many SMs are what takes the time, a block of four (64 sequences of one token
// and 32 heads: a layer 53 us, 58 with blocks for 2048 rows; 16 sequences 27.7, 28.2 with a warp for each). Rows that are written already (no prefix, one run) are left alone.
constexpr int kSharedFewRows = 512;

struct Parts {                       // of a row in one segment
  int run, count;                    // the first run with tiles of the segment, and their number; 1: a record
};
__device__ __forceinline__ Parts parts_of(const AttendParams& p, const Division& d, int64_t all, int64_t first_unit, int n) {
  Parts x;
  x.run = run_of(all, p.groups, first_unit + d.seg_cost);
  x.count = run_of(all, p.groups, first_unit + n - 1) - x.run + 1;
  return x;
}

template <typename T, int kCols, bool kTensor>
__global__ void __launch_bounds__(32 * kJoinWarps)
attend_shared_join_kernel(AttendParams p, bool few) {
  __shared__ float4 s_o[kJoinWarps][kCols][32];
  __shared__ float2 s_ml[kJoinWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int D = p.c.head_dim, pitch = D + kPartPad;
  const int64_t id = few ? blockIdx.x : (int64_t)blockIdx.x * kJoinWarps + warp;
  if (id >= (int64_t)p.B * p.T * p.q_heads) return;
  const int64_t token = id / p.q_heads;
  const int h = (int)(id - token * p.q_heads), b = (int)(token / p.T), t = (int)(token - (int64_t)b * p.T);
  const int head = h / p.group, row = t * p.group + h - head * p.group;
  pdl_wait();
  pdl_trigger();
  // the loads go out together, whether the row needs them or not
  const Division cut = plan_division<kTensor>(p);
  const int nodes = p.num_nodes ? min(max(__ldcg(p.num_nodes + b), 0), p.T) : p.T;
  const int32_t* units = p.sh.units + p.max_groups + b;
  const int u0 = __ldcg(units), own_units = __ldcg(units + 1) - u0, first = __ldcg(p.sh.first + b), g = __ldcg(p.sh.entry_group + b);
  const int member = __ldcg(p.sh.entry_place + b);
  const int64_t all = (int64_t)__ldcg(p.sh.units + p.max_groups + p.B) * p.c.kv_heads;
  const bool grouped = g >= 0 && g < p.max_groups;
  const int start = grouped ? __ldcg(p.sh.group_start + g) : 0, v0 = grouped ? __ldcg(p.sh.units + g) : 0, group_units = grouped ? __ldcg(p.sh.units + g + 1) - v0 : 0;
  if (t >= nodes || own_units == 0) return;            // own_units == 0: a padding sequence
  const int blocks = row_blocks_of(cut, p.rows), block = row / cut.rows_per_block, n = own_units / blocks;
  const Parts own = parts_of(p, cut, all, (int64_t)u0 * p.c.kv_heads + ((int64_t)head * blocks + block) * n, n);
  if (first == 0 && own.count == 1) return;
  Parts group = {0, 0};
  int64_t group_row = 0;             // among the rows of all groups; in its block
  int group_place = 0;
  if (first > 0 && grouped) {
    const int at = member * p.rows + row, gn = cut.seg_cost + (first >> p.tile_shift), gblocks = group_units / gn;
    const int gblock = at / cut.rows_per_block;
    group_row = (int64_t)start * p.rows + at;
    group_place = at - gblock * cut.rows_per_block;
    group = parts_of(p, cut, all, (int64_t)v0 * p.c.kv_heads + ((int64_t)head * gblocks + gblock) * gn, gn);
  }
  auto at = [&](int i) -> const float* {               // part i: the group's first
    const bool of_group = i < group.count;
    if (!of_group) i -= group.count;
    const Parts x = of_group ? group : own;
    if (x.count == 1) return (of_group ? p.sh.rec_group + (group_row * p.c.kv_heads + head) * pitch : p.sh.rec_own + (((int64_t)b * p.rows + row) * p.c.kv_heads + head) * pitch);
    return p.part + (((int64_t)(x.run + i) * 2 + (i == 0 ? 1 : 0)) * cut.part_rows + (of_group ? group_place : row - block * cut.rows_per_block)) * pitch;
  };
  const int last = group.count + own.count - 1;
  auto write = [&](int d, const float* o, float m, float l) {   // columns d .. d + 3
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const float y[4] = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
    if (d < D) store4(reinterpret_cast<T*>(p.out + token * p.out_stride) + (int64_t)h * D + d, y);
    if (d == 0 && p.lse) p.lse[id] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
  };
  if (!few) {
    const RowSum<kCols> s = sum_parts<kCols>(0, last, 1, D, lane, at);
#pragma unroll
    for (int j = 0; j < kCols; ++j) write(128 * j + lane * 4, s.o[j], s.m, s.l);
    return;
  }
  const RowSum<kCols> s = sum_parts<kCols>(warp, last, kJoinWarps, D, lane, at);
#pragma unroll
  for (int j = 0; j < kCols; ++j) s_o[warp][j][lane] = make_float4(s.o[j][0], s.o[j][1], s.o[j][2], s.o[j][3]);
  if (lane == 0) s_ml[warp] = make_float2(s.m, s.l);
  __syncthreads();
  if (warp < kCols) {
    float y[4], m, l;
    add_warps<kCols>(s_o, s_ml, warp, lane, y, m, l);
    write(128 * warp + lane * 4, y, m, l);
  }
}

template <typename T>
cudaError_t launch_simt(const AttendParams& p, cudaStream_t st) {
  const bool few = p.rows_per_block == 4;
  auto kernel = p.c.head_dim <= 128 ? (few ? attend_simt_kernel<T, 1, 4> : attend_simt_kernel<T, 1, 16>)
                                    : (few ? attend_simt_kernel<T, 2, 4> : attend_simt_kernel<T, 2, 16>);
  return launch_chained(kernel, dim3((unsigned)(p.groups * p.row_blocks)), dim3(kThreads), simt_smem(p.c.head_dim, p.rows_per_block), st, p);
}
// the pairs of shared_forms()
template <typename T>
cudaError_t launch_simt_shared(const AttendParams& p, cudaStream_t st) {
  const bool few = p.rows_per_block == 4, two = p.second_rows != p.rows_per_block;
  auto kernel = p.c.head_dim <= 128 ? (two ? attend_simt_shared_kernel<T, 1, 4, 16> : few ? attend_simt_shared_kernel<T, 1, 4, 4> : attend_simt_shared_kernel<T, 1, 16, 16>)
                                    : (few ? attend_simt_shared_kernel<T, 2, 4, 4> : attend_simt_shared_kernel<T, 2, 16, 16>);
  return launch_chained(kernel, dim3((unsigned)p.groups), dim3(kThreads), simt_smem(p.c.head_dim, std::max(p.rows_per_block, p.second_rows)), st, p);
}

template <typename K>
bool raise_limit(K kernel, size_t bytes) {
  return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) == cudaSuccess;
}

}  // namespace

cudaError_t run_attend_simt(const AttendParams& p, int dtype, cudaStream_t st) {
  return dtype == JD_DTYPE_F32 ? launch_simt<float>(p, st) : launch_simt<__nv_bfloat16>(p, st);
}

cudaError_t run_attend_shared_simt(const AttendParams& p, int dtype, cudaStream_t st) {
  return dtype == JD_DTYPE_F32 ? launch_simt_shared<float>(p, st) : launch_simt_shared<__nv_bfloat16>(p, st);
}

cudaError_t run_attend_join(const AttendParams& p, int dtype, cudaStream_t st) {
  const int n = join_rows(p.rows);
  const int64_t segments = (int64_t)p.B * p.c.kv_heads;
  const dim3 grid((unsigned)((p.rows + n - 1) / n), (unsigned)(2 * segments < p.groups ? segments : p.groups));
  auto kernel = dtype == JD_DTYPE_F32 ? (p.c.head_dim <= 128 ? attend_join_kernel<float, 1> : attend_join_kernel<float, 2>)
                                      : (p.c.head_dim <= 128 ? attend_join_kernel<__nv_bfloat16, 1> : attend_join_kernel<__nv_bfloat16, 2>);
  return launch_chained(kernel, grid, dim3(32 * kJoinWarps), 0, st, p);
}

cudaError_t run_attend_shared_join(const AttendParams& p, int dtype, cudaStream_t st) {
  const int64_t rows = (int64_t)p.B * p.T * p.q_heads;
  const bool few = rows <= kSharedFewRows, tensor = p.tile_shift == kTensorTileShift;
  const dim3 grid((unsigned)(few ? rows : (rows + kJoinWarps - 1) / kJoinWarps));
  auto kernel = dtype == JD_DTYPE_F32 ? (p.c.head_dim <= 128 ? attend_shared_join_kernel<float, 1, false> : attend_shared_join_kernel<float, 2, false>)
                : tensor              ? attend_shared_join_kernel<__nv_bfloat16, 1, true>
                                      : (p.c.head_dim <= 128 ? attend_shared_join_kernel<__nv_bfloat16, 1, false> : attend_shared_join_kernel<__nv_bfloat16, 2, false>);
  return launch_chained(kernel, grid, dim3(32 * kJoinWarps), 0, st, p, few);
}

template <typename T>
bool raise_limits() {
  return raise_limit(attend_simt_kernel<T, 1, 4>, simt_smem(128, 4)) && raise_limit(attend_simt_kernel<T, 1, 16>, simt_smem(128, 16)) &&
         raise_limit(attend_simt_kernel<T, 2, 4>, simt_smem(256, 4)) && raise_limit(attend_simt_kernel<T, 2, 16>, simt_smem(256, 16)) &&
         raise_limit(attend_simt_shared_kernel<T, 1, 4, 4>, simt_smem(128, 4)) && raise_limit(attend_simt_shared_kernel<T, 1, 4, 16>, simt_smem(128, 16)) &&
         raise_limit(attend_simt_shared_kernel<T, 1, 16, 16>, simt_smem(128, 16)) && raise_limit(attend_simt_shared_kernel<T, 2, 4, 4>, simt_smem(256, 4)) &&
         raise_limit(attend_simt_shared_kernel<T, 2, 16, 16>, simt_smem(256, 16));
}
bool simt_attend_configure() { return raise_limits<float>() && raise_limits<__nv_bfloat16>(); }

}  // namespace jd
