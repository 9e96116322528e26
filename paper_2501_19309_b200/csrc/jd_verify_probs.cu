// Verification of drafted tokens, chains or trees, against the target's probabilities, from given random numbers (jd_verify_probs).
//
// The walk stands at a node, first the last context token. With w = the target's weights there, W = 1, q = the draft's and Q = 1, its children
// are tried in order: x is accepted where u W q(x) < w(x) Q, and the walk goes on at that child; else
//     w <- max(0, w Q - W q),   W <- sum w,   distinct siblings: q(x) <- 0, Q <- what is left of q.
// (W and Q are what w and q would be divided by.) What is left is 1 - the rejected tokens' q as long as that is half of the row: a row of stored weights adds up to 1 within half
// a step of their type, so Q is off by a step at most. A confident draft leaves less than that rounding: there Q is summed, by the pass that sums w. Where nothing
// is left of either, a sibling leaves w as it is. The products of W and Q on the way would leave float64 behind some 80 siblings of a confident draft: each pair is taken times the
// power of two that brings their product near 1, which rounds nothing, so that a step's sum is what the step itself leaves. Where no child is left the next token is the first whose running sum of w exceeds u W. Only a
// node where something was rejected, and the last one, cost a pass over their rows; all other tests are single entries.
//
// Latency bounds the small calls and the rows' bytes the large ones. A thread-block cluster takes a sequence: the threads of each block fetch the
// entries of all nodes side by side, and a warp walks. A pass gives every warp of the cluster a stretch of the vocabulary, the next loads under way beside the sums;
// another rejection at the node finds its rows in L1. The blocks' sums go into each other's shared memory by stores that count on a barrier there (a
// cluster barrier and its fences take twice as long). The draw narrows down block, warp and part of its stretch by the sums that the pass has left, then step
// and lane. Loops are kept small: code that a block runs once or twice is fetched line by line, and unrolled eight times over it took longer than its work
// (16 trees of 25 drafted tokens, vocabulary 128,256: 40 us, 25 so; 27 with independent siblings, which are rejected more often). 64 chains of 16: 22 us, where the rows' bytes
// take 10; one chain of 8: 11 us, of which the fetches and the first tests take 2, the pass 3, the sums' way through the cluster and the draw 3. 64 registers for two blocks
// spill 16 (float32) to 104 bytes (bfloat16) with distinct siblings, 0 to 76 else.
// A token of 10^-6 is to be told from its neighbour behind 10^5 others, and every launch shape is to find the same one: sums are float64, or, behind up to one rejection,
// pairs of float32 that are off by some 2^-48 (LongSum); a pass whose sum float32 does not hold is taken again in float64.
#include <algorithm>
#include <cmath>

#include "jd_rope.cuh"
#include "jd_sm100_ptx.cuh"

namespace jd {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;   // two blocks on an SM: the next call's can begin while this one's end
constexpr int kParts = 8;                  // of a warp's stretch whose sums are kept for the draw
constexpr int kMaxCluster = 8;             // the largest that every launch may have

struct ProbsParams {
  int B, T, V, range, part;                // entries of a warp and of a part of them, whole pairs of steps
  const void *target, *draft;
  int64_t target_stride, draft_stride;     // elements between rows
  const int32_t *tokens, *parents, *num_nodes;
  int64_t parents_stride;                  // 0: shared
  const float *accept_u, *sample_u, *judge;
  float tau;
  int mode, resample, distinct;            // distinct: never of chains, whose nodes have one child
  int32_t *accept_len, *next_token, *path;
  unsigned* status;
};

template <typename T> constexpr int kWide = 16 / sizeof(T);   // entries of a lane and step

// A lane's entries of a step, as they lie in memory; zeroes behind the row's end.
template <typename T, bool kVec>
__device__ __forceinline__ uint4 load_entries(const T* row, int v, int end) {
  constexpr int kW = kWide<T>;
  if constexpr (kVec) {                    // the end is a multiple of kW
    return v < end ? *reinterpret_cast<const uint4*>(row + v) : make_uint4(0u, 0u, 0u, 0u);
  } else {
    uint32_t w[4] = {};
#pragma unroll
    for (int e = 0; e < kW; ++e) {
      if (v + e >= end) continue;
      if constexpr (sizeof(T) == 4) w[e] = __float_as_uint(row[v + e]);
      else w[e / 2] |= (uint32_t)__bfloat16_as_ushort(row[v + e]) << (16 * (e & 1));
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
}
template <typename T> __device__ __forceinline__ float entry(const uint4& r, int e) {
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
  if constexpr (sizeof(T) == 4) return __uint_as_float(w[e]);
  else return __uint_as_float((e & 1) ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
}

struct Rejections {                        // of the node that the walk stands at
  double W[kMaxNodes], Q[kMaxNodes];       // in front of each, times a power of two
  int x[kMaxNodes];                        // distinct siblings: the token; -1: none
};
// 2^-e of x = m 2^e, m from 1 to 2
__device__ __forceinline__ double to_one(double x) { return __hiloint2double(0x7FE00000 - (__double2hiint(x) & 0x7FF00000), 0); }
__device__ __forceinline__ double positive(double x) { return x > 0.0 ? x : 0.0; }
// w Q - W q, both products rounded alike: of the last token that is left of either nothing stays.
__device__ __forceinline__ double less(double w, double Q, double W, double q) { return positive(__dsub_rn(__dmul_rn(w, Q), __dmul_rn(W, q))); }
// What is left of the lane's entries v .. after n rejections; d: of the draft's, the last rejected token among them still.
template <typename T, int kW>
__device__ __forceinline__ void weights_of(const Rejections& r, bool distinct, int n, const uint4& x, const uint4& y, int v, double* w, double* d) {
#pragma unroll
  for (int e = 0; e < kW; ++e) {
    d[e] = entry<T>(y, e);
    w[e] = positive((double)entry<T>(x, e) - (n > 0 ? d[e] : 0.0));      // W = Q = 1
  }
#pragma unroll 1
  for (int j = 1; j < n; ++j) {
    const double W = r.W[j], Q = r.Q[j];
    const int gone = distinct ? r.x[j - 1] - v : -1;
#pragma unroll
    for (int e = 0; e < kW; ++e) {
      if (gone == e) d[e] = 0.0;
      w[e] = less(w[e], Q, W, d[e]);
    }
  }
}

// A sum of max(0, p - q) that loses nothing to speak of without float64, whose conversions and additions take five times as long as the rest of a pass. With
// q' = min(p, q) the difference is d + e exactly, d = p - q' rounded and e = (p - d) - q' (Dekker); and s + d is t + f exactly, t rounded and f from six
// operations (Knuth). The small parts go into a float32 sum of their own, which is off by 2^-48 of the sum for every entry; in the
// end both become float64. Two entries at a time.
struct LongSum {
  uint64_t s = 0ull, low = 0ull;
  __device__ __forceinline__ void add(uint64_t p, uint64_t q) {
    const uint64_t one = pack2(-1.f, -1.f);
    float p0, p1, q0, q1;
    unpack2(p, p0, p1);
    unpack2(q, q0, q1);
    q = pack2(fminf(p0, q0), fminf(p1, q1));
    const uint64_t d = fma2(q, one, p), t = add2(s, d), b = fma2(s, one, t);
    low = add2(low, fma2(q, one, fma2(d, one, p)));
    low = add2(low, add2(fma2(fma2(b, one, t), one, s), fma2(b, one, d)));
    s = t;
  }
  __device__ __forceinline__ double take() {
    float s0, s1, l0, l1;
    unpack2(s, s0, s1);
    unpack2(low, l0, l1);
    return ((double)s0 + (double)s1) + ((double)l0 + (double)l1);
  }
};

// An address of this block's shared memory in block `rank` of the cluster.
__device__ __forceinline__ uint32_t in_block(uint32_t addr, int rank) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
// 8 bytes to another block, counted on the barrier there.
__device__ __forceinline__ void send(uint32_t to, double v, uint32_t barrier) {
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.b64 [%0], %1, [%2];" ::"r"(to), "l"(__double_as_longlong(v)), "r"(barrier) : "memory");
}
__device__ __forceinline__ bool wait_cluster(uint32_t barrier, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok) : "r"(barrier), "r"(parity) : "memory");
  return ok != 0;
}

// Where the walk stands: in shared memory between passes, since registers that warp 0 alone needs are every warp's.
struct WalkState {
  int cur, last, len, rejected;
  bool ended, drawing, lost;               // no child left; the weights of the draw have been summed; a block's sum did not come
  bool sum_left, wide;                     // Q is summed; float32 has not held a sum
  double W, Q, total;
};

// Among the lanes' masses, in order: the one in which a running sum passes the goal, the last with mass if none does (-1: there is no mass); and what of the
// goal is left there.
struct Found {
  int who;
  bool passed;
  double left;
};
template <int kLanes>
__device__ __forceinline__ Found find(double m, double goal, int lane) {
  if (lane >= kLanes) m = 0.0;
  double run = m;
#pragma unroll
  for (int o = 1; o < kLanes; o <<= 1) {
    const double z = __shfl_up_sync(0xffffffffu, run, o);
    if (lane >= o) run += z;
  }
  const unsigned behind = __ballot_sync(0xffffffffu, run > goal && m > 0.0), some = __ballot_sync(0xffffffffu, m > 0.0);   // lanes behind kLanes have no mass
  Found f;
  f.passed = behind != 0;
  f.who = behind ? __ffs(behind) - 1 : (some ? 31 - __clz(some) : -1);
  const double before = __shfl_up_sync(0xffffffffu, run, 1);
  f.left = goal - __shfl_sync(0xffffffffu, lane > 0 ? before : 0.0, max(f.who, 0));
  return f;
}

// kDistinct apart: what is left of the draft's row costs calls that have no use for it 0.3 (chains) to 3 us (16 trees of 25), by its code and registers alone.
template <typename T, bool kVec, bool kDistinct>
__global__ void __launch_bounds__(kThreads, 2) verify_probs_kernel(const __grid_constant__ ProbsParams p) {
  constexpr int kW = kWide<T>, kStep = 32 * kW;        // entries of a lane and of a warp at a time
  __shared__ int s_token[kMaxNodes], s_path[kMaxNodes], s_parent[kMaxNodes];
  __shared__ float s_u[kMaxNodes], s_p[kMaxNodes], s_q[kMaxNodes];
  __shared__ uint8_t s_judge[kMaxNodes], s_first[kMaxNodes];      // by the judge; as a first child
  __shared__ Rejections s_rej;
  __shared__ WalkState s_walk;
  __shared__ double s_warp[kWarps], s_left[kWarps], s_part[kWarps][kParts], s_step[kWarps], s_goal;
  __shared__ __align__(8) double s_block[2][kMaxCluster], s_block_left[2][kMaxCluster];
  __shared__ __align__(8) uint64_t s_arrived[2];
  __shared__ int s_pass, s_at, s_begin;    // s_pass: weights after that many rejections are to be summed; < 0: the draw; < -1: given up
  int rank, blocks;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(blocks));
  const int b = blockIdx.x / blocks, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_wait();
  pdl_trigger();
  const int T_ = p.T, nodes = p.num_nodes ? min(max(__ldcg(p.num_nodes + b), 0), T_) : T_;
  if (nodes == 0) return;                  // the whole cluster
  if (tid == 0) {
    mbar_init(smem_u32(&s_arrived[0]), 1);
    mbar_init(smem_u32(&s_arrived[1]), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");   // waited for in front of the first word to another block
  const T* target = reinterpret_cast<const T*>(p.target) + (int64_t)b * T_ * p.target_stride;
  const T* draft = reinterpret_cast<const T*>(p.draft) + (int64_t)b * (T_ - 1) * p.draft_stride;

  if (tid < kMaxNodes) {
    int x = -1, parent = -1;
    if (tid > 0 && tid < nodes) {
      const int64_t at = (int64_t)b * (T_ - 1) + tid - 1;
      x = __ldcg(p.tokens + at);
      parent = p.parents ? __ldcg(p.parents + (int64_t)b * p.parents_stride + tid) : tid - 1;
      const float u = __ldcg(p.accept_u + at);
      const bool judge = p.mode != JD_MODE_STANDARD && __ldcg(p.judge + at) > p.tau;
      const bool in = x >= 0 && x < p.V, child = parent >= 0 && parent < tid;
      const float w = in && child ? to_float(target[parent * p.target_stride + x]) : 0.f;
      const float d = in && child ? to_float(draft[parent * p.draft_stride + x]) : 0.f;
      if (rank == 0 && p.status) {
        if (!in) set_status(p.status, JD_ERR_BAD_TOKEN);
        if (!child) set_status(p.status, JD_ERR_BAD_INDEX);
      }
      if (!in) x = -1;
      if (!child) parent = -1;
      s_u[tid] = u;
      s_p[tid] = w;
      s_q[tid] = d;
      s_judge[tid] = judge;
      s_first[tid] = in && ((p.mode != JD_MODE_JUDGE && (double)u * (double)d < (double)w) || judge);   // W = Q = 1
    }
    s_token[tid] = x;
    s_parent[tid] = parent;
  }
  if (tid == 0) s_walk = WalkState{0, 0, 0, 0, false, false, false, false, false, 1.0, 1.0, 0.0};
  __syncthreads();

  const int v0 = (rank * kWarps + warp) * p.range, v1 = min(v0 + p.range, p.V);   // this warp's stretch
  for (int pass = 0;; ++pass) {
    if (warp == 0) {                       // the walk goes on, alike in all lanes; every block's takes the same steps
      WalkState x = s_walk;
      int want = -1;
      if (!x.wide && !(x.W < INFINITY)) {  // the same pass again, in float64
        x.wide = true;
        want = x.rejected;
      } else if (!x.ended && !p.parents && pass == 0) {   // a chain: up to its first rejection at once
        int stop = nodes;
#pragma unroll 1
        for (int k = (nodes - 1) >> 5; k >= 0; --k) {
          const int i = lane + 32 * k;
          const unsigned no = __ballot_sync(0xffffffffu, i > 0 && i < nodes && !s_first[i < nodes ? i : 0]);
          if (no) stop = 32 * k + __ffs(no) - 1;
          if (i > 0 && i < nodes) s_path[i - 1] = i;
        }
        x.cur = x.len = stop - 1;
        x.last = kMaxNodes;                // no other child
        x.ended = stop == nodes;
        x.rejected = x.ended ? 0 : 1;
        want = x.rejected;
        if (lane == 0 && !x.ended) { s_rej.W[0] = s_rej.Q[0] = 1.0; s_rej.x[0] = s_token[stop]; }
      } else if (!x.ended) {
        x.ended = true;
        int parents[kMaxNodes / 32];       // of nodes lane, lane + 32, ..
#pragma unroll
        for (int k = 0; k < kMaxNodes / 32; ++k) parents[k] = s_parent[lane + 32 * k];
#pragma unroll 1
        for (;;) {
          int next = -1;                   // the lowest child behind the last one
#pragma unroll
          for (int k = kMaxNodes / 32 - 1; k >= 0; --k) {
            const unsigned hit = __ballot_sync(0xffffffffu, parents[k] == x.cur && lane + 32 * k > x.last);
            if (hit) next = 32 * k + __ffs(hit) - 1;
          }
          if (next < 0) break;
          x.last = next;
          bool ok = s_first[next] != 0;
          double d = s_q[next];
          const int token = s_token[next];
          if (x.rejected > 0) {
            double w = s_p[next];
#pragma unroll 1
            for (int j = 0; j < x.rejected; ++j) {
              w = less(w, s_rej.Q[j], s_rej.W[j], d);
              if (kDistinct && token == s_rej.x[j]) d = 0.0;
            }
            ok = token >= 0 && ((p.mode != JD_MODE_JUDGE && (double)s_u[next] * x.W * d < w * x.Q) || s_judge[next]);
          }
          if (ok) {
            if (lane == 0) s_path[x.len] = next;
            ++x.len;
            x.cur = next;
            x.W = x.Q = 1.0;
            x.rejected = 0;
            x.sum_left = false;
            continue;
          }
          if (!(x.W > 0.0 && x.Q > 0.0)) continue;     // nothing to take, or to take from
          __syncwarp();
          if (lane == 0) {
            const double f = to_one(x.W) * to_one(x.Q);
            s_rej.W[x.rejected] = x.W * f;
            s_rej.Q[x.rejected] = x.Q * f;
            s_rej.x[x.rejected] = token;
          }
          want = ++x.rejected;
          if (kDistinct) {
            x.Q -= d;
            x.sum_left |= x.Q < 0.5;
          }
          x.ended = false;
          break;
        }
        if (x.ended) {                     // what the draw goes by: the rest after the last rejection, summed already, or the target's own weights
          const bool rest = x.rejected > 0 && x.W > 0.0 && p.resample == JD_RESAMPLE_RESIDUAL;
          if (rest) x.drawing = true;
          else { x.rejected = 0; want = 0; x.sum_left = false; }
        }
      } else {
        x.drawing = true;
      }
      x.total = x.W;
      __syncwarp();
      if (lane == 0) {
        s_walk = x;
        s_pass = x.lost ? -2 : (x.drawing ? -1 : want);
      }
    }
    __syncthreads();
    const int n = s_pass;
    if (n < 0) break;
    // ---- a pass: sums of what is left of the node's row
    const int node = s_walk.cur;
    const T* prow = target + node * p.target_stride;
    const T* qrow = draft + node * p.draft_stride;
    const bool sum_left = kDistinct && s_walk.sum_left, in_double = n > 1 || sum_left || s_walk.wide;
    double sum = 0.0, left = 0.0;          // of the warp; of the lane
#pragma unroll 1
    for (int w0 = v0, i = 0; w0 < v1; w0 += p.part, ++i) {
      const int w1 = min(w0 + p.part, v1);
      double part = 0.0;
      if (!in_double) {                    // of no rejection: q = 0
        uint4 x[2], y[2];
        auto fetch = [&](int v) {
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const int at = v + k * kStep + lane * kW;
            x[k] = load_entries<T, kVec>(prow, at, w1);
            y[k] = n > 0 ? load_entries<T, kVec>(qrow, at, w1) : make_uint4(0u, 0u, 0u, 0u);
          }
        };
        fetch(w0);
        LongSum two;
#pragma unroll 1
        for (int v = w0; v < w1; v += 2 * kStep) {
          const uint4 a[2] = {x[0], x[1]}, d[2] = {y[0], y[1]};
          fetch(v + 2 * kStep);
#pragma unroll
          for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int e = 0; e < kW; e += 2)
              two.add(pack2(entry<T>(a[k], e), entry<T>(a[k], e + 1)), pack2(entry<T>(d[k], e), entry<T>(d[k], e + 1)));
        }
        part = two.take();
      } else {
        uint4 x = load_entries<T, kVec>(prow, w0 + lane * kW, w1), y = load_entries<T, kVec>(qrow, w0 + lane * kW, w1);
#pragma unroll 1
        for (int v = w0 + lane * kW; v < w1 + lane * kW; v += kStep) {
          const uint4 a = x, d = y;
          x = load_entries<T, kVec>(prow, v + kStep, w1);
          y = load_entries<T, kVec>(qrow, v + kStep, w1);
          double w[kW], of_q[kW];
          weights_of<T, kW>(s_rej, kDistinct, n, a, d, v, w, of_q);
#pragma unroll
          for (int e = 0; e < kW; ++e) part += w[e];
          if (sum_left) {
            const int gone = s_rej.x[n - 1] - v;
#pragma unroll
            for (int e = 0; e < kW; ++e) left += gone == e ? 0.0 : of_q[e];
          }
        }
      }
      part = warp_sum_double(part);
      if (lane == 0) s_part[warp][i] = part;
      sum += part;
    }
    if (sum_left) left = warp_sum_double(left);
    if (lane == 0) { s_warp[warp] = sum; s_left[warp] = left; }
    if (pass == 0) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");   // every block has begun, its barriers are there
    __syncthreads();
    if (warp == 0) {
      // Buffers and barriers in turn: a block sends its sum of the next pass when it has every sum of this one.
      const uint32_t barrier = smem_u32(&s_arrived[pass & 1]);
      if (lane == 0) mbar_expect_tx(barrier, (sum_left ? 16 : 8) * blocks);
      const double s = warp_sum_double(lane < kWarps ? s_warp[lane] : 0.0);
      __syncwarp();
      if (lane < blocks) send(in_block(smem_u32(&s_block[pass & 1][rank]), lane), s, in_block(barrier, lane));
      if (sum_left) {
        const double q = warp_sum_double(lane < kWarps ? s_left[lane] : 0.0);
        if (lane < blocks) send(in_block(smem_u32(&s_block_left[pass & 1][rank]), lane), q, in_block(barrier, lane));
      }
      unsigned it = 0;
      bool lost = false;
      while (!wait_cluster(barrier, (pass >> 1) & 1) && !lost) lost = ++it >= kSpinLimit;
      double all = lane < blocks ? s_block[pass & 1][lane] : 0.0;
#pragma unroll
      for (int o = kMaxCluster / 2; o > 0; o >>= 1) all += __shfl_xor_sync(0xffffffffu, all, o);
      if (sum_left) {
        double rest = lane < blocks ? s_block_left[pass & 1][lane] : 0.0;
#pragma unroll
        for (int o = kMaxCluster / 2; o > 0; o >>= 1) rest += __shfl_xor_sync(0xffffffffu, rest, o);
        if (lane == 0) s_walk.Q = rest;
      }
      if (lane == 0) {
        s_walk.W = all;
        s_walk.lost = lost;
        s_at = pass & 1;
        if (lost && p.status) set_status(p.status, JD_ERR_TIMEOUT);
      }
      __syncwarp();
    }
  }
  if (s_pass < -1) {                       // words that are under way to this block land before it goes
    for (int i = 0; i < 64; ++i) __nanosleep(2000);
    return;
  }
  // ---- the draw: W > 0 unless the row has no mass at all
  const int n = s_walk.rejected, node = s_walk.cur;
  if (rank == 0) {
    if (tid < T_ - 1 && p.path) p.path[(int64_t)b * (T_ - 1) + tid] = tid < s_walk.len ? s_path[tid] : -1;
    if (tid == 0) p.accept_len[b] = s_walk.len;
  }
  // Goal: u times the sum. Rounding apart, a sum in front of the goal and one behind it lie in one block, warp, part, batch and lane; where nothing lies
  // behind (u not below 1, or rounding), the last with mass counts.
  if (warp == 0) {
    const double goal = (double)__ldcg(p.sample_u + b) * s_walk.total;
    const Found block = find<kMaxCluster>(lane < blocks ? s_block[s_at][lane] : 0.0, goal, lane);
    if (block.who < 0 && rank == 0 && lane == 0) p.next_token[b] = p.V - 1;
    const Found owner = find<kWarps>(lane < kWarps ? s_warp[lane] : 0.0, block.left, lane);
    const int from = (rank * kWarps + max(owner.who, 0)) * p.range, parts = (min(from + p.range, p.V) - from + p.part - 1) / p.part;
    const Found part = find<kParts>(lane < min(parts, kParts) ? s_part[max(owner.who, 0)][lane] : 0.0, owner.left, lane);
    __syncwarp();                          // everybody has read s_at
    if (lane == 0) {
      s_at = block.who == rank && owner.who >= 0;
      s_begin = from + max(part.who, 0) * p.part;
      s_goal = part.left;
    }
  }
  __syncthreads();
  if (!s_at) return;
  // the part's steps, one for each warp at a time
  const T* prow = target + node * p.target_stride;
  const T* qrow = draft + node * p.draft_stride;
  const int begin = s_begin, end = min((int)min((int64_t)begin + p.part, (int64_t)(begin / p.range + 1) * p.range), p.V);
  double goal = s_goal, last_goal = goal;
  int found = -1, last_found = begin;
  double w[kW], of_q[kW], of_lane = 0.0;
  int held = -1;                           // the step that this warp has in hand
  auto take_step = [&](int v) {
    const int at = v + lane * kW;
    const uint4 x = load_entries<T, kVec>(prow, at, end), y = n > 0 ? load_entries<T, kVec>(qrow, at, end) : make_uint4(0u, 0u, 0u, 0u);
    weights_of<T, kW>(s_rej, kDistinct, n, x, y, at, w, of_q);
    of_lane = 0.0;
#pragma unroll
    for (int e = 0; e < kW; ++e) of_lane += w[e];
    held = v;
  };
#pragma unroll 1
  for (int v = begin; v < end && found < 0; v += kWarps * kStep) {
    __syncthreads();
    take_step(v + warp * kStep);
    const double all = warp_sum_double(of_lane);
    if (lane == 0) s_step[warp] = all;
    __syncthreads();
    const double of_step = lane < kWarps ? s_step[lane] : 0.0, sum = warp_sum_double(of_step);
    const Found step = find<kWarps>(of_step, goal, lane);
    if (step.who >= 0) {
      last_found = v + step.who * kStep;
      last_goal = step.left;
      if (step.passed) found = last_found;
    }
    goal -= sum;
  }
  found = last_found;                      // where nothing lies behind: the last with mass
  if ((found - begin) / kStep % kWarps != warp) return;
  if (held != found) take_step(found);
  const Found at_lane = find<32>(of_lane, last_goal, lane);
  if (lane != max(at_lane.who, 0)) return;
  const int at = found + lane * kW;
  double in = 0.0;
  int token = -1, last_token = min(at, p.V - 1);
#pragma unroll
  for (int e = 0; e < kW; ++e) {
    in += w[e];
    if (w[e] > 0.0) {
      last_token = at + e;
      if (token < 0 && in > at_lane.left) token = at + e;
    }
  }
  p.next_token[b] = token < 0 ? last_token : token;
}

template <typename T, bool kVec>
cudaError_t launch_probs(const ProbsParams& p, int blocks, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(p.B * blocks));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)blocks;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, p.distinct ? verify_probs_kernel<T, kVec, true> : verify_probs_kernel<T, kVec, false>, p);
}

bool on(const void* p, uintptr_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

}  // namespace
}  // namespace jd

using namespace jd;

extern "C" jd_status_t jd_verify_probs(const jd_verify_probs_args_t* a, void* cuda_stream) {
  if (!a || a->B < 0 || a->B > 65535 || a->nodes < 1 || a->nodes > kMaxNodes || a->V < 1 || a->V > (1 << 28)) return JD_ERR_INVALID_ARG;
  if (a->dtype != JD_DTYPE_F32 && a->dtype != JD_DTYPE_BF16) return JD_ERR_INVALID_ARG;
  if (a->mode < JD_MODE_STANDARD || a->mode > JD_MODE_JUDGE_OR_STANDARD || (a->resample != JD_RESAMPLE_RESIDUAL && a->resample != JD_RESAMPLE_TARGET_P) ||
      (a->siblings != JD_SIBLINGS_INDEPENDENT && a->siblings != JD_SIBLINGS_DISTINCT) || (a->per_seq != 0 && a->per_seq != 1))
    return JD_ERR_INVALID_ARG;
  const bool drafted = a->nodes > 1, judged = drafted && a->mode != JD_MODE_STANDARD;
  if (judged && !(a->tau >= 0.f && a->tau <= 1.f)) return JD_ERR_INVALID_ARG;
  const uintptr_t e = a->dtype == JD_DTYPE_F32 ? 4 : 2;
  const int64_t ts = a->target_stride ? a->target_stride : a->V, ds = a->draft_stride ? a->draft_stride : a->V;
  if (ts < a->V || ds < a->V || ts > ((int64_t)1 << 40) || ds > ((int64_t)1 << 40)) return JD_ERR_INVALID_ARG;
  if (a->B == 0) return JD_OK;
  if (!a->target || !on(a->target, e) || !a->sample_u || !a->accept_len || !a->next_token) return JD_ERR_INVALID_ARG;
  if (drafted && (!a->draft || !on(a->draft, e) || !a->tokens || !a->accept_u || (judged && !a->judge_scores))) return JD_ERR_INVALID_ARG;
  for (const void* x : {(const void*)a->tokens, (const void*)a->parents, (const void*)a->num_nodes, (const void*)a->accept_u, (const void*)a->sample_u,
                        (const void*)a->judge_scores, (const void*)a->accept_len, (const void*)a->next_token, (const void*)a->path, (const void*)a->device_status})
    if (!on(x, 4)) return JD_ERR_INVALID_ARG;
  int device = 0, sms = 0;
  if (cudaGetDevice(&device) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device) != cudaSuccess) {
    cudaGetLastError();
    return JD_ERR_CUDA;
  }
  ProbsParams p;
  p.B = a->B; p.T = a->nodes; p.V = a->V;
  p.target = a->target; p.draft = a->draft; p.target_stride = ts; p.draft_stride = ds;
  p.tokens = a->tokens; p.parents = a->parents; p.num_nodes = a->num_nodes;
  p.parents_stride = a->per_seq ? a->nodes : 0;
  p.accept_u = a->accept_u; p.sample_u = a->sample_u; p.judge = a->judge_scores;
  p.tau = a->tau; p.mode = a->mode; p.resample = a->resample; p.distinct = a->siblings == JD_SIBLINGS_DISTINCT && a->parents;
  p.accept_len = a->accept_len; p.next_token = a->next_token; p.path = a->path;
  p.status = a->device_status;
  // As many blocks for a sequence as keep all sequences on the device at once
  int blocks = kMaxCluster;
  while (blocks > 1 && a->B * blocks > 2 * sms) blocks /= 2;
  const int64_t warps = blocks * kWarps, two = 2 * 32 * 16 / (int64_t)e, pairs = (a->V + warps * two - 1) / (warps * two);
  p.part = (int)(std::max<int64_t>(kWarps / 2, (pairs + kParts - 1) / kParts) * two);   // a step for each warp of the draw, or more
  p.range = (int)(pairs * two);
  const bool vec = on(a->target, 16) && (!drafted || on(a->draft, 16)) && a->V % (16 / (int)e) == 0 && ts * e % 16 == 0 && ds * e % 16 == 0;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  cudaError_t err;
  if (a->dtype == JD_DTYPE_F32) err = vec ? launch_probs<float, true>(p, blocks, st) : launch_probs<float, false>(p, blocks, st);
  else err = vec ? launch_probs<__nv_bfloat16, true>(p, blocks, st) : launch_probs<__nv_bfloat16, false>(p, blocks, st);
  if (err != cudaSuccess) { cudaGetLastError(); return JD_ERR_CUDA; }
  return JD_OK;
}
