// Verification of drafted tokens, chains or trees, against the target's probabilities, from given random numbers (jd_verify_probs).
//
// The walk stands at a node, first the last context token. With w = the target's weights there, W = 1, q = the draft's and Q = 1, its children
// are tried in order: x is accepted where u W q(x) < w(x) Q, and the walk goes on at that child; else
//     w <- max(0, w Q - W q),   W <- sum w,   distinct siblings: q(x) <- 0, Q <- Q - q(x).
// (W and Q are what w and q would be divided by.) Where no child is left the next token is the first whose running sum of w exceeds u W. Only a
// node where something was rejected, and the last one, cost a pass over their rows; all other tests are single entries.
//
// Latency bounds the small calls and the rows' bytes the large ones. A thread-block cluster takes a sequence: the threads of each block fetch the
// entries of all nodes side by side and one thread walks; a pass gives every warp of the cluster a stretch of the vocabulary, and the sums meet in
// each block's shared memory, one cluster barrier a pass. The draw narrows down block, warp, step of the warp and lane from sums, so two short
// reads find the token. Sums are float64: a token of 10^-6 is to be told from its neighbour behind 10^5 others, and so every launch shape finds the
// same one.
#include <cooperative_groups.h>

#include <algorithm>
#include <cmath>

#include "jd_cache.h"
#include "jd_rope.cuh"

namespace cg = cooperative_groups;

namespace jd {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;             // the largest that every launch may have

struct ProbsParams {
  int B, T, V, range;                      // range: entries of a warp, whole steps
  const void *target, *draft;
  int64_t target_stride, draft_stride;     // elements between rows
  const int32_t *tokens, *parents, *num_nodes;
  int64_t parents_stride;                  // 0: shared
  const float *accept_u, *sample_u, *judge;
  float tau;
  int mode, resample, distinct;
  int32_t *accept_len, *next_token, *path;
  unsigned* status;
};

template <typename T> constexpr int kWide = 16 / sizeof(T);   // entries of a lane and step

template <typename T, bool kVec>
__device__ __forceinline__ void load_entries(const T* row, int v, int V, float* x) {   // entries v .. of the row, zeroes behind its end
  constexpr int kW = kWide<T>;
  if constexpr (kVec) {                    // V is a multiple of kW
    if (v < V) {
      if constexpr (kW == 8) load8(row + v, x);
      else { const float4 a = *reinterpret_cast<const float4*>(row + v); x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; }
      return;
    }
#pragma unroll
    for (int e = 0; e < kW; ++e) x[e] = 0.f;
  } else {
#pragma unroll
    for (int e = 0; e < kW; ++e) x[e] = v + e < V ? to_float(row[v + e]) : 0.f;
  }
}

struct Rejections {                        // of the node that the walk stands at
  int n;
  double W[kMaxNodes], Q[kMaxNodes];       // in front of each
  int x[kMaxNodes];                        // distinct siblings: the token; -1: none
};
// what is left of entry v
__device__ __forceinline__ double weight_of(const Rejections& r, bool distinct, int n, float p, float q, int v) {
  double w = p;
  if (n == 0) return w;
  double d = q;
  w = fmax(w - d, 0.0);                    // W = Q = 1
  for (int j = 1; j < n; ++j) {
    if (distinct && v == r.x[j - 1]) d = 0.0;
    w = fmax(w * r.Q[j] - r.W[j] * d, 0.0);
  }
  return w;
}

template <typename T, bool kVec>
__global__ void __launch_bounds__(kThreads, 2) verify_probs_kernel(const __grid_constant__ ProbsParams p) {
  constexpr int kW = kWide<T>, kStep = 32 * kW, kAhead = kW == 8 ? 2 : 4;
  __shared__ int s_token[kMaxNodes], s_parent[kMaxNodes], s_path[kMaxNodes];
  __shared__ float s_u[kMaxNodes], s_p[kMaxNodes], s_q[kMaxNodes];
  __shared__ uint8_t s_judge[kMaxNodes];
  __shared__ Rejections s_rej;
  __shared__ double s_warp[kWarps], s_step[kWarps], s_block[2][kMaxCluster];
  __shared__ int s_cur, s_pass, s_len;     // s_pass: weights after that many rejections are to be summed; < 0: the draw
  __shared__ int s_at;
  __shared__ double s_goal;
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = (int)cluster.block_rank(), blocks = (int)cluster.num_blocks();
  const int b = blockIdx.x / blocks, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_wait();
  pdl_trigger();
  const int T_ = p.T, nodes = p.num_nodes ? min(max(__ldcg(p.num_nodes + b), 0), T_) : T_;
  if (nodes == 0) return;                  // the whole cluster
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");   // waited for in front of the first write to another block
  const T* target = reinterpret_cast<const T*>(p.target) + (int64_t)b * T_ * p.target_stride;
  const T* draft = reinterpret_cast<const T*>(p.draft) + (int64_t)b * (T_ - 1) * p.draft_stride;

  for (int i = tid; i < nodes; i += kThreads) {
    if (i == 0) continue;
    const int64_t at = (int64_t)b * (T_ - 1) + i - 1;
    const int x = __ldcg(p.tokens + at), parent = p.parents ? __ldcg(p.parents + (int64_t)b * p.parents_stride + i) : i - 1;
    const bool in = x >= 0 && x < p.V, child = parent >= 0 && parent < i;
    s_token[i] = in ? x : -1;
    s_parent[i] = child ? parent : -1;
    s_u[i] = __ldcg(p.accept_u + at);
    s_judge[i] = p.mode != JD_MODE_STANDARD && __ldcg(p.judge + at) > p.tau;
    s_p[i] = in && child ? to_float(target[parent * p.target_stride + x]) : 0.f;
    s_q[i] = in && child ? to_float(draft[parent * p.draft_stride + x]) : 0.f;
    if (rank == 0 && p.status) {
      if (!in) set_status(p.status, JD_ERR_BAD_TOKEN);
      if (!child) set_status(p.status, JD_ERR_BAD_INDEX);
    }
  }
  if (tid == 0) { s_cur = 0; s_len = 0; s_rej.n = 0; }
  __syncthreads();

  // The walk's state lives in thread 0; every block's takes the same steps.
  int cur = 0, next = 1, len = 0;
  double W = 1.0, Q = 1.0, total = 0.0;
  bool ended = false, drawing = false;     // no child left; the weights of the draw have been summed
  for (int pass = 0;; ++pass) {
    if (tid == 0) {
      int n = s_rej.n, want = -1;
      if (!ended) {
        ended = true;
        for (; next < nodes; ++next) {
          if (s_parent[next] != cur) continue;
          const int x = s_token[next];
          double w = s_p[next], d = s_q[next];
          for (int j = 0; j < n; ++j) {
            w = fmax(w * s_rej.Q[j] - s_rej.W[j] * d, 0.0);
            if (p.distinct && x == s_rej.x[j]) d = 0.0;
          }
          const bool standard = (double)s_u[next] * W * d < w * Q;
          const bool ok = x >= 0 && ((p.mode != JD_MODE_JUDGE && standard) || s_judge[next]);
          if (ok) {
            s_path[len++] = next;
            cur = next;
            W = Q = 1.0;
            n = 0;
            continue;
          }
          s_rej.W[n] = W;
          s_rej.Q[n] = Q;
          s_rej.x[n] = x;
          ++n;
          if (p.distinct) Q -= d;
          ++next;
          want = n;
          ended = false;
          break;
        }
        s_rej.n = n;
        if (ended) {                       // what the draw goes by: the rest after the last rejection, summed already, or the target's own weights
          const bool rest = n > 0 && W > 0.0 && p.resample == JD_RESAMPLE_RESIDUAL;
          if (rest) { drawing = true; total = W; }
          else { s_rej.n = 0; want = 0; }
        }
      } else {
        drawing = true;
        total = W;
      }
      s_cur = cur;
      s_len = len;
      s_pass = drawing ? -1 : want;
    }
    __syncthreads();
    const int n = s_pass;
    if (n < 0) break;
    // ---- a pass: sums of what is left of the node's row
    const T* prow = target + s_cur * p.target_stride;
    const T* qrow = draft + s_cur * p.draft_stride;
    const int v0 = (rank * kWarps + warp) * p.range, v1 = min(v0 + p.range, p.V);
    double sum = 0.0;
    for (int v = v0; v < v1; v += kAhead * kStep) {
      float x[kAhead][kW], y[kAhead][kW];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int at = v + k * kStep + lane * kW;
        load_entries<T, kVec>(prow, at, v1, x[k]);
        if (n > 0) load_entries<T, kVec>(qrow, at, v1, y[k]);
        else {
#pragma unroll
          for (int e = 0; e < kW; ++e) y[k][e] = 0.f;
        }
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
#pragma unroll
        for (int e = 0; e < kW; ++e) sum += weight_of(s_rej, p.distinct, n, x[k][e], y[k][e], v + k * kStep + lane * kW + e);
    }
    sum = warp_sum_double(sum);
    if (lane == 0) s_warp[warp] = sum;
    if (pass == 0) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");   // every block has begun
    __syncthreads();
    if (tid < blocks) {
      double s = 0.0;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) s += s_warp[w];
      *cluster.map_shared_rank(&s_block[pass & 1][rank], tid) = s;     // buffers in turn: the next pass's writes come behind this one's barrier
    }
    cluster.sync();
    if (tid == 0) {
      W = 0.0;
      for (int k = 0; k < blocks; ++k) W += s_block[pass & 1][k];
      s_at = pass & 1;
    }
  }
  // ---- the draw: W > 0 unless the row has no mass at all
  const int n = s_rej.n, node = s_cur;
  if (rank == 0) {
    if (tid < T_ - 1 && p.path) p.path[(int64_t)b * (T_ - 1) + tid] = tid < s_len ? s_path[tid] : -1;
    if (tid == 0) p.accept_len[b] = s_len;
  }
  if (tid == 0) {
    // Goal: u times the sum. Rounding apart, a sum in front of the goal and one behind it lie in one block, warp and step; where nothing lies
    // behind (u not below 1, or rounding), the last with mass counts.
    const double goal = (double)__ldcg(p.sample_u + b) * total;
    double before = 0.0, mine = 0.0;
    int owner = -1, last = -1;
    double last_before = 0.0;
    for (int k = 0; k < blocks; ++k) {
      const double m = s_block[s_at][k];
      if (m > 0.0) { last = k; last_before = before; }
      if (owner < 0 && before + m > goal) { owner = k; mine = before; }
      before += m;
    }
    if (owner < 0) { owner = last; mine = last_before; }
    int at = -1;
    double in = mine;
    if (owner == rank) {
      int last_warp = -1;
      double last_in = mine;
      for (int w = 0; w < kWarps; ++w) {
        if (s_warp[w] > 0.0) { last_warp = w; last_in = in; }
        if (at < 0 && in + s_warp[w] > goal) { at = w; break; }
        in += s_warp[w];
      }
      if (at < 0) { at = last_warp; in = last_in; }
    }
    s_at = at;
    s_goal = goal - in;
    if (owner < 0 && rank == 0) p.next_token[b] = p.V - 1;
  }
  __syncthreads();
  if (s_at < 0) return;
  const T* prow = target + node * p.target_stride;
  const T* qrow = draft + node * p.draft_stride;
  const int v0 = (rank * kWarps + s_at) * p.range, v1 = min(v0 + p.range, p.V), steps = (v1 - v0 + kStep - 1) / kStep;
  double goal = s_goal;
  // the step: warps take a step each; batches of them where a warp's range has more
  int found = -1;
  for (int base = 0; base < steps && found < 0; base += kWarps) {
    __syncthreads();
    double sum = 0.0;
    if (base + warp < steps) {
      float x[kW], y[kW] = {};
      const int at = v0 + (base + warp) * kStep + lane * kW;
      load_entries<T, kVec>(prow, at, v1, x);
      if (n > 0) load_entries<T, kVec>(qrow, at, v1, y);
#pragma unroll
      for (int e = 0; e < kW; ++e) sum += weight_of(s_rej, p.distinct, n, x[e], y[e], at + e);
    }
    sum = warp_sum_double(sum);
    if (lane == 0) s_step[warp] = sum;
    __syncthreads();
    int last = -1;
    double last_goal = goal;
    for (int k = 0; k < kWarps && base + k < steps; ++k) {
      const double m = s_step[k];
      if (m > 0.0) { last = base + k; last_goal = goal; }
      if (m > goal) { found = base + k; break; }
      goal -= m;
    }
    if (found < 0 && base + kWarps >= steps && last >= 0) { found = last; goal = last_goal; }
  }
  if (warp != 0) return;
  if (found < 0) found = steps - 1;
  float x[kW], y[kW] = {};
  const int at = v0 + found * kStep + lane * kW;
  load_entries<T, kVec>(prow, at, v1, x);
  if (n > 0) load_entries<T, kVec>(qrow, at, v1, y);
  double w[kW], mine = 0.0;
#pragma unroll
  for (int e = 0; e < kW; ++e) { w[e] = weight_of(s_rej, p.distinct, n, x[e], y[e], at + e); mine += w[e]; }
  double run = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const double z = __shfl_up_sync(0xffffffffu, run, o);
    if (lane >= o) run += z;
  }
  const unsigned behind = __ballot_sync(0xffffffffu, run > goal), some = __ballot_sync(0xffffffffu, mine > 0.0);
  const int who = behind ? __ffs(behind) - 1 : (some ? 31 - __clz(some) : 31);
  if (lane != who) return;
  double in = run - mine;
  int token = -1, last = min(at, p.V - 1);
#pragma unroll
  for (int e = 0; e < kW; ++e) {
    in += w[e];
    if (w[e] > 0.0) {
      last = at + e;
      if (token < 0 && in > goal) token = at + e;
    }
  }
  p.next_token[b] = token < 0 ? last : token;
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
  return cudaLaunchKernelEx(&cfg, verify_probs_kernel<T, kVec>, p);
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
  p.tau = a->tau; p.mode = a->mode; p.resample = a->resample; p.distinct = a->siblings == JD_SIBLINGS_DISTINCT;
  p.accept_len = a->accept_len; p.next_token = a->next_token; p.path = a->path;
  p.status = a->device_status;
  // As many blocks for a sequence as keep all sequences on the device at once, two blocks on an SM
  int blocks = kMaxCluster;
  while (blocks > 1 && a->B * blocks > 2 * sms) blocks /= 2;
  const int step = 32 * 16 / (int)e, warps = blocks * kWarps;
  p.range = (int)(((int64_t)a->V + (int64_t)warps * step - 1) / ((int64_t)warps * step)) * step;
  const bool vec = on(a->target, 16) && (!drafted || on(a->draft, 16)) && a->V % (16 / (int)e) == 0 && ts * e % 16 == 0 && ds * e % 16 == 0;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  cudaError_t err;
  if (a->dtype == JD_DTYPE_F32) err = vec ? launch_probs<float, true>(p, blocks, st) : launch_probs<float, false>(p, blocks, st);
  else err = vec ? launch_probs<__nv_bfloat16, true>(p, blocks, st) : launch_probs<__nv_bfloat16, false>(p, blocks, st);
  if (err != cudaSuccess) { cudaGetLastError(); return JD_ERR_CUDA; }
  return JD_OK;
}
