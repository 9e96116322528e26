// RMS norms of query and key heads and their rotary positions in one pass: alone (jd_head_rope), backwards (jd_head_rope_grad) and on
// the way into the cache (jd_cache_append_heads). A frequency takes one of a token's positions (time, row and column of an image, say).
//
//   r = 1 / sqrt(mean x^2 + eps),   n = r x,   y = R(n w)      R: the rotation of jd_rope.cu, amplitude included
//   g = R' dy (the transpose),      dx = r (g w - n mean(g w n)),      dw = sum over tokens and heads of g n
//
// Everything between the loads and the one rounding at the end is float32, so the floor is the bytes over the HBM rate. As many lanes as a head
// has pieces of 16 bytes (or, half a rotation apart, pairs of them) hold it in registers: a sum over the head is a few shuffles, and nothing is
// read twice. Angles are formed once for a block's tokens and shared by their heads. In shared memory, pair e of piece u stands at
// e x pieces + u, so that the lanes of a head read neighbouring words.
#include <algorithm>
#include <cmath>

#include "jd_rope.cuh"

namespace jd {
namespace {

constexpr int kThreads = 256;
constexpr int kTokensPerBlock = 8;
constexpr int kMaxDim = 256;
constexpr int kMaxAxes = 4;
constexpr int kGradBlocks = 592;          // persistent blocks of the backward pass, each with a partial sum of dw: four for every SM of a B200

enum Form { kScalar = 0, kHalfVec = 1, kPairVec = 2 };   // single pairs; 8 + 8 elements half a rotation apart; 8 elements, 4 pairs

struct AxisMap {
  int axes;
  uint8_t of[kMaxHalf];
};

struct HeadShape {
  int head_dim, half, layout;
  float amplitude;
  const float* inv_freq;
  const float *wq, *wk;      // null: ones
  float eps;
  bool normalize;
};

// A lane's part of a head: kUnits pieces of kPairs pairs (a, b). Pieces behind the turning ones pass through; kHalfVec has no b there.
template <int kForm> struct Lane {
  static constexpr int kPairs = kForm == kHalfVec ? 8 : (kForm == kPairVec ? 4 : 1);
  static constexpr int kUnits = kForm == kScalar ? 8 : 1;       // 32 lanes x 8 single pairs or elements: the widest head
  static constexpr int kN = kPairs * kUnits;
};
template <int kForm> __host__ __device__ __forceinline__ int turning_units(int half) { return half / Lane<kForm>::kPairs; }
template <int kForm> __host__ __device__ __forceinline__ int all_units(int head_dim, int half) {
  return turning_units<kForm>(half) + (head_dim - 2 * half) / (kForm == kScalar ? 1 : 8);
}
// elements of pair e of piece u; b < 0: there is none
template <int kForm> __device__ __forceinline__ void elements_of(const HeadShape& s, int turning, int u, int e, int& a, int& b) {
  if (u < turning) {
    const int f = u * Lane<kForm>::kPairs + e;
    if (kForm == kHalfVec || (kForm == kScalar && s.layout == JD_ROPE_HALF)) { a = f; b = f + s.half; }
    else { a = 2 * f; b = a + 1; }
  } else {
    const int v = u - turning;
    if (kForm == kPairVec) { a = 2 * s.half + 8 * v + 2 * e; b = a + 1; }
    else { a = 2 * s.half + (kForm == kHalfVec ? 8 * v + e : v); b = -1; }
  }
}

template <typename T, int kForm>
__device__ __forceinline__ void load_unit(const T* x, const HeadShape& s, int turning, int u, float* a, float* b) {
  int ia, ib;
  elements_of<kForm>(s, turning, u, 0, ia, ib);
  if constexpr (kForm == kScalar) {
    a[0] = to_float(x[ia]);
    b[0] = ib < 0 ? 0.f : to_float(x[ib]);
  } else if constexpr (kForm == kHalfVec) {
    load8(x + ia, a);
    if (ib >= 0) load8(x + ib, b);
    else {
#pragma unroll
      for (int e = 0; e < 8; ++e) b[e] = 0.f;
    }
  } else {
    float v[8];
    load8(x + ia, v);
#pragma unroll
    for (int e = 0; e < 4; ++e) { a[e] = v[2 * e]; b[e] = v[2 * e + 1]; }
  }
}
template <typename T, int kForm>
__device__ __forceinline__ void store_unit(T* y, const HeadShape& s, int turning, int u, const float* a, const float* b) {
  int ia, ib;
  elements_of<kForm>(s, turning, u, 0, ia, ib);
  if constexpr (kForm == kScalar) {
    y[ia] = from_float(a[0], T());
    if (ib >= 0) y[ib] = from_float(b[0], T());
  } else if constexpr (kForm == kHalfVec) {
    store8(y + ia, a);
    if (ib >= 0) store8(y + ib, b);
  } else {
    float v[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) { v[2 * e] = a[e]; v[2 * e + 1] = b[e]; }
    store8(y + ia, v);
  }
}

__device__ __forceinline__ float sum_over(float v, int lanes) {
  for (int o = lanes >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Weights of both kinds of heads as pairs, by the whole block.
template <int kForm>
__device__ __forceinline__ void fill_weights(const HeadShape& s, float2 (*sw)[kMaxDim], int turning, int units) {
  for (int i = threadIdx.x; i < 2 * Lane<kForm>::kPairs * units; i += kThreads) {
    const int kind = i / (Lane<kForm>::kPairs * units), j = i - kind * Lane<kForm>::kPairs * units, e = j / units, u = j - e * units;
    const float* w = kind ? s.wk : s.wq;
    int a, b;
    elements_of<kForm>(s, turning, u, e, a, b);
    sw[kind][j] = make_float2(w ? __ldcg(w + a) : 1.f, w && b >= 0 ? __ldcg(w + b) : 1.f);
  }
}
// the place of frequency f
template <int kForm> __device__ __forceinline__ int turn_at(int f, int turning) {
  return (f % Lane<kForm>::kPairs) * turning + f / Lane<kForm>::kPairs;
}

// One head: the lanes of a group (`lane` of `lanes`) take its pieces. Every lane of the warp comes here; `live` says whether the group has a head.
template <typename T, int kForm>
__device__ __forceinline__ void forward_head(const T* x, T* y, const HeadShape& s, const float2* cs, const float2* sw, int turning, int units, int lane,
                                             int lanes, bool live) {
  using L = Lane<kForm>;
  float a[L::kN], b[L::kN];
  float sum = 0.f;
#pragma unroll
  for (int k = 0; k < L::kUnits; ++k) {
    const int u = lane + k * lanes;
    float *pa = a + k * L::kPairs, *pb = b + k * L::kPairs;
    if (live && u < units) load_unit<T, kForm>(x, s, turning, u, pa, pb);
    else {
#pragma unroll
      for (int e = 0; e < L::kPairs; ++e) pa[e] = pb[e] = 0.f;
    }
  }
  float r = 1.f;
  if (s.normalize) {
#pragma unroll
    for (int i = 0; i < L::kN; ++i) sum = fmaf(a[i], a[i], fmaf(b[i], b[i], sum));
    r = rsqrtf(sum_over(sum, lanes) / (float)s.head_dim + s.eps);
  }
#pragma unroll
  for (int k = 0; k < L::kUnits; ++k) {
    const int u = lane + k * lanes;
    if (!live || u >= units) continue;
    float *pa = a + k * L::kPairs, *pb = b + k * L::kPairs;
#pragma unroll
    for (int e = 0; e < L::kPairs; ++e) {
      if (s.normalize) {
        const float2 w = sw[e * units + u];
        pa[e] = pa[e] * r * w.x;
        pb[e] = pb[e] * r * w.y;
      }
      if (u < turning) {
        const float2 t = cs[e * turning + u];
        const float p = pa[e] * t.x - pb[e] * t.y;
        pb[e] = pb[e] * t.x + pa[e] * t.y;
        pa[e] = p;
      }
    }
    store_unit<T, kForm>(y, s, turning, u, pa, pb);
  }
}

struct HeadParams {
  HeadShape s;
  int64_t tokens;
  int q_heads, k_heads, per_block, lanes;
  const void *q, *k, *gq, *gk;       // gradients of the outputs: backward alone
  void *q_out, *k_out;
  int64_t q_stride, k_stride, q_out_stride, k_out_stride, gq_stride, gk_stride;   // elements
  const int32_t* positions;          // [tokens][axes]
  int inverse;
  float* part;                       // backward: [blocks][2][head_dim] partial sums of dw; null: no weight gradients
};

template <int kForm>
__device__ __forceinline__ void fill_turns(const HeadParams& p, const AxisMap& m, float2 (*cs)[kMaxHalf], int64_t t0, int n, int turning, bool inverse) {
  const int half = p.s.half;
  for (int i = threadIdx.x; i < n * half; i += kThreads) {
    const int t = i / half, f = i - t * half;
    cs[t][turn_at<kForm>(f, turning)] = turn_of(__ldcg(p.positions + (t0 + t) * m.axes + m.of[f]), __ldcg(p.s.inv_freq + f), p.s.amplitude, inverse);
  }
}

template <typename T, int kForm>
__global__ void __launch_bounds__(kThreads) head_rope_kernel(const __grid_constant__ HeadParams p, const __grid_constant__ AxisMap m) {
  __shared__ float2 cs[kTokensPerBlock][kMaxHalf];
  __shared__ float2 sw[2][kMaxDim];
  pdl_wait();
  pdl_trigger();
  const HeadShape& s = p.s;
  const int turning = turning_units<kForm>(s.half), units = all_units<kForm>(s.head_dim, s.half);
  const int64_t t0 = (int64_t)blockIdx.x * p.per_block;
  const int n = (int)min((int64_t)p.per_block, p.tokens - t0);
  if (s.normalize) fill_weights<kForm>(s, sw, turning, units);
  fill_turns<kForm>(p, m, cs, t0, n, turning, p.inverse != 0);
  __syncthreads();
  const int lanes = p.lanes, groups = kThreads / lanes, group = threadIdx.x / lanes, lane = threadIdx.x & (lanes - 1);
  const int heads = p.q_heads + p.k_heads, items = n * heads;
  for (int i0 = 0; i0 < items; i0 += groups) {
    const int i = i0 + group;
    const bool live = i < items;
    const int t = live ? i / heads : 0, j = live ? i - t * heads : 0;
    const bool key = j >= p.q_heads;
    const int h = key ? j - p.q_heads : j;
    const T* x = reinterpret_cast<const T*>(key ? p.k : p.q) + (t0 + t) * (key ? p.k_stride : p.q_stride) + (int64_t)h * s.head_dim;
    T* y = reinterpret_cast<T*>(key ? p.k_out : p.q_out) + (t0 + t) * (key ? p.k_out_stride : p.q_out_stride) + (int64_t)h * s.head_dim;
    forward_head<T, kForm>(x, y, s, cs[t], sw[key], turning, units, lane, lanes, live);
  }
}

// Blocks walk over the tokens; queries first, then keys, so that a lane's sums of g n, whose elements stay the same, are registers. Blocks add
// theirs up in a fixed order (partial sums, then head_rope_weights_kernel): results repeat bit for bit.
template <typename T, int kForm>
__global__ void __launch_bounds__(kThreads) head_rope_grad_kernel(const __grid_constant__ HeadParams p, const __grid_constant__ AxisMap m) {
  using L = Lane<kForm>;
  __shared__ float2 cs[kTokensPerBlock][kMaxHalf];
  __shared__ float2 sw[2][kMaxDim];
  extern __shared__ float s_sum[];                     // [groups][head_dim]
  pdl_wait();
  pdl_trigger();
  const HeadShape& s = p.s;
  const int turning = turning_units<kForm>(s.half), units = all_units<kForm>(s.head_dim, s.half);
  const int lanes = p.lanes, groups = kThreads / lanes, group = threadIdx.x / lanes, lane = threadIdx.x & (lanes - 1);
  fill_weights<kForm>(s, sw, turning, units);
  float sum_a[2][L::kN], sum_b[2][L::kN];
#pragma unroll
  for (int i = 0; i < L::kN; ++i) sum_a[0][i] = sum_a[1][i] = sum_b[0][i] = sum_b[1][i] = 0.f;
  const float per_dim = 1.f / (float)s.head_dim;
  for (int64_t t0 = (int64_t)blockIdx.x * p.per_block; t0 < p.tokens; t0 += (int64_t)gridDim.x * p.per_block) {
    const int n = (int)min((int64_t)p.per_block, p.tokens - t0);
    __syncthreads();                                   // the last tokens' angles have been used
    fill_turns<kForm>(p, m, cs, t0, n, turning, false);
    __syncthreads();
#pragma unroll
    for (int kind = 0; kind < 2; ++kind) {
      const int heads = kind ? p.k_heads : p.q_heads, items = n * heads;
      const T* xs = reinterpret_cast<const T*>(kind ? p.k : p.q);
      const T* gs = reinterpret_cast<const T*>(kind ? p.gk : p.gq);
      T* ds = reinterpret_cast<T*>(kind ? p.k_out : p.q_out);
      const int64_t x_stride = kind ? p.k_stride : p.q_stride, g_stride = kind ? p.gk_stride : p.gq_stride, d_stride = kind ? p.k_out_stride : p.q_out_stride;
      for (int i0 = 0; i0 < items; i0 += groups) {
        const int i = i0 + group;
        const bool live = i < items;
        const int t = live ? i / heads : 0, h = live ? i - t * heads : 0;
        const T* x = xs + (t0 + t) * x_stride + (int64_t)h * s.head_dim;
        const T* g = gs + (t0 + t) * g_stride + (int64_t)h * s.head_dim;
        float xa[L::kN], xb[L::kN], ga[L::kN], gb[L::kN];
#pragma unroll
        for (int k = 0; k < L::kUnits; ++k) {
          const int u = lane + k * lanes, at = k * L::kPairs;
          if (live && u < units) {
            load_unit<T, kForm>(x, s, turning, u, xa + at, xb + at);
            load_unit<T, kForm>(g, s, turning, u, ga + at, gb + at);
          } else {
#pragma unroll
            for (int e = 0; e < L::kPairs; ++e) xa[at + e] = xb[at + e] = ga[at + e] = gb[at + e] = 0.f;
          }
        }
        float squares = 0.f, dot = 0.f;
#pragma unroll
        for (int k = 0; k < L::kUnits; ++k) {
          const int u = lane + k * lanes, at = k * L::kPairs;
          if (!live || u >= units) continue;
#pragma unroll
          for (int e = 0; e < L::kPairs; ++e) {
            float &pa = ga[at + e], &pb = gb[at + e];
            if (u < turning) {                         // the transpose: turned back
              const float2 c = cs[t][e * turning + u];
              const float q = pa * c.x + pb * c.y;
              pb = pb * c.x - pa * c.y;
              pa = q;
            }
            const float2 w = sw[kind][e * units + u];
            squares = fmaf(xa[at + e], xa[at + e], fmaf(xb[at + e], xb[at + e], squares));
            dot = fmaf(pa * w.x, xa[at + e], fmaf(pb * w.y, xb[at + e], dot));
          }
        }
        squares = sum_over(squares, lanes);
        dot = sum_over(dot, lanes);
        const float r = rsqrtf(squares * per_dim + s.eps);
        const float mean = dot * r * per_dim;           // of g w n
#pragma unroll
        for (int k = 0; k < L::kUnits; ++k) {
          const int u = lane + k * lanes, at = k * L::kPairs;
          if (!live || u >= units) continue;
          float da[L::kPairs], db[L::kPairs];
#pragma unroll
          for (int e = 0; e < L::kPairs; ++e) {
            const float2 w = sw[kind][e * units + u];
            const float na = xa[at + e] * r, nb = xb[at + e] * r;
            da[e] = r * (ga[at + e] * w.x - na * mean);
            db[e] = r * (gb[at + e] * w.y - nb * mean);
            sum_a[kind][at + e] = fmaf(ga[at + e], na, sum_a[kind][at + e]);
            sum_b[kind][at + e] = fmaf(gb[at + e], nb, sum_b[kind][at + e]);
          }
          store_unit<T, kForm>(ds + (t0 + t) * d_stride + (int64_t)h * s.head_dim, s, turning, u, da, db);
        }
      }
    }
  }
  if (!p.part) return;
#pragma unroll
  for (int kind = 0; kind < 2; ++kind) {
    __syncthreads();
#pragma unroll
    for (int k = 0; k < L::kUnits; ++k) {
      const int u = lane + k * lanes;
      if (u >= units) continue;
#pragma unroll
      for (int e = 0; e < L::kPairs; ++e) {
        int a, b;
        elements_of<kForm>(s, turning, u, e, a, b);
        s_sum[group * s.head_dim + a] = sum_a[kind][k * L::kPairs + e];
        if (b >= 0) s_sum[group * s.head_dim + b] = sum_b[kind][k * L::kPairs + e];
      }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < s.head_dim; i += kThreads) {
      float v = 0.f;
      for (int g = 0; g < groups; ++g) v += s_sum[g * s.head_dim + i];
      p.part[((int64_t)blockIdx.x * 2 + kind) * s.head_dim + i] = v;
    }
  }
}

// dw of 32 elements: eight warps take a block's partial sums each in turn.
__global__ void __launch_bounds__(kThreads) head_rope_weights_kernel(const float* part, int blocks, int head_dim, float* dwq, float* dwk) {
  __shared__ float s_sum[kThreads / 32][32];
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, i = blockIdx.x * 32 + lane, kind = blockIdx.y;
  float v[4] = {};
  if (i < head_dim)
    for (int b = warp; b < blocks; b += kThreads / 8) {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (b + k * (kThreads / 32) < blocks) v[k] += __ldcg(part + ((int64_t)(b + k * (kThreads / 32)) * 2 + kind) * head_dim + i);
    }
  s_sum[warp][lane] = (v[0] + v[1]) + (v[2] + v[3]);
  __syncthreads();
  float* out = kind ? dwk : dwq;
  if (warp == 0 && i < head_dim && out) {
    float x = 0.f;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) x += s_sum[w][lane];
    out[i] = x;
  }
}

struct AppendHeadsParams {
  CacheView c;
  HeadShape s;
  int B, T, layer, q_heads, lanes;
  const int32_t* slots;
  const int32_t* depth;
  int64_t depth_stride;          // 0: shared
  const int32_t* num_nodes;
  const int32_t* positions;      // [B][T][axes]; null: seq_len + depth on every axis
  const char *k, *v, *q;
  char* q_out;
  int64_t k_stride, v_stride, q_stride, q_out_stride;   // bytes
};

// One block per node and part of its heads, as append_kernel; values are copied as they are.
template <typename T, int kForm>
__global__ void __launch_bounds__(kThreads) append_heads_kernel(const __grid_constant__ AppendHeadsParams p, const __grid_constant__ AxisMap m) {
  __shared__ float2 cs[kMaxHalf];
  __shared__ float2 sw[2][kMaxDim];
  __shared__ int dup;
  pdl_wait();
  pdl_trigger();
  const int b = blockIdx.x / p.T, t = blockIdx.x - b * p.T;
  const CacheView& c = p.c;
  const HeadShape& s = p.s;
  const int slot = slot_of(c, p.slots, b);
  if (slot < 0) return;
  if (p.num_nodes && t >= __ldcg(p.num_nodes + b)) return;
  if (threadIdx.x == 0) dup = 0;
  __syncthreads();
  if (p.slots)
    for (int i = threadIdx.x; i < b; i += kThreads)
      if (__ldcg(p.slots + i) == slot) dup = 1;
  int len, held;
  slot_state(c, slot, len, held);
  const int at = len + t;
  const int64_t token = (int64_t)b * p.T + t;
  const int pos = p.positions ? 0 : len + (p.depth ? __ldcg(p.depth + (int64_t)b * p.depth_stride + t) : t);
  const int turning = turning_units<kForm>(s.half), units = all_units<kForm>(s.head_dim, s.half);
  for (int f = threadIdx.x; f < s.half; f += kThreads)
    cs[turn_at<kForm>(f, turning)] = turn_of(p.positions ? __ldcg(p.positions + token * m.axes + m.of[f]) : pos, __ldcg(s.inv_freq + f), s.amplitude, false);
  if (s.normalize) fill_weights<kForm>(s, sw, turning, units);
  // the row's page: held, in range, and this sequence's alone
  int page = -1;
  if ((at >> c.page_shift) < held) {
    page = __ldcg(c.table + (int64_t)slot * c.max_pages + (at >> c.page_shift));
    if (page < 0 || page >= c.pages || __ldcg(c.refs + page) > 1) page = -1;
  }
  __syncthreads();
  if (dup) {   // an earlier entry names this slot: it counts
    if (threadIdx.x == 0 && t == 0) set_status(c.status, JD_ERR_BAD_INDEX);
    return;
  }
  if (page < 0 && threadIdx.x == 0) set_status(c.status, JD_ERR_BAD_INDEX);
  const int row = at & (c.page_size - 1);
  const int lanes = p.lanes, groups = kThreads / lanes, group = threadIdx.x / lanes, lane = threadIdx.x & (lanes - 1);
  const int items = p.q_heads + (page < 0 ? 0 : c.kv_heads);
  const T* q = reinterpret_cast<const T*>(p.q + token * p.q_stride);
  T* qo = reinterpret_cast<T*>(p.q_out + token * p.q_out_stride);
  const T* k = reinterpret_cast<const T*>(p.k + token * p.k_stride);
  if (page >= 0) {
    const int vunits = c.row_bytes / 16;
    for (int j = blockIdx.y * kThreads + threadIdx.x; j < c.kv_heads * vunits; j += gridDim.y * kThreads) {
      const int h = j / vunits, u = j - h * vunits;
      const char* src = p.v + token * p.v_stride + (int64_t)h * c.row_bytes;
      char* dst = c.v + page_row(c, p.layer, page, h, row) * c.row_bytes;
      reinterpret_cast<uint4*>(dst)[u] = reinterpret_cast<const uint4*>(src)[u];
    }
  }
  for (int i0 = blockIdx.y * groups; i0 < items; i0 += gridDim.y * groups) {
    const int i = i0 + group;
    const bool live = i < items, key = i >= p.q_heads;
    const int h = !live ? 0 : (key ? i - p.q_heads : i);
    const T* x = (key ? k : q) + h * s.head_dim;
    T* y = key ? (live ? reinterpret_cast<T*>(c.k + page_row(c, p.layer, page, h, row) * c.row_bytes) : nullptr) : qo + h * s.head_dim;
    forward_head<T, kForm>(x, y, s, cs, sw[key], turning, units, lane, lanes, live);
  }
}

// ------------------------------------------------------------------------------------------ host side

bool axes_ok(const jd_rope_axes_t* a, int half, AxisMap* m) {
  m->axes = 1;
  for (int i = 0; i < kMaxHalf; ++i) m->of[i] = 0;
  if (!a) return true;
  if (a->num_axes < 1 || a->num_axes > kMaxAxes) return false;
  m->axes = a->num_axes;
  if (!a->axis_of) return true;
  for (int i = 0; i < half; ++i) {
    if (a->axis_of[i] >= a->num_axes) return false;
    m->of[i] = a->axis_of[i];
  }
  return true;
}
bool on4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
bool norm_ok(const jd_head_norm_t* n) { return !n || (on4(n->q_weight) && on4(n->k_weight) && n->eps >= 0.f && std::isfinite(n->eps)); }

HeadShape shape_of(const jd_rope_t* r, const jd_head_norm_t* n, int head_dim) {
  HeadShape s;
  s.head_dim = head_dim;
  s.half = r ? r->rot_dim / 2 : 0;
  s.layout = r ? r->layout : JD_ROPE_HALF;
  s.amplitude = r ? r->amplitude : 1.f;
  s.inv_freq = r ? r->inv_freq : nullptr;
  s.normalize = n != nullptr;
  s.wq = n ? n->q_weight : nullptr;
  s.wk = n ? n->k_weight : nullptr;
  s.eps = n ? n->eps : 0.f;
  return s;
}
Form form_of(const HeadShape& s, bool vec) { return !vec ? kScalar : (s.layout == JD_ROPE_HALF ? kHalfVec : kPairVec); }
// lanes of a group: a power of two that holds the head's pieces
int lanes_of(const HeadShape& s, Form f) {
  if (f == kScalar) return 32;
  const int units = f == kHalfVec ? all_units<kHalfVec>(s.head_dim, s.half) : all_units<kPairVec>(s.head_dim, s.half);
  int n = 1;
  while (n < units) n *= 2;
  return n;
}

struct Rows {                        // one of the call's arrays of heads
  const void* p;
  int64_t stride;                    // 0: dense
};
bool rows_ok(const Rows& r, int heads, int head_dim, uintptr_t e) {
  return r.p && reinterpret_cast<uintptr_t>(r.p) % e == 0 && (r.stride == 0 || r.stride >= (int64_t)heads * head_dim) && r.stride <= ((int64_t)1 << 40);
}
int64_t step_of(const Rows& r, int heads, int head_dim) { return r.stride ? r.stride : (int64_t)heads * head_dim; }
bool rows_on16(const Rows& r, int heads, int head_dim, int e) {
  return reinterpret_cast<uintptr_t>(r.p) % 16 == 0 && step_of(r, heads, head_dim) * e % 16 == 0;
}

bool shape_args_ok(int64_t tokens, int q_heads, int k_heads, int head_dim, int dtype, const jd_rope_t& r) {
  if (tokens < 0 || tokens > 0x7FFFFFFF || q_heads < 0 || k_heads < 0 || q_heads > 65536 || k_heads > 65536 || q_heads + k_heads < 1) return false;
  return head_dim >= 1 && head_dim <= kMaxDim && (dtype == JD_DTYPE_F32 || dtype == JD_DTYPE_BF16) && rope_valid(r, head_dim);
}

// tokens of a block: about 16 elements of head a thread and turn, so that the angles pay for themselves
int tokens_per_block(const HeadParams& p) {
  const int groups = kThreads / p.lanes;
  return std::max(1, std::min(kTokensPerBlock, 4 * groups / (p.q_heads + p.k_heads)));
}

template <template <typename, int> class Run, typename... Args>
cudaError_t by_form(int dtype, Form f, Args&&... args) {
  if (dtype == JD_DTYPE_F32) {
    if (f == kScalar) return Run<float, kScalar>::go(args...);
    return f == kHalfVec ? Run<float, kHalfVec>::go(args...) : Run<float, kPairVec>::go(args...);
  }
  if (f == kScalar) return Run<__nv_bfloat16, kScalar>::go(args...);
  return f == kHalfVec ? Run<__nv_bfloat16, kHalfVec>::go(args...) : Run<__nv_bfloat16, kPairVec>::go(args...);
}
template <typename T, int kForm> struct Forward {
  static cudaError_t go(const HeadParams& p, const AxisMap& m, cudaStream_t st) {
    const int64_t blocks = (p.tokens + p.per_block - 1) / p.per_block;
    return launch_chained(head_rope_kernel<T, kForm>, dim3((unsigned)blocks), dim3(kThreads), 0, st, p, m);
  }
};
int grad_blocks(int64_t tokens, int per_block) { return (int)std::min<int64_t>(kGradBlocks, (tokens + per_block - 1) / per_block); }
template <typename T, int kForm> struct Backward {
  static cudaError_t go(const HeadParams& p, const AxisMap& m, cudaStream_t st) {
    return launch_chained(head_rope_grad_kernel<T, kForm>, dim3((unsigned)grad_blocks(p.tokens, p.per_block)), dim3(kThreads),
                          (size_t)(p.part ? kThreads / p.lanes * p.s.head_dim * 4 : 0), st, p, m);
  }
};
template <typename T, int kForm> struct Append {
  static cudaError_t go(const AppendHeadsParams& p, const AxisMap& m, dim3 grid, cudaStream_t st) {
    return launch_chained(append_heads_kernel<T, kForm>, grid, dim3(kThreads), 0, st, p, m);
  }
};

}  // namespace

bool append_heads_valid(const jd_head_norm_t* n, const jd_rope_axes_t* a, const jd_rope_t* r) {
  AxisMap m;
  return norm_ok(n) && axes_ok(a, r ? r->rot_dim / 2 : 0, &m);
}

cudaError_t run_append_heads(const CacheView& c, const jd_append_args_t& a, const jd_append_heads_t& x, int q_heads, int dtype, cudaStream_t st) {
  const int e = dtype == JD_DTYPE_F32 ? 4 : 2;
  AppendHeadsParams p;
  AxisMap m;
  if (!axes_ok(x.axes, a.rope ? a.rope->rot_dim / 2 : 0, &m)) return cudaErrorInvalidValue;
  p.c = c;
  p.s = shape_of(a.rope, x.norm, c.head_dim);
  p.B = a.B; p.T = a.tree.nodes; p.layer = a.layer;
  p.q_heads = a.q ? q_heads : 0;
  p.slots = a.slots;
  p.depth = a.tree.depth;
  p.depth_stride = a.tree.per_seq ? a.tree.nodes : 0;
  p.num_nodes = a.tree.num_nodes;
  p.positions = x.positions;
  p.k = (const char*)a.k; p.v = (const char*)a.v; p.q = (const char*)a.q; p.q_out = (char*)a.q_out;
  auto bytes = [&](int64_t s, int heads) { return (s ? s : (int64_t)heads * c.head_dim) * e; };
  p.k_stride = bytes(a.k_stride, c.kv_heads); p.v_stride = bytes(a.v_stride, c.kv_heads);
  p.q_stride = bytes(a.q_stride, q_heads); p.q_out_stride = bytes(a.q_out_stride, q_heads);
  const Form f = form_of(p.s, vec_ok(2 * p.s.half, c.head_dim));     // the cache's rows and the call's start on 16 bytes
  p.lanes = lanes_of(p.s, f);
  const int nodes = a.B * a.tree.nodes, groups = kThreads / p.lanes;
  // few nodes: one head for each group of lanes, spread over the SMs; many: a block per node
  const int parts = nodes >= 512 ? 1 : std::max(1, std::min(8, (p.q_heads + c.kv_heads + groups - 1) / groups));
  return by_form<Append>(dtype, f, p, m, dim3((unsigned)nodes, (unsigned)parts), st);
}

}  // namespace jd

using namespace jd;

extern "C" {

jd_status_t jd_head_rope(const jd_head_rope_args_t* a, void* cuda_stream) {
  if (!a || !shape_args_ok(a->tokens, a->q_heads, a->k_heads, a->head_dim, a->dtype, a->rope) || !norm_ok(a->norm)) return JD_ERR_INVALID_ARG;
  HeadParams p = {};
  AxisMap m;
  if (!axes_ok(a->axes, a->rope.rot_dim / 2, &m) || (a->inverse != 0 && a->inverse != 1) || (a->inverse && a->norm)) return JD_ERR_INVALID_ARG;
  if (a->tokens == 0) return JD_OK;
  const int e = a->dtype == JD_DTYPE_F32 ? 4 : 2, D = a->head_dim;
  bool vec = vec_ok(a->rope.rot_dim, D);
  const Rows in[2] = {{a->q, a->q_stride}, {a->k, a->k_stride}}, out[2] = {{a->q_out, a->q_out_stride}, {a->k_out, a->k_out_stride}};
  for (int i = 0; i < 2; ++i) {
    const int heads = i ? a->k_heads : a->q_heads;
    if (heads == 0) continue;
    if (!rows_ok(in[i], heads, D, e) || !rows_ok(out[i], heads, D, e)) return JD_ERR_INVALID_ARG;
    if (in[i].p == out[i].p && step_of(in[i], heads, D) != step_of(out[i], heads, D)) return JD_ERR_INVALID_ARG;
    vec = vec && rows_on16(in[i], heads, D, e) && rows_on16(out[i], heads, D, e);
  }
  if (!a->positions || !on4(a->positions)) return JD_ERR_INVALID_ARG;
  p.s = shape_of(&a->rope, a->norm, D);
  const Form f = form_of(p.s, vec);
  p.lanes = lanes_of(p.s, f);
  p.tokens = a->tokens; p.q_heads = a->q_heads; p.k_heads = a->k_heads;
  p.q = a->q; p.k = a->k; p.q_out = a->q_out; p.k_out = a->k_out;
  p.q_stride = step_of(in[0], a->q_heads, D); p.k_stride = step_of(in[1], a->k_heads, D);
  p.q_out_stride = step_of(out[0], a->q_heads, D); p.k_out_stride = step_of(out[1], a->k_heads, D);
  p.positions = a->positions;
  p.inverse = a->inverse;
  p.per_block = tokens_per_block(p);
  if (by_form<Forward>(a->dtype, f, p, m, (cudaStream_t)cuda_stream) != cudaSuccess) { cudaGetLastError(); return JD_ERR_CUDA; }
  return JD_OK;
}

size_t jd_head_rope_grad_workspace_bytes(int32_t head_dim) {
  return head_dim >= 1 && head_dim <= kMaxDim ? (size_t)kGradBlocks * 2 * head_dim * sizeof(float) : 0;
}

jd_status_t jd_head_rope_grad(const jd_head_rope_grad_args_t* a, void* cuda_stream) {
  if (!a || !shape_args_ok(a->tokens, a->q_heads, a->k_heads, a->head_dim, a->dtype, a->rope) || !a->norm || !norm_ok(a->norm)) return JD_ERR_INVALID_ARG;
  HeadParams p = {};
  AxisMap m;
  if (!axes_ok(a->axes, a->rope.rot_dim / 2, &m) || !on4(a->q_weight_grad) || !on4(a->k_weight_grad)) return JD_ERR_INVALID_ARG;
  const bool weights = a->q_weight_grad || a->k_weight_grad;
  if (weights && (!a->workspace || !on4(a->workspace) || a->workspace_bytes < jd_head_rope_grad_workspace_bytes(a->head_dim))) return JD_ERR_INVALID_ARG;
  const int e = a->dtype == JD_DTYPE_F32 ? 4 : 2, D = a->head_dim;
  bool vec = vec_ok(a->rope.rot_dim, D);
  const Rows x[2] = {{a->q, a->q_stride}, {a->k, a->k_stride}}, g[2] = {{a->q_out_grad, a->q_out_grad_stride}, {a->k_out_grad, a->k_out_grad_stride}},
             d[2] = {{a->q_grad, a->q_grad_stride}, {a->k_grad, a->k_grad_stride}};
  for (int i = 0; i < 2 && a->tokens > 0; ++i) {
    const int heads = i ? a->k_heads : a->q_heads;
    if (heads == 0) continue;
    if (!rows_ok(x[i], heads, D, e) || !rows_ok(g[i], heads, D, e) || !rows_ok(d[i], heads, D, e)) return JD_ERR_INVALID_ARG;
    if ((d[i].p == g[i].p && step_of(d[i], heads, D) != step_of(g[i], heads, D)) || (d[i].p == x[i].p && step_of(d[i], heads, D) != step_of(x[i], heads, D)))
      return JD_ERR_INVALID_ARG;
    vec = vec && rows_on16(x[i], heads, D, e) && rows_on16(g[i], heads, D, e) && rows_on16(d[i], heads, D, e);
  }
  if (a->tokens > 0 && (!a->positions || !on4(a->positions))) return JD_ERR_INVALID_ARG;
  p.s = shape_of(&a->rope, a->norm, D);
  const Form f = form_of(p.s, vec);
  p.lanes = lanes_of(p.s, f);
  p.tokens = a->tokens; p.q_heads = a->q_heads; p.k_heads = a->k_heads;
  p.q = a->q; p.k = a->k; p.gq = a->q_out_grad; p.gk = a->k_out_grad; p.q_out = a->q_grad; p.k_out = a->k_grad;
  p.q_stride = step_of(x[0], a->q_heads, D); p.k_stride = step_of(x[1], a->k_heads, D);
  p.gq_stride = step_of(g[0], a->q_heads, D); p.gk_stride = step_of(g[1], a->k_heads, D);
  p.q_out_stride = step_of(d[0], a->q_heads, D); p.k_out_stride = step_of(d[1], a->k_heads, D);
  p.positions = a->positions;
  p.part = weights ? (float*)a->workspace : nullptr;
  p.per_block = tokens_per_block(p);
  cudaStream_t st = (cudaStream_t)cuda_stream;
  cudaError_t err = cudaSuccess;
  if (a->tokens > 0) err = by_form<Backward>(a->dtype, f, p, m, st);
  if (err == cudaSuccess && weights)     // without tokens: zeroes
    err = launch_chained(head_rope_weights_kernel, dim3((unsigned)((D + 31) / 32), 2u), dim3(kThreads), 0, st, (const float*)p.part,
                         a->tokens > 0 ? grad_blocks(a->tokens, p.per_block) : 0, D, a->q_weight_grad, a->k_weight_grad);
  if (err != cudaSuccess) { cudaGetLastError(); return JD_ERR_CUDA; }
  return JD_OK;
}

}  // extern "C"
