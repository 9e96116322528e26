// RMS norms of query and key heads and their rotary positions in one pass: alone (jd_head_rope), backwards (jd_head_rope_grad) and on
// the way into the cache (jd_cache_append_heads). A frequency takes one of a token's positions (time, row and column of an image, say).
//
//   r = 1 / sqrt(mean x^2 + eps),   n = r x,   y = R(n w)      R: the rotation of jd_rope.cu, amplitude included
//   g = R' dy (the transpose),      dx = r (g w - n mean(g w n)),      dw = sum over tokens and heads of g n
//
// Everything between the loads and the one rounding at the end is float32, so the floor is the bytes over the HBM rate. As many lanes as a head
// has pieces of 16 bytes (or, half a rotation apart, pairs of them) hold it in registers: a sum over the head is a few shuffles, and nothing is
// read twice. A block takes a few tokens: it forms the cosines and sines of their angles once, times the weights, and shares them among the heads through
// shared memory, while the first heads' loads are under way. Shapes that are no multiple of 16 bytes take single elements, a warp for a head.
// 16,384 tokens of 32 + 8 heads of 128, bf16: 58 us, 5.8 TB/s (issue slots 75 %); backwards, 8,192 tokens: 63.5 us, 4.0 TB/s (16 warps an SM, issue slots 56 %).
#include <algorithm>
#include <cmath>

#include "jd_rope.cuh"

namespace jd {
namespace {

constexpr int kThreads = 256;
constexpr int kTokensPerBlock = 4;        // scalar form
constexpr int kMaxDim = 256;
constexpr int kMaxAxes = 4;
constexpr int kGradBlocks = 1024;         // most blocks of the backward pass, each with a partial sum of dw
// Blocks on an SM, and the tokens whose angles a block forms at most, that many heads a group of lanes at a time: 16,384 tokens of 32 + 8 heads of 128 take
// 62 us with 8 tokens, 64 with 4 or 16, 75 with 2; backwards (8,192 tokens) 65 us with 16, 70 with 8, 76 with 32; with three blocks an SM, whose registers do not
// hold the sums, 89. Pairs side by side need half the registers: 72 us with three blocks (70 since), 84 with two, 73 with four.
constexpr int kForwardBlocks = 4, kForwardTokens = 8, kForwardTurns = 20;
constexpr int kBackwardTokens = 16, kBackwardTurns = 40;
constexpr int backward_blocks(bool half) { return half ? 2 : 3; }

enum Form { kScalar = 0, kHalfVec = 1, kPairVec = 2 };   // single elements; 8 + 8 of them half a rotation apart; 8 that hold 4 pairs

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

// ------------------------------------------------------------------------------------------ single elements
// A lane's part of a head: up to eight of its pairs, or of the elements behind them that pass through (32 lanes x 8: the widest head).
constexpr int kScalarUnits = kMaxDim / 32;

// elements of piece u; b < 0: there is none
__device__ __forceinline__ void elements_of(const HeadShape& s, int u, int& a, int& b) {
  if (u < s.half) {
    if (s.layout == JD_ROPE_HALF) { a = u; b = u + s.half; }
    else { a = 2 * u; b = a + 1; }
  } else { a = u + s.half; b = -1; }
}
__device__ __forceinline__ int scalar_units(const HeadShape& s) { return s.head_dim - s.half; }

__device__ __forceinline__ float sum_over(float v, int lanes) {
  for (int o = lanes >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// two sums at once, their shuffles' latencies beside one another: 8,192 tokens of 32 + 8 heads of 128 backwards 63.5 us, 64.8 one behind the other
__device__ __forceinline__ void sums_over(float& v, float& w, int lanes) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    if (o >= lanes) continue;
    const float x = __shfl_xor_sync(0xffffffffu, v, o), y = __shfl_xor_sync(0xffffffffu, w, o);
    v += x;
    w += y;
  }
}

// One head by a warp: y = R(n w).
template <typename T>
__device__ __forceinline__ void scalar_head(const T* x, T* y, const HeadShape& s, const float* w, const float2* cs, int lane) {
  const int units = scalar_units(s);
  float a[kScalarUnits], b[kScalarUnits], sum = 0.f;
#pragma unroll
  for (int k = 0; k < kScalarUnits; ++k) {
    const int u = lane + 32 * k;
    a[k] = b[k] = 0.f;
    if (u < units) {
      int ia, ib;
      elements_of(s, u, ia, ib);
      a[k] = to_float(x[ia]);
      if (ib >= 0) b[k] = to_float(x[ib]);
    }
    sum = fmaf(a[k], a[k], fmaf(b[k], b[k], sum));
  }
  const float r = s.normalize ? rsqrtf(sum_over(sum, 32) / (float)s.head_dim + s.eps) : 1.f;
  __syncwarp();                                          // y may be x
#pragma unroll
  for (int k = 0; k < kScalarUnits; ++k) {
    const int u = lane + 32 * k;
    if (u >= units) continue;
    int ia, ib;
    elements_of(s, u, ia, ib);
    float p = a[k], q = b[k];
    if (s.normalize) {
      p *= r * (w ? w[ia] : 1.f);
      if (ib >= 0) q *= r * (w ? w[ib] : 1.f);
    }
    if (ib >= 0) {
      const float2 t = cs[u];
      y[ia] = from_float(p * t.x - q * t.y, T());
      y[ib] = from_float(q * t.x + p * t.y, T());
    } else y[ia] = from_float(p, T());
  }
}

struct HeadParams {
  HeadShape s;
  int64_t tokens;
  int q_heads, k_heads, per_block, lanes;
  int units;                         // pieces of a head
  int q_blocks;                      // backward: blocks that take queries
  const void *q, *k, *gq, *gk;       // gradients of the outputs: backward alone
  void *q_out, *k_out;
  int64_t q_stride, k_stride, q_out_stride, k_out_stride, gq_stride, gk_stride;   // elements
  const int32_t* positions;          // [tokens][axes]
  int inverse;
  float* part;                       // backward: [blocks][head_dim] partial sums of dw; null: no weight gradients
};

// Cosines and sines of n tokens' angles, by the whole block.
__device__ __forceinline__ void fill_turns(const HeadParams& p, const AxisMap& m, float2 (*cs)[kMaxHalf], int64_t t0, int n, bool inverse) {
  const int half = p.s.half;
  for (int i = threadIdx.x; i < n * half; i += kThreads) {
    const int t = i / half, f = i - t * half;
    cs[t][f] = turn_of(__ldcg(p.positions + (t0 + t) * m.axes + m.of[f]), p.s.inv_freq[f], p.s.amplitude, inverse);
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) head_rope_scalar_kernel(const __grid_constant__ HeadParams p, const __grid_constant__ AxisMap m) {
  __shared__ float2 cs[kTokensPerBlock][kMaxHalf];
  pdl_wait();
  pdl_trigger();
  const HeadShape& s = p.s;
  const int64_t t0 = (int64_t)blockIdx.x * p.per_block;
  const int n = (int)min((int64_t)p.per_block, p.tokens - t0);
  fill_turns(p, m, cs, t0, n, p.inverse != 0);
  __syncthreads();
  const int heads = p.q_heads + p.k_heads, items = n * heads;
  for (int i = threadIdx.x >> 5; i < items; i += kThreads / 32) {
    const int t = i / heads, j = i - t * heads;
    const bool key = j >= p.q_heads;
    const int h = key ? j - p.q_heads : j;
    const T* x = reinterpret_cast<const T*>(key ? p.k : p.q) + (t0 + t) * (key ? p.k_stride : p.q_stride) + (int64_t)h * s.head_dim;
    T* y = reinterpret_cast<T*>(key ? p.k_out : p.q_out) + (t0 + t) * (key ? p.k_out_stride : p.q_out_stride) + (int64_t)h * s.head_dim;
    scalar_head<T>(x, y, s, key ? s.wk : s.wq, cs[t], threadIdx.x & 31);
  }
}

// Blocks [0, q_blocks) walk over the tokens' queries, the others over the keys, so that a lane's sums of g n, whose elements stay the same, are registers. Blocks
// leave partial sums, which head_rope_weights_kernel adds up in a fixed order: results repeat bit for bit.
template <typename T>
__global__ void __launch_bounds__(kThreads) head_rope_grad_scalar_kernel(const __grid_constant__ HeadParams p, const __grid_constant__ AxisMap m) {
  __shared__ float2 cs[kTokensPerBlock][kMaxHalf];
  __shared__ float s_sum[kThreads / 32][kMaxDim];
  pdl_wait();
  pdl_trigger();
  const HeadShape& s = p.s;
  const bool key = (int)blockIdx.x >= p.q_blocks;
  const int block = key ? blockIdx.x - p.q_blocks : blockIdx.x, blocks = key ? gridDim.x - p.q_blocks : p.q_blocks;
  const int heads = key ? p.k_heads : p.q_heads, units = scalar_units(s), lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const T* xs = reinterpret_cast<const T*>(key ? p.k : p.q);
  const T* gs = reinterpret_cast<const T*>(key ? p.gk : p.gq);
  T* ds = reinterpret_cast<T*>(key ? p.k_out : p.q_out);
  const float* w = key ? s.wk : s.wq;
  const int64_t x_stride = key ? p.k_stride : p.q_stride, g_stride = key ? p.gk_stride : p.gq_stride, d_stride = key ? p.k_out_stride : p.q_out_stride;
  float sum_a[kScalarUnits] = {}, sum_b[kScalarUnits] = {}, wa[kScalarUnits], wb[kScalarUnits];
#pragma unroll
  for (int k = 0; k < kScalarUnits; ++k) {
    const int u = lane + 32 * k;
    wa[k] = wb[k] = 1.f;
    if (u < units && w) {
      int ia, ib;
      elements_of(s, u, ia, ib);
      wa[k] = w[ia];
      if (ib >= 0) wb[k] = w[ib];
    }
  }
  const float per_dim = 1.f / (float)s.head_dim;
  for (int64_t t0 = (int64_t)block * p.per_block; t0 < p.tokens; t0 += (int64_t)blocks * p.per_block) {
    const int n = (int)min((int64_t)p.per_block, p.tokens - t0);
    __syncthreads();                                   // the last tokens' angles have been used
    fill_turns(p, m, cs, t0, n, false);
    __syncthreads();
    for (int i = warp; i < n * heads; i += kThreads / 32) {
      const int t = i / heads, h = i - t * heads;
      const T* x = xs + (t0 + t) * x_stride + (int64_t)h * s.head_dim;
      const T* g = gs + (t0 + t) * g_stride + (int64_t)h * s.head_dim;
      T* d = ds + (t0 + t) * d_stride + (int64_t)h * s.head_dim;
      float xa[kScalarUnits], xb[kScalarUnits], ga[kScalarUnits], gb[kScalarUnits], squares = 0.f, dot = 0.f;
#pragma unroll
      for (int k = 0; k < kScalarUnits; ++k) {
        const int u = lane + 32 * k;
        xa[k] = xb[k] = ga[k] = gb[k] = 0.f;
        if (u < units) {
          int ia, ib;
          elements_of(s, u, ia, ib);
          xa[k] = to_float(x[ia]);
          ga[k] = to_float(g[ia]);
          if (ib >= 0) {                               // the transpose: turned back
            xb[k] = to_float(x[ib]);
            const float v = to_float(g[ib]);
            const float2 c = cs[t][u];
            gb[k] = v * c.x - ga[k] * c.y;
            ga[k] = ga[k] * c.x + v * c.y;
          }
        }
        squares = fmaf(xa[k], xa[k], fmaf(xb[k], xb[k], squares));
        dot = fmaf(ga[k] * wa[k], xa[k], fmaf(gb[k] * wb[k], xb[k], dot));
      }
      sums_over(squares, dot, 32);
      const float r = rsqrtf(squares * per_dim + s.eps), mean = dot * r * per_dim;   // mean of g w n
      __syncwarp();                                    // d may be x or g
#pragma unroll
      for (int k = 0; k < kScalarUnits; ++k) {
        const int u = lane + 32 * k;
        if (u >= units) continue;
        int ia, ib;
        elements_of(s, u, ia, ib);
        const float na = xa[k] * r, nb = xb[k] * r;
        d[ia] = from_float(r * (ga[k] * wa[k] - na * mean), T());
        if (ib >= 0) d[ib] = from_float(r * (gb[k] * wb[k] - nb * mean), T());
        sum_a[k] = fmaf(ga[k], na, sum_a[k]);
        sum_b[k] = fmaf(gb[k], nb, sum_b[k]);
      }
    }
  }
  if (!p.part) return;
#pragma unroll
  for (int k = 0; k < kScalarUnits; ++k) {
    const int u = lane + 32 * k;
    if (u >= units) continue;
    int ia, ib;
    elements_of(s, u, ia, ib);
    s_sum[warp][ia] = sum_a[k];
    if (ib >= 0) s_sum[warp][ib] = sum_b[k];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < s.head_dim; i += kThreads) {
    float v = 0.f;
#pragma unroll
    for (int g = 0; g < kThreads / 32; ++g) v += s_sum[g][i];
    p.part[(int64_t)blockIdx.x * s.head_dim + i] = v;
  }
}

// ------------------------------------------------------------------------------------------ pieces of 16 bytes
// A lane's pairs of a head: 8 (elements 8 u .. and half a rotation behind them) or 4 (elements 8 u ..); pieces behind the turning ones pass
// through, and in the first form have no second half. Two float32 at a time.
template <typename T, bool kHalf> struct Piece8 {
  static constexpr int kPairs = kHalf ? 8 : 4, kTwos = kPairs / 2;
  static constexpr int kWords = (int)sizeof(T) / 2;       // 16-byte words of 8 elements
  static constexpr int kLoads = (kHalf ? 2 : 1) * kWords;
  static constexpr int kAhead = kLoads == 1 ? 3 : (kLoads == 2 ? 2 : 1);   // heads under way beside the one in hand
  struct Raw { uint4 w[kLoads]; };

  __device__ static __forceinline__ Raw load(const T* a, const T* b) {     // b: null where there is none
    Raw r;
#pragma unroll
    for (int i = 0; i < kWords; ++i) r.w[i] = reinterpret_cast<const uint4*>(a)[i];
    if constexpr (kHalf) {
#pragma unroll
      for (int i = 0; i < kWords; ++i) r.w[kWords + i] = b ? reinterpret_cast<const uint4*>(b)[i] : make_uint4(0u, 0u, 0u, 0u);
    }
    return r;
  }
  __device__ static __forceinline__ Raw none() {
    Raw r;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) r.w[i] = make_uint4(0u, 0u, 0u, 0u);
    return r;
  }
  __device__ static __forceinline__ void put(const Raw& r, T* a, T* b) {
#pragma unroll
    for (int i = 0; i < kWords; ++i) reinterpret_cast<uint4*>(a)[i] = r.w[i];
    if constexpr (kHalf) {
      if (b) {
#pragma unroll
        for (int i = 0; i < kWords; ++i) reinterpret_cast<uint4*>(b)[i] = r.w[kWords + i];
      }
    }
  }
  __device__ static __forceinline__ void eight(const uint4* w, float* v) {
    if constexpr (sizeof(T) == 2) {
      const uint32_t x[4] = {w[0].x, w[0].y, w[0].z, w[0].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(x[i] << 16); v[2 * i + 1] = __uint_as_float(x[i] & 0xFFFF0000u); }
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        v[4 * i] = __uint_as_float(w[i].x); v[4 * i + 1] = __uint_as_float(w[i].y);
        v[4 * i + 2] = __uint_as_float(w[i].z); v[4 * i + 3] = __uint_as_float(w[i].w);
      }
    }
  }
  // as packed pairs: a[i] holds the first elements of pairs 2 i and 2 i + 1
  __device__ static __forceinline__ void open(const Raw& r, uint64_t* a, uint64_t* b) {
    float v[8];
    eight(r.w, v);
    if constexpr (kHalf) {
      float u[8];
      eight(r.w + kWords, u);
#pragma unroll
      for (int i = 0; i < kTwos; ++i) { a[i] = pack2(v[2 * i], v[2 * i + 1]); b[i] = pack2(u[2 * i], u[2 * i + 1]); }
    } else {
#pragma unroll
      for (int i = 0; i < kTwos; ++i) { a[i] = pack2(v[4 * i], v[4 * i + 2]); b[i] = pack2(v[4 * i + 1], v[4 * i + 3]); }
    }
  }
  __device__ static __forceinline__ void store(T* ya, T* yb, const uint64_t* a, const uint64_t* b) {
    float v[8];
    if constexpr (kHalf) {
#pragma unroll
      for (int i = 0; i < kTwos; ++i) unpack2(a[i], v[2 * i], v[2 * i + 1]);
      store8(ya, v);
      if (yb) {
#pragma unroll
        for (int i = 0; i < kTwos; ++i) unpack2(b[i], v[2 * i], v[2 * i + 1]);
        store8(yb, v);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kTwos; ++i) { unpack2(a[i], v[4 * i], v[4 * i + 2]); unpack2(b[i], v[4 * i + 1], v[4 * i + 3]); }
      store8(ya, v);
    }
  }
};

// Where a lane stands: which group of lanes (token) and which piece of its head.
struct Place {
  int lanes, groups, group, unit;
  bool mine, turns;                                    // the head has this piece; the piece turns
  int a, b;                                            // first elements of the piece's halves; b < 0: none
};
template <bool kHalf> __device__ __forceinline__ Place place_of(const HeadShape& s, int lanes) {
  Place x;
  const int lane = threadIdx.x & 31, turning = s.half / (kHalf ? 8 : 4);
  x.lanes = lanes;
  x.groups = 32 / lanes;
  x.group = lane / lanes;
  x.unit = lane & (lanes - 1);
  x.mine = x.unit < turning + (s.head_dim - 2 * s.half) / 8;
  x.turns = x.unit < turning;
  x.a = x.turns || !kHalf ? 8 * x.unit : 2 * s.half + 8 * (x.unit - turning);
  x.b = kHalf && x.turns ? x.a + s.half : -1;
  if (!x.mine) x.unit = 0;                             // lanes without a piece read the first one's turns
  return x;
}
// What two pairs are turned by, in shared memory as the packed arithmetic takes it: pairs 2 i and 2 i + 1 of piece u at i x pieces + u, so that the lanes
// of a head read neighbouring words. Forward, with the weights in: y_a = r (x_a ca + x_b sb), y_b = r (x_b cb + x_a sa).
struct __align__(16) Two { uint64_t x, y; };

// An angle as a 64-bit fraction of a turn: position times frequency wraps by itself. The frequency's turns are a float64 product, rounded to 2^-63, and its error counts
// once for every position, as in turn_of; of the product the upper 32 bits are taken, 2^-32 of a turn. One integer product a token in place of turn_of's float64 operations.
__device__ __forceinline__ uint64_t turn_fraction(float freq) {
  const double turns = (double)freq * 0.15915494309189533577;   // 1 / (2 pi)
  return (uint64_t)(int64_t)__double2ll_rn((turns - rint(turns)) * 18446744073709551616.0 * 0.5) * 2u;
}
__device__ __forceinline__ float2 turn_by(int pos, uint64_t fraction, float amplitude) {
  const uint64_t t = (uint64_t)(int64_t)pos * fraction;
  float s, c;
  sincospif((float)(int)(uint32_t)(t >> 32) * 0x1p-31f, &s, &c);
  return make_float2(c * amplitude, s * amplitude);
}

// Elements of pair e of piece u; b < 0: there is none.
template <bool kHalf> __device__ __forceinline__ void pair_at(const HeadShape& s, int turning, int u, int e, int& a, int& b) {
  if (kHalf) {
    a = u < turning ? 8 * u + e : 2 * s.half + 8 * (u - turning) + e;
    b = u < turning ? a + s.half : -1;
  } else {
    a = 8 * u + 2 * e;
    b = a + 1;
  }
}
// Frequencies and weights are read by every block, by plain loads, which L1 serves: from L2 alone, thousands of blocks that read the same few lines wait for
// one another (1,373 tokens of 15 heads of 80: 15 us, 7 so).
// A thread's pair, the same for all tokens that it takes: threads t0, t0 + step, .. of the block's tokens.
struct PairJob {
  bool mine;
  int place;                                           // floats in front of it among a token's p (and q)
  int first, step, axis;
  uint64_t fraction;
  bool turns;
  int a, b;
};
template <bool kHalf> __device__ __forceinline__ PairJob pair_job(const HeadShape& s, const AxisMap& m, int units) {
  constexpr int kPairs = kHalf ? 8 : 4;
  const int pairs = kPairs * units, turning = s.half / kPairs;         // at most 256 pairs, never more than the block's threads
  PairJob x;
  x.step = kThreads / pairs;
  x.first = threadIdx.x / pairs;
  x.mine = x.first < x.step;
  const int j = threadIdx.x - x.first * pairs, u = j / kPairs, e = j - u * kPairs;
  x.place = ((e >> 1) * units + u) * 4 + (e & 1);      // its sine: two floats behind
  x.turns = u < turning;
  x.axis = x.turns ? (m.axes == 1 ? 0 : m.of[j]) : 0;
  x.fraction = x.mine && x.turns ? turn_fraction(s.inv_freq[j]) : 0ull;
  pair_at<kHalf>(s, turning, u, e, x.a, x.b);
  return x;
}
__device__ __forceinline__ float2 turn_of_job(const HeadShape& s, const PairJob& x, int pos, bool inverse) {
  if (!x.turns) return make_float2(1.f, 0.f);
  float2 c = turn_by(pos, x.fraction, s.amplitude);
  if (inverse) c.y = -c.y;
  return c;
}
__device__ __forceinline__ float2 weight_of_job(const PairJob& x, const float* w) {
  return make_float2(w && x.mine ? w[x.a] : 1.f, w && x.mine && x.b >= 0 ? w[x.b] : 1.f);
}
// the forward turn of a pair with its weights, to p (and q, `next` floats behind)
__device__ __forceinline__ void put_turn(float* p, int next, float2 c, float2 w) {
  p[0] = w.x * c.x;
  p[2] = -w.y * c.y;
  p[next] = w.y * c.x;
  p[next + 2] = w.x * c.y;
}

// Items of tokens x heads that a group of lanes takes, the same number of heads apart.
struct Walk {
  int t, h, step_t, step_h, heads;
  __device__ __forceinline__ void on() {
    t += step_t;
    h += step_h;
    if (h >= heads) { h -= heads; ++t; }
  }
};

// One head, a piece of it in this lane, (a, b) in place: y = R(n w). p, q: this piece's turns for the head's token.
template <typename P, bool kNorm>
__device__ __forceinline__ void turn_head(const Two* p, const Two* q, int units, const Place& x, float per_dim, float eps, uint64_t* a, uint64_t* b) {
  uint64_t r2 = 0ull;
  if constexpr (kNorm) {
    uint64_t sum = 0ull;
#pragma unroll
    for (int i = 0; i < P::kTwos; ++i) sum = fma2(b[i], b[i], fma2(a[i], a[i], sum));
    float s0, s1;
    unpack2(sum, s0, s1);
    const float r = rsqrtf(sum_over(s0 + s1, x.lanes) * per_dim + eps);
    r2 = pack2(r, r);
  }
#pragma unroll
  for (int i = 0; i < P::kTwos; ++i) {
    const Two t0 = p[i * units], t1 = q[i * units];
    if constexpr (kNorm) { a[i] = mul2(a[i], r2); b[i] = mul2(b[i], r2); }
    uint64_t ya = mul2(a[i], t0.x), yb = mul2(b[i], t1.x);
    if (x.turns) {                                     // a piece that passes through takes nothing of its neighbour, not even 0 x inf
      ya = fma2(b[i], t0.y, ya);
      yb = fma2(a[i], t1.y, yb);
    }
    a[i] = ya;
    b[i] = yb;
  }
}

// Group g of lanes takes items g, g + groups, .. of n tokens x heads; parts (blockIdx.y) of a token's heads spread few tokens over the SMs.
template <typename T, bool kHalf, bool kNorm>
__global__ void __launch_bounds__(kThreads, kForwardBlocks) head_rope_kernel(const __grid_constant__ HeadParams p, const __grid_constant__ AxisMap m) {
  using P = Piece8<T, kHalf>;
  extern __shared__ Two turns[];                       // [tokens][query, key heads][p, q][twos][pieces]
  pdl_wait();
  pdl_trigger();
  const HeadShape& s = p.s;
  const Place x = place_of<kHalf>(s, p.lanes);
  const int64_t t0 = (int64_t)blockIdx.x * p.per_block;
  const int n = (int)min((int64_t)p.per_block, p.tokens - t0), units = p.units, part = P::kTwos * units;
  const int groups = kThreads / x.lanes, group = threadIdx.x / x.lanes, heads = p.q_heads + p.k_heads;
  const float per_dim = 1.f / (float)s.head_dim;
  // this group's items: token t, head h of queries and keys, every `step` groups
  const int step = groups * gridDim.y, first = blockIdx.y * groups + group;
  Walk at = {first / heads, first % heads, step / heads, step % heads, heads}, ahead = at;
  auto place = [&](const Walk& i, bool out) {
    const bool key = i.h >= p.q_heads;
    const int64_t stride = key ? (out ? p.k_out_stride : p.k_stride) : (out ? p.q_out_stride : p.q_stride);
    return (T*)(key ? (out ? p.k_out : p.k) : (out ? p.q_out : p.q)) + (t0 + i.t) * stride + (int64_t)(key ? i.h - p.q_heads : i.h) * s.head_dim + x.a;
  };
  auto fetch = [&](const Walk& i) {
    if (!x.mine || i.t >= n) return P::none();
    const T* from = place(i, false);
    return P::load(from, x.b >= 0 ? from + (x.b - x.a) : nullptr);
  };
  typename P::Raw raw[P::kAhead];                      // under way beside the angles
#pragma unroll
  for (int k = 0; k < P::kAhead; ++k) { raw[k] = fetch(ahead); ahead.on(); }
  {
    const PairJob job = pair_job<kHalf>(s, m, units);
    const float2 wq = weight_of_job(job, kNorm ? s.wq : nullptr), wk = weight_of_job(job, kNorm ? s.wk : nullptr);
    if (job.mine)
      for (int t = job.first; t < n; t += job.step) {
        const float2 c = turn_of_job(s, job, __ldcg(p.positions + (t0 + t) * m.axes + job.axis), p.inverse != 0);
        float* to = reinterpret_cast<float*>(turns + 4 * t * part) + job.place;
        put_turn(to, 4 * part, c, wq);
        put_turn(to + 8 * part, 4 * part, c, wk);
      }
  }
  __syncthreads();
  while (__any_sync(0xffffffffu, at.t < n)) {
#pragma unroll
    for (int k = 0; k < P::kAhead; ++k) {
      uint64_t a[P::kTwos], b[P::kTwos];
      const Two* turn = turns + (4 * min(at.t, n - 1) + (at.h >= p.q_heads ? 2 : 0)) * part + x.unit;
      P::open(raw[k], a, b);
      raw[k] = fetch(ahead);
      turn_head<P, kNorm>(turn, turn + part, units, x, per_dim, s.eps, a, b);
      if (x.mine && at.t < n) {
        T* to = place(at, true);
        P::store(to, x.b >= 0 ? to + (x.b - x.a) : nullptr, a, b);
      }
      at.on();
      ahead.on();
    }
  }
}

// Blocks [0, q_blocks) walk over the tokens' queries, the others over the keys, so that a lane's sums of g n, whose elements stay the same, are registers.
template <typename T, bool kHalf>
__global__ void __launch_bounds__(kThreads, backward_blocks(kHalf)) head_rope_grad_kernel(const __grid_constant__ HeadParams p, const __grid_constant__ AxisMap m) {
  using P = Piece8<T, kHalf>;
  constexpr int kTwos = P::kTwos;
  extern __shared__ Two turns[];                       // [tokens][twos][pieces] cosines and sines, then the weights; in the end the warps' sums
  pdl_wait();
  pdl_trigger();
  const HeadShape& s = p.s;
  const bool key = (int)blockIdx.x >= p.q_blocks;
  const int block = key ? blockIdx.x - p.q_blocks : blockIdx.x, blocks = key ? gridDim.x - p.q_blocks : p.q_blocks;
  const int heads = key ? p.k_heads : p.q_heads, units = p.units, part = kTwos * units;
  const Place x = place_of<kHalf>(s, p.lanes);
  const int groups = kThreads / x.lanes, group = threadIdx.x / x.lanes;
  const T* xs = reinterpret_cast<const T*>(key ? p.k : p.q) + x.a;
  const T* gs = reinterpret_cast<const T*>(key ? p.gk : p.gq) + x.a;
  T* ds = reinterpret_cast<T*>(key ? p.k_out : p.q_out) + x.a;
  const float* w = key ? s.wk : s.wq;
  const int64_t x_stride = key ? p.k_stride : p.q_stride, g_stride = key ? p.gk_stride : p.gq_stride, d_stride = key ? p.k_out_stride : p.q_out_stride;
  const float per_dim = 1.f / (float)s.head_dim;
  const int step_t = groups / heads, step_h = groups - step_t * heads, t_first = group / heads, h_first = group - t_first * heads;
  uint64_t sum_a[kTwos], sum_b[kTwos];
#pragma unroll
  for (int k = 0; k < kTwos; ++k) sum_a[k] = sum_b[k] = 0ull;
  const PairJob job = pair_job<kHalf>(s, m, units);
  const Two* weights = turns + p.per_block * part + x.unit;
  if (job.mine && job.first == 0) {
    const float2 v = weight_of_job(job, w);
    float* to = reinterpret_cast<float*>(turns + p.per_block * part) + job.place;
    to[0] = v.x;
    to[2] = v.y;
  }
  for (int64_t t0 = (int64_t)block * p.per_block; t0 < p.tokens; t0 += (int64_t)blocks * p.per_block) {
    const int n = (int)min((int64_t)p.per_block, p.tokens - t0);
    int t = t_first, h = h_first;
    auto fetch = [&](const T* base, int64_t stride, int t, int h) {
      if (!x.mine || t >= n) return P::none();
      const T* from = base + (t0 + t) * stride + (int64_t)h * s.head_dim;
      return P::load(from, x.b >= 0 ? from + (x.b - x.a) : nullptr);
    };
    typename P::Raw raw_x = fetch(xs, x_stride, t, h), raw_g = fetch(gs, g_stride, t, h);
    __syncthreads();                                   // the last tokens' turns have been used
    if (job.mine)
      for (int t = job.first; t < n; t += job.step) {
        const float2 c = turn_of_job(s, job, __ldcg(p.positions + (t0 + t) * m.axes + job.axis), false);
        float* to = reinterpret_cast<float*>(turns + t * part) + job.place;
        to[0] = c.x;
        to[2] = c.y;
      }
    __syncthreads();
    while (__any_sync(0xffffffffu, t < n)) {
      int t_next = t + step_t, h_next = h + step_h;
      if (h_next >= heads) { h_next -= heads; ++t_next; }
      uint64_t va[kTwos], vb[kTwos], na[kTwos], nb[kTwos];
      P::open(raw_g, va, vb);
      P::open(raw_x, na, nb);
      raw_x = fetch(xs, x_stride, t_next, h_next);
      raw_g = fetch(gs, g_stride, t_next, h_next);
      uint64_t squares = 0ull, dot = 0ull;
      const Two* turn = turns + min(t, n - 1) * part + x.unit;
#pragma unroll
      for (int j = 0; j < kTwos; ++j) {
        squares = fma2(nb[j], nb[j], fma2(na[j], na[j], squares));
        if (x.turns) {                                 // the transpose: turned back
          const Two c = turn[j * units];
          const uint64_t q = fma2(vb[j], c.y, mul2(va[j], c.x));
          vb[j] = fma2(neg2(va[j]), c.y, mul2(vb[j], c.x));
          va[j] = q;
        }
        const Two v = weights[j * units];
        dot = fma2(mul2(vb[j], v.y), nb[j], fma2(mul2(va[j], v.x), na[j], dot));
      }
      float s0, s1, d0, d1;
      unpack2(squares, s0, s1);
      unpack2(dot, d0, d1);
      s0 += s1;
      d0 += d1;
      sums_over(s0, d0, x.lanes);
      // 0 for a group of lanes whose item is behind the last: its zeroes add nothing to the weights' sums, where 1 / sqrt(0) times them would be NaN
      const float r = t < n ? rsqrtf(s0 * per_dim + s.eps) : 0.f, mean = d0 * r * per_dim;   // mean of g w n
      const uint64_t r2 = pack2(r, r), mean2 = pack2(-mean, -mean);
#pragma unroll
      for (int j = 0; j < kTwos; ++j) {
        const Two v = weights[j * units];
        na[j] = mul2(na[j], r2);
        nb[j] = mul2(nb[j], r2);
        sum_a[j] = fma2(va[j], na[j], sum_a[j]);
        sum_b[j] = fma2(vb[j], nb[j], sum_b[j]);
        va[j] = mul2(r2, fma2(na[j], mean2, mul2(va[j], v.x)));
        vb[j] = mul2(r2, fma2(nb[j], mean2, mul2(vb[j], v.y)));
      }
      if (x.mine && t < n) {
        T* to = ds + (t0 + t) * d_stride + (int64_t)h * s.head_dim;
        P::store(to, x.b >= 0 ? to + (x.b - x.a) : nullptr, va, vb);
      }
      t = t_next;
      h = h_next;
    }
  }
  if (!p.part) return;
  // the warp's groups of lanes, then the block's warps
  __syncthreads();
  float* sums = reinterpret_cast<float*>(turns);       // [warps][head_dim]
#pragma unroll
  for (int k = 0; k < kTwos; ++k) {
    float a0, a1, b0, b1;
    unpack2(sum_a[k], a0, a1);
    unpack2(sum_b[k], b0, b1);
    for (int o = x.lanes; o < 32; o <<= 1) {
      a0 += __shfl_xor_sync(0xffffffffu, a0, o);
      a1 += __shfl_xor_sync(0xffffffffu, a1, o);
      b0 += __shfl_xor_sync(0xffffffffu, b0, o);
      b1 += __shfl_xor_sync(0xffffffffu, b1, o);
    }
    if (x.group == 0 && x.mine) {
      float* to = sums + (threadIdx.x >> 5) * s.head_dim;
      if constexpr (kHalf) {
        to[x.a + 2 * k] = a0;
        to[x.a + 2 * k + 1] = a1;
        if (x.b >= 0) { to[x.b + 2 * k] = b0; to[x.b + 2 * k + 1] = b1; }
      } else {
        to[x.a + 4 * k] = a0;
        to[x.a + 4 * k + 1] = b0;
        to[x.a + 4 * k + 2] = a1;
        to[x.a + 4 * k + 3] = b1;
      }
    }
  }
  __syncthreads();
  for (int e = threadIdx.x; e < s.head_dim; e += kThreads) {
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < kThreads / 32; ++k) v += sums[k * s.head_dim + e];
    p.part[(int64_t)blockIdx.x * s.head_dim + e] = v;
  }
}

// dw of 32 elements: eight warps take a block's partial sums each in turn, four under way.
__global__ void __launch_bounds__(kThreads) head_rope_weights_kernel(const float* part, int q_blocks, int blocks, int head_dim, float* dwq, float* dwk) {
  __shared__ float s_sum[kThreads / 32][32];
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, i = blockIdx.x * 32 + lane, end = blockIdx.y ? blocks : q_blocks;
  float v[4] = {};
  if (i < head_dim)
    for (int b = (blockIdx.y ? q_blocks : 0) + warp; b < end; b += 4 * (kThreads / 32)) {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (b + k * (kThreads / 32) < end) v[k] += __ldcg(part + (int64_t)(b + k * (kThreads / 32)) * head_dim + i);
    }
  s_sum[warp][lane] = (v[0] + v[1]) + (v[2] + v[3]);
  __syncthreads();
  float* out = blockIdx.y ? dwk : dwq;
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
  int units, per_block;          // pieces of a head; nodes of a block
  const int32_t* slots;
  const int32_t* depth;
  int64_t depth_stride;          // 0: shared
  const int32_t* num_nodes;
  const int32_t* positions;      // [B][T][axes]; null: seq_len + depth on every axis
  const char *k, *v, *q;
  char* q_out;
  int64_t k_stride, v_stride, q_stride, q_out_stride;   // bytes
};

// The place of token b T + t: its sequence's length, and the page of its row, held, in range and the sequence's alone (else -1, reported). slot < 0: the
// node is no token. The warp's lanes call it together, those of a group (`lane` of `lanes`) for one node.
struct NodePlace {
  int slot, len, page, row;
};
__device__ __forceinline__ NodePlace node_place(const AppendHeadsParams& p, int b, int t, int lane, int lanes) {
  const CacheView& c = p.c;
  NodePlace x;
  x.slot = slot_of(c, p.slots, b);
  x.page = -1;
  x.len = x.row = 0;
  if (x.slot >= 0 && p.num_nodes && t >= __ldcg(p.num_nodes + b)) x.slot = -1;
  bool named = false;                                  // by an earlier entry, which counts
  if (p.slots) {
    if (x.slot >= 0)
      for (int i = lane; i < b; i += lanes) named |= __ldcg(p.slots + i) == x.slot;
    for (int o = lanes >> 1; o > 0; o >>= 1) named |= __shfl_xor_sync(0xffffffffu, (int)named, o) != 0;
  }
  if (x.slot < 0) return x;
  int held;
  slot_state(c, x.slot, x.len, held);
  const int at = x.len + t;
  if ((at >> c.page_shift) < held) {
    x.page = __ldcg(c.table + (int64_t)x.slot * c.max_pages + (at >> c.page_shift));
    if (x.page < 0 || x.page >= c.pages || __ldcg(c.refs + x.page) > 1) x.page = -1;
  }
  x.row = at & (c.page_size - 1);
  if (named) x.slot = x.page = -1;
  if (x.page < 0) set_status(c.status, JD_ERR_BAD_INDEX);
  return x;
}

// A block takes a few nodes, whose places its warps look up side by side; few nodes: parts of their heads.
template <typename T, bool kHalf, bool kNorm>
__global__ void __launch_bounds__(kThreads, kForwardBlocks) append_heads_kernel(const __grid_constant__ AppendHeadsParams p, const __grid_constant__ AxisMap m) {
  using P = Piece8<T, kHalf>;
  extern __shared__ Two turns[];                       // [nodes][query, key heads][p, q][twos][pieces]
  __shared__ NodePlace s_node[kForwardTokens];
  pdl_wait();
  pdl_trigger();
  const HeadShape& s = p.s;
  const CacheView& c = p.c;
  const int t0 = blockIdx.x * p.per_block, n = min(p.per_block, p.B * p.T - t0);
  const Place x = place_of<kHalf>(s, p.lanes);
  const int groups = kThreads / x.lanes, group = threadIdx.x / x.lanes, units = p.units, part = P::kTwos * units;
  const float per_dim = 1.f / (float)s.head_dim;
  // a node's items: queries, keys, values
  const int first_v = p.q_heads + c.kv_heads, items = first_v + c.kv_heads, step = groups * gridDim.y, first = blockIdx.y * groups + group;
  Walk at = {first / items, first % items, step / items, step % items, items}, ahead = at;
  auto fetch = [&](const Walk& i) {
    if (!x.mine || i.t >= n) return P::none();
    const int64_t token = t0 + i.t;
    const char* base = i.h < p.q_heads ? p.q + token * p.q_stride : (i.h < first_v ? p.k + token * p.k_stride : p.v + token * p.v_stride);
    const T* from = reinterpret_cast<const T*>(base) + (int64_t)(i.h < p.q_heads ? i.h : (i.h < first_v ? i.h - p.q_heads : i.h - first_v)) * s.head_dim + x.a;
    return P::load(from, x.b >= 0 ? from + (x.b - x.a) : nullptr);
  };
  typename P::Raw raw[P::kAhead];                      // under way beside the nodes' places and angles
#pragma unroll
  for (int k = 0; k < P::kAhead; ++k) { raw[k] = fetch(ahead); ahead.on(); }
  for (int i = threadIdx.x >> 5; i < n; i += kThreads / 32) {
    const int b = (t0 + i) / p.T;
    const NodePlace node = node_place(p, b, t0 + i - b * p.T, threadIdx.x & 31, 32);
    if ((threadIdx.x & 31) == 0) s_node[i] = node;
  }
  const PairJob job = pair_job<kHalf>(s, m, units);
  const float2 wq = weight_of_job(job, kNorm ? s.wq : nullptr), wk = weight_of_job(job, kNorm ? s.wk : nullptr);
  __syncthreads();
  if (job.mine)
    for (int i = job.first; i < n; i += job.step) {
      const int token = t0 + i, b = token / p.T, t = token - b * p.T;
      const int pos = p.positions ? __ldcg(p.positions + (int64_t)token * m.axes + job.axis)
                                  : s_node[i].len + (p.depth ? __ldcg(p.depth + (int64_t)b * p.depth_stride + t) : t);
      const float2 cs = turn_of_job(s, job, pos, false);
      float* to = reinterpret_cast<float*>(turns + 4 * i * part) + job.place;
      put_turn(to, 4 * part, cs, wq);
      put_turn(to + 8 * part, 4 * part, cs, wk);
    }
  __syncthreads();
  while (__any_sync(0xffffffffu, at.t < n)) {
#pragma unroll
    for (int k = 0; k < P::kAhead; ++k) {
      const int i = min(at.t, n - 1);
      const NodePlace node = s_node[i];
      const bool query = at.h < p.q_heads, value = at.h >= first_v, live = x.mine && at.t < n && node.slot >= 0 && (query || node.page >= 0);
      T* to;
      if (query) to = reinterpret_cast<T*>(p.q_out + (int64_t)(t0 + i) * p.q_out_stride) + (int64_t)at.h * s.head_dim + x.a;
      else to = reinterpret_cast<T*>(value ? c.v : c.k) + page_row(c, p.layer, max(node.page, 0), value ? at.h - first_v : at.h - p.q_heads, node.row) * s.head_dim + x.a;
      T* to_b = x.b >= 0 ? to + (x.b - x.a) : nullptr;
      if (value && live) P::put(raw[k], to, to_b);     // bits as they are
      uint64_t a[P::kTwos], b[P::kTwos];
      P::open(raw[k], a, b);
      raw[k] = fetch(ahead);
      const Two* turn = turns + (4 * i + (query ? 0 : 2)) * part + x.unit;
      turn_head<P, kNorm>(turn, turn + part, units, x, per_dim, s.eps, a, b);
      if (!value && live) P::store(to, to_b, a, b);
      at.on();
      ahead.on();
    }
  }
}

// Single elements: a block for each node and part of its heads, a warp for a head.
template <typename T>
__global__ void __launch_bounds__(kThreads) append_heads_scalar_kernel(const __grid_constant__ AppendHeadsParams p, const __grid_constant__ AxisMap m) {
  __shared__ float2 cs[kMaxHalf];
  __shared__ NodePlace s_node;
  pdl_wait();
  pdl_trigger();
  const int b = blockIdx.x / p.T, t = blockIdx.x - b * p.T;
  const CacheView& c = p.c;
  const HeadShape& s = p.s;
  if (threadIdx.x < 32) {
    const NodePlace x = node_place(p, b, t, threadIdx.x, 32);
    if (threadIdx.x == 0) s_node = x;
  }
  __syncthreads();
  const NodePlace node = s_node;
  if (node.slot < 0) return;
  const int64_t token = (int64_t)b * p.T + t;
  const int pos = node.len + (p.depth ? __ldcg(p.depth + (int64_t)b * p.depth_stride + t) : t);
  for (int f = threadIdx.x; f < s.half; f += kThreads)
    cs[f] = turn_of(p.positions ? __ldcg(p.positions + token * m.axes + m.of[f]) : pos, s.inv_freq[f], s.amplitude, false);
  __syncthreads();
  if (node.page >= 0) {
    const int vunits = c.row_bytes / 16;
    for (int j = blockIdx.y * kThreads + threadIdx.x; j < c.kv_heads * vunits; j += gridDim.y * kThreads) {
      const int h = j / vunits, u = j - h * vunits;
      const char* src = p.v + token * p.v_stride + (int64_t)h * c.row_bytes;
      char* dst = c.v + page_row(c, p.layer, node.page, h, node.row) * c.row_bytes;
      reinterpret_cast<uint4*>(dst)[u] = reinterpret_cast<const uint4*>(src)[u];
    }
  }
  const int items = p.q_heads + (node.page < 0 ? 0 : c.kv_heads);
  const T* q = reinterpret_cast<const T*>(p.q + token * p.q_stride);
  T* qo = reinterpret_cast<T*>(p.q_out + token * p.q_out_stride);
  const T* k = reinterpret_cast<const T*>(p.k + token * p.k_stride);
  for (int i = blockIdx.y * (kThreads / 32) + (threadIdx.x >> 5); i < items; i += gridDim.y * (kThreads / 32)) {
    const bool key = i >= p.q_heads;
    const int h = key ? i - p.q_heads : i;
    T* y = key ? reinterpret_cast<T*>(c.k + page_row(c, p.layer, node.page, h, node.row) * c.row_bytes) : qo + h * s.head_dim;
    scalar_head<T>((key ? k : q) + h * s.head_dim, y, s, key ? s.wk : s.wq, cs, threadIdx.x & 31);
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
// pieces of a head, and lanes of a group: a power of two that holds them
int units_of(const HeadShape& s, Form f) { return f == kScalar ? 32 : s.half / (f == kHalfVec ? 8 : 4) + (s.head_dim - 2 * s.half) / 8; }
int lanes_of(int units) {
  int n = 1;
  while (n < units) n *= 2;
  return n;
}
int num_sms() {
  int device = 0, sms = 0;
  if (cudaGetDevice(&device) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device) != cudaSuccess) sms = 1;
  return sms;
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

template <template <typename, int> class Run, typename... Args>
cudaError_t by_form(int dtype, Form f, Args&&... args) {
  if (dtype == JD_DTYPE_F32) {
    if (f == kScalar) return Run<float, kScalar>::go(args...);
    return f == kHalfVec ? Run<float, kHalfVec>::go(args...) : Run<float, kPairVec>::go(args...);
  }
  if (f == kScalar) return Run<__nv_bfloat16, kScalar>::go(args...);
  return f == kHalfVec ? Run<__nv_bfloat16, kHalfVec>::go(args...) : Run<__nv_bfloat16, kPairVec>::go(args...);
}
template <int kForm> constexpr size_t part_of(int units) { return (kForm == kHalfVec ? 4 : 2) * units * sizeof(Two); }   // a token's p or q
// So many tokens a block that its groups of lanes have some heads each, for the angles to pay; few tokens: parts of their heads, spread over the SMs.
struct Shape {
  int per_block;
  dim3 grid;
};
Shape shape_for(int64_t tokens, int heads, int groups, size_t bytes_per_token) {
  Shape x;
  const int64_t wave = (int64_t)num_sms() * kForwardBlocks * groups, turns = std::min<int64_t>(kForwardTurns, (tokens * heads + wave - 1) / wave);
  const int64_t most = std::min<int64_t>(kForwardTokens, 40960 / (int64_t)bytes_per_token);   // within what every launch may have of shared memory
  x.per_block = (int)std::max<int64_t>(1, std::min<int64_t>(most, turns * groups / heads));
  const int64_t blocks = (tokens + x.per_block - 1) / x.per_block;
  const int64_t parts = std::max<int64_t>(1, std::min<int64_t>((heads * x.per_block + groups - 1) / groups, 2 * num_sms() / blocks));
  x.grid = dim3((unsigned)blocks, (unsigned)parts);
  return x;
}
template <typename T, int kForm> struct Forward {
  static cudaError_t go(HeadParams& p, const AxisMap& m, cudaStream_t st) {
    if constexpr (kForm == kScalar) {
      p.per_block = kTokensPerBlock;
      return launch_chained(head_rope_scalar_kernel<T>, dim3((unsigned)((p.tokens + p.per_block - 1) / p.per_block)), dim3(kThreads), 0, st, p, m);
    } else {
      const Shape x = shape_for(p.tokens, p.q_heads + p.k_heads, kThreads / p.lanes, 4 * part_of<kForm>(p.units));
      p.per_block = x.per_block;
      auto kernel = p.s.normalize ? head_rope_kernel<T, kForm == kHalfVec, true> : head_rope_kernel<T, kForm == kHalfVec, false>;
      return launch_chained(kernel, x.grid, dim3(kThreads), 4 * p.per_block * part_of<kForm>(p.units), st, p, m);
    }
  }
};
template <typename T, int kForm> struct Backward {
  static cudaError_t go(HeadParams& p, int* blocks, const AxisMap& m, cudaStream_t st) {
    const int groups = kThreads / p.lanes, heads = p.q_heads + p.k_heads;
    const int64_t most = std::min(kGradBlocks - 1, num_sms() * backward_blocks(kForm != kPairVec));
    // an even share of the tokens for every block, but three heads a group of lanes at least
    const int64_t more = std::max(p.q_heads, p.k_heads), least = (3 * groups + more - 1) / more;
    p.per_block = kForm == kScalar ? kTokensPerBlock
                                   : (int)std::max<int64_t>(1, std::min<int64_t>({(int64_t)kBackwardTokens, kBackwardTurns * groups / more, std::max(least, p.tokens / most)}));
    const int64_t chunks = (p.tokens + p.per_block - 1) / p.per_block;
    // blocks of one kind each, in the proportion of the heads
    auto share = [&](int n) { return n == 0 ? 0 : (int)std::min(chunks, std::max<int64_t>(1, (most * n + heads / 2) / heads)); };
    p.q_blocks = share(p.q_heads);
    *blocks = p.q_blocks + share(p.k_heads);
    if constexpr (kForm == kScalar) {
      return launch_chained(head_rope_grad_scalar_kernel<T>, dim3((unsigned)*blocks), dim3(kThreads), 0, st, p, m);
    } else {
      const size_t smem = std::max((p.per_block + 1) * part_of<kForm>(p.units), (size_t)kThreads / 32 * p.s.head_dim * sizeof(float));
      return launch_chained(head_rope_grad_kernel<T, kForm == kHalfVec>, dim3((unsigned)*blocks), dim3(kThreads), smem, st, p, m);
    }
  }
};
template <typename T, int kForm> struct Append {
  static cudaError_t go(AppendHeadsParams& p, const AxisMap& m, cudaStream_t st) {
    const int nodes = p.B * p.T;
    if constexpr (kForm == kScalar) {
      // few nodes: a head for each warp, spread over the SMs; many: a block for each node
      const int parts = nodes >= 512 ? 1 : std::max(1, std::min(8, (p.q_heads + p.c.kv_heads + kThreads / 32 - 1) / (kThreads / 32)));
      return launch_chained(append_heads_scalar_kernel<T>, dim3((unsigned)nodes, (unsigned)parts), dim3(kThreads), 0, st, p, m);
    } else {
      const Shape x = shape_for(nodes, p.q_heads + 2 * p.c.kv_heads, kThreads / p.lanes, 4 * part_of<kForm>(p.units));
      p.per_block = x.per_block;
      auto kernel = p.s.normalize ? append_heads_kernel<T, kForm == kHalfVec, true> : append_heads_kernel<T, kForm == kHalfVec, false>;
      return launch_chained(kernel, x.grid, dim3(kThreads), 4 * p.per_block * part_of<kForm>(p.units), st, p, m);
    }
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
  p.units = units_of(p.s, f);
  p.lanes = lanes_of(p.units);
  return by_form<Append>(dtype, f, p, m, st);
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
  p.units = units_of(p.s, f);
  p.lanes = lanes_of(p.units);
  p.tokens = a->tokens; p.q_heads = a->q_heads; p.k_heads = a->k_heads;
  p.q = a->q; p.k = a->k; p.q_out = a->q_out; p.k_out = a->k_out;
  p.q_stride = step_of(in[0], a->q_heads, D); p.k_stride = step_of(in[1], a->k_heads, D);
  p.q_out_stride = step_of(out[0], a->q_heads, D); p.k_out_stride = step_of(out[1], a->k_heads, D);
  p.positions = a->positions;
  p.inverse = a->inverse;
  if (by_form<Forward>(a->dtype, f, p, m, (cudaStream_t)cuda_stream) != cudaSuccess) { cudaGetLastError(); return JD_ERR_CUDA; }
  return JD_OK;
}

size_t jd_head_rope_grad_workspace_bytes(int32_t head_dim) {
  return head_dim >= 1 && head_dim <= kMaxDim ? (size_t)kGradBlocks * head_dim * sizeof(float) : 0;
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
  p.units = units_of(p.s, f);
  p.lanes = lanes_of(p.units);
  p.tokens = a->tokens; p.q_heads = a->q_heads; p.k_heads = a->k_heads;
  p.q = a->q; p.k = a->k; p.gq = a->q_out_grad; p.gk = a->k_out_grad; p.q_out = a->q_grad; p.k_out = a->k_grad;
  p.q_stride = step_of(x[0], a->q_heads, D); p.k_stride = step_of(x[1], a->k_heads, D);
  p.gq_stride = step_of(g[0], a->q_heads, D); p.gk_stride = step_of(g[1], a->k_heads, D);
  p.q_out_stride = step_of(d[0], a->q_heads, D); p.k_out_stride = step_of(d[1], a->k_heads, D);
  p.positions = a->positions;
  p.part = weights ? (float*)a->workspace : nullptr;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  cudaError_t err = cudaSuccess;
  int blocks = 0;
  if (a->tokens > 0) err = by_form<Backward>(a->dtype, f, p, &blocks, m, st);
  if (err == cudaSuccess && weights)     // without tokens: zeroes
    err = launch_chained(head_rope_weights_kernel, dim3((unsigned)((D + 31) / 32), 2u), dim3(kThreads), 0, st, (const float*)p.part, p.q_blocks, blocks, D,
                         a->q_weight_grad, a->k_weight_grad);
  if (err != cudaSuccess) { cudaGetLastError(); return JD_ERR_CUDA; }
  return JD_OK;
}

}  // extern "C"
