// Rotary positions, alone (jd_rope) and on the way into the cache (jd_cache_append).
//
//   (a, b) -> amplitude (a cos t - b sin t, b cos t + a sin t),   t = position x inv_freq
//
// Every element is read and written once, so the floor is the bytes over the HBM rate. A block takes a few tokens
// whole: it forms the cosines and sines of their angles once (float64 product with 1 / 2 pi, reduced to half a turn
// before it is rounded to float32: a far position times a float32 frequency has more bits than a float32 angle keeps)
// and shares them among the heads through shared memory. Then every thread turns 16-byte pieces of a head: two of
// them half a rotation apart, or one that holds whole pairs, by layout.
#include <algorithm>
#include <cmath>

#include "jd_rope.cuh"

namespace jd {
namespace {

constexpr int kRopeThreads = 256;
constexpr int kRopeUnitsPerThread = 4;
constexpr int kTokensPerBlock = 8;

// One unit of a head: the unit-th piece that turns, or behind those a piece that passes through.
// kVec: pieces of 8 elements, rot_dim % 16 == 0, head_dim % 8 == 0 and 16-byte rows; else single pairs / elements.
template <typename T, bool kVec>
__device__ __forceinline__ void turn_unit(const T* x, T* y, int unit, const float2* cs, int half, int layout, bool copy_rest) {
  constexpr int kW = kVec ? 8 : 1;
  if (layout == JD_ROPE_HALF) {
    const int n = half / kW;
    if (unit < n) {
      const int i = unit * kW;
      float a[kW], b[kW], p[kW], q[kW];
      if constexpr (kVec) { load8(x + i, a); load8(x + i + half, b); }
      else { a[0] = to_float(x[i]); b[0] = to_float(x[i + half]); }
#pragma unroll
      for (int k = 0; k < kW; ++k) {
        const float2 t = cs[i + k];
        p[k] = a[k] * t.x - b[k] * t.y;
        q[k] = b[k] * t.x + a[k] * t.y;
      }
      if constexpr (kVec) { store8(y + i, p); store8(y + i + half, q); }
      else { y[i] = from_float(p[0], T()); y[i + half] = from_float(q[0], T()); }
      return;
    }
    unit -= n;
  } else {
    const int n = kVec ? half / 4 : half;
    if (unit < n) {
      if constexpr (kVec) {
        float a[8], p[8];
        load8(x + unit * 8, a);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float2 t = cs[unit * 4 + k];
          p[2 * k] = a[2 * k] * t.x - a[2 * k + 1] * t.y;
          p[2 * k + 1] = a[2 * k + 1] * t.x + a[2 * k] * t.y;
        }
        store8(y + unit * 8, p);
      } else {
        const float a = to_float(x[2 * unit]), b = to_float(x[2 * unit + 1]);
        const float2 t = cs[unit];
        y[2 * unit] = from_float(a * t.x - b * t.y, T());
        y[2 * unit + 1] = from_float(b * t.x + a * t.y, T());
      }
      return;
    }
    unit -= n;
  }
  if (copy_rest) {
    const int i = 2 * half + unit * kW;
    if constexpr (kVec) {   // bits as they are
      const uint4* s = reinterpret_cast<const uint4*>(x + i);
      uint4* d = reinterpret_cast<uint4*>(y + i);
#pragma unroll
      for (int k = 0; k < (int)sizeof(T) / 2; ++k) d[k] = s[k];
    } else {
      y[i] = x[i];
    }
  }
}

__host__ __device__ __forceinline__ int units_of_head(int head_dim, int half, int layout, bool vec) {
  const int turning = layout == JD_ROPE_HALF ? (vec ? half / 8 : half) : (vec ? half / 4 : half);
  return turning + (head_dim - 2 * half) / (vec ? 8 : 1);
}

// 16,384 tokens x 40 heads x 128, bf16: 58 us, 5.8 TB/s (half layout), 65 us (interleaved; 76 without the register limit, which keeps eight
// blocks of the narrow type on an SM). Loading several pieces ahead of the angles took the registers of two of them: 68 us.
template <typename T, bool kVec>
__global__ void __launch_bounds__(kRopeThreads, sizeof(T) == 2 ? 8 : 1) rope_kernel(const T* x, T* out, int64_t tokens, int heads,
                                                            int head_dim, int64_t x_stride, int64_t out_stride,
                                                            const int32_t* positions, const float* inv_freq,
                                                            int half, int layout, float amplitude, int inverse, int per_block) {
  __shared__ float2 cs[kTokensPerBlock][kMaxHalf];
  pdl_wait();
  pdl_trigger();
  const int64_t t0 = (int64_t)blockIdx.x * per_block;
  const int n = (int)min((int64_t)per_block, tokens - t0);
  for (int i = threadIdx.x; i < n * half; i += kRopeThreads) {
    const int t = i / half, f = i - t * half;
    cs[t][f] = turn_of(__ldcg(positions + t0 + t), __ldcg(inv_freq + f), amplitude, inverse != 0);
  }
  __syncthreads();
  const int units = units_of_head(head_dim, half, layout, kVec), per_token = units * heads;
  for (int i = threadIdx.x; i < n * per_token; i += kRopeThreads) {
    const int t = i / per_token, j = i - t * per_token, h = j / units, u = j - h * units;
    turn_unit<T, kVec>(x + (t0 + t) * x_stride + (int64_t)h * head_dim, out + (t0 + t) * out_stride + (int64_t)h * head_dim, u,
                       cs[t], half, layout, out != x);
  }
}

struct AppendParams {
  CacheView c;
  int B, T, layer, q_heads;
  const int32_t* slots;
  const int32_t* depth;
  int64_t depth_stride;          // 0: shared
  const int32_t* num_nodes;
  const char *k, *v, *q;
  char* q_out;
  int64_t k_stride, v_stride, q_stride, q_out_stride;   // bytes
  const float* inv_freq;         // null: nothing turns
  int half, layout;
  float amplitude;
  bool copy_q;                   // q_out is not q
};

// One block per node and part of its heads. Blocks of the same node repeat the angles; with few nodes that is what
// spreads the work over the SMs, with many there is one block per node.
template <typename T, bool kVec>
__global__ void __launch_bounds__(kRopeThreads) append_kernel(AppendParams p) {
  __shared__ float2 cs[kMaxHalf];
  __shared__ int dup;
  pdl_wait();
  pdl_trigger();
  const int b = blockIdx.x / p.T, t = blockIdx.x - b * p.T;
  const CacheView& c = p.c;
  const int slot = slot_of(c, p.slots, b);
  if (slot < 0) return;
  if (p.num_nodes && t >= __ldcg(p.num_nodes + b)) return;
  if (threadIdx.x == 0) dup = 0;
  __syncthreads();
  if (p.slots)
    for (int i = threadIdx.x; i < b; i += kRopeThreads)
      if (__ldcg(p.slots + i) == slot) dup = 1;
  int len, held;
  slot_state(c, slot, len, held);
  const int at = len + t;
  const int pos = len + (p.depth ? __ldcg(p.depth + (int64_t)b * p.depth_stride + t) : t);
  for (int f = threadIdx.x; f < p.half; f += kRopeThreads) cs[f] = turn_of(pos, __ldcg(p.inv_freq + f), p.amplitude, false);
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
  const int64_t token = (int64_t)b * p.T + t;
  const int units = units_of_head(c.head_dim, p.half, p.layout, kVec);
  const int vunits = c.row_bytes / 16;
  const int nq = p.q_heads * units, nk = page < 0 ? 0 : c.kv_heads * units, nv = page < 0 ? 0 : c.kv_heads * vunits;
  const T* q = reinterpret_cast<const T*>(p.q + token * p.q_stride);
  T* qo = reinterpret_cast<T*>(p.q_out + token * p.q_out_stride);
  const T* k = reinterpret_cast<const T*>(p.k + token * p.k_stride);
  for (int i = blockIdx.y * kRopeThreads + threadIdx.x; i < nq + nk + nv; i += gridDim.y * kRopeThreads) {
    if (i < nq) {
      const int h = i / units;
      turn_unit<T, kVec>(q + h * c.head_dim, qo + h * c.head_dim, i - h * units, cs, p.half, p.layout, p.copy_q);
    } else if (i < nq + nk) {
      const int j = i - nq, h = j / units;
      T* dst = reinterpret_cast<T*>(c.k + page_row(c, p.layer, page, h, row) * c.row_bytes);
      turn_unit<T, kVec>(k + h * c.head_dim, dst, j - h * units, cs, p.half, p.layout, true);
    } else {
      const int j = i - nq - nk, h = j / vunits, u = j - h * vunits;
      const char* src = p.v + token * p.v_stride + (int64_t)h * c.row_bytes;
      char* dst = c.v + page_row(c, p.layer, page, h, row) * c.row_bytes;
      reinterpret_cast<uint4*>(dst)[u] = reinterpret_cast<const uint4*>(src)[u];
    }
  }
}

bool rope_ok(const jd_rope_t& r, int head_dim) {
  return r.inv_freq && (reinterpret_cast<uintptr_t>(r.inv_freq) & 3) == 0 && r.rot_dim >= 2 && r.rot_dim % 2 == 0 &&
         r.rot_dim <= head_dim && r.rot_dim <= 2 * kMaxHalf && (r.layout == JD_ROPE_HALF || r.layout == JD_ROPE_INTERLEAVED) &&
         std::isfinite(r.amplitude);
}

template <typename T>
cudaError_t launch_rope(const jd_rope_args_t& a, int64_t xs, int64_t os, cudaStream_t st) {
  const bool vec = vec_ok(a.rope.rot_dim, a.head_dim) && (reinterpret_cast<uintptr_t>(a.x) % 16 == 0) &&
                   (reinterpret_cast<uintptr_t>(a.out) % 16 == 0) && xs * sizeof(T) % 16 == 0 && os * sizeof(T) % 16 == 0;
  const int half = a.rope.rot_dim / 2;
  const int units = units_of_head(a.head_dim, half, a.rope.layout, vec) * a.heads;
  // about kRopeUnitsPerThread pieces per thread, so that a block's angles pay for themselves
  const int per_block = std::max(1, std::min(kTokensPerBlock, kRopeThreads * kRopeUnitsPerThread / std::max(1, units)));
  const int64_t blocks = (a.tokens + per_block - 1) / per_block;
  return launch_chained(vec ? rope_kernel<T, true> : rope_kernel<T, false>, dim3((unsigned)blocks), dim3(kRopeThreads), 0, st, (const T*)a.x,
                        (T*)a.out, a.tokens, a.heads, a.head_dim, xs, os, a.positions, a.rope.inv_freq, half, a.rope.layout, a.rope.amplitude,
                        a.inverse, per_block);
}

}  // namespace

cudaError_t run_append(const CacheView& c, const jd_append_args_t& a, int q_heads, int dtype, cudaStream_t st) {
  const int e = dtype == JD_DTYPE_F32 ? 4 : 2;
  AppendParams p;
  p.c = c;
  p.B = a.B; p.T = a.tree.nodes; p.layer = a.layer;
  p.q_heads = a.q ? q_heads : 0;
  p.slots = a.slots;
  p.depth = a.tree.depth;
  p.depth_stride = a.tree.per_seq ? a.tree.nodes : 0;
  p.num_nodes = a.tree.num_nodes;
  p.k = (const char*)a.k; p.v = (const char*)a.v; p.q = (const char*)a.q; p.q_out = (char*)a.q_out;
  auto bytes = [&](int64_t s, int heads) { return (s ? s : (int64_t)heads * c.head_dim) * e; };
  p.k_stride = bytes(a.k_stride, c.kv_heads); p.v_stride = bytes(a.v_stride, c.kv_heads);
  p.q_stride = bytes(a.q_stride, q_heads); p.q_out_stride = bytes(a.q_out_stride, q_heads);
  p.inv_freq = a.rope ? a.rope->inv_freq : nullptr;
  p.half = a.rope ? a.rope->rot_dim / 2 : 0;
  p.layout = a.rope ? a.rope->layout : JD_ROPE_HALF;
  p.amplitude = a.rope ? a.rope->amplitude : 1.f;
  p.copy_q = a.q != a.q_out;
  const bool vec = vec_ok(2 * p.half, c.head_dim);
  const int units = (p.q_heads + c.kv_heads) * units_of_head(c.head_dim, p.half, p.layout, vec) + c.kv_heads * c.row_bytes / 16;
  const int nodes = a.B * a.tree.nodes;
  // few nodes: one piece per thread, spread over the SMs; many: a block per node
  const int parts = nodes >= 512 ? 1 : std::max(1, std::min(8, (units + kRopeThreads - 1) / kRopeThreads));
  const dim3 grid((unsigned)nodes, (unsigned)parts);
  auto kernel = dtype == JD_DTYPE_F32 ? (vec ? append_kernel<float, true> : append_kernel<float, false>)
                                      : (vec ? append_kernel<__nv_bfloat16, true> : append_kernel<__nv_bfloat16, false>);
  return launch_chained(kernel, grid, dim3(kRopeThreads), 0, st, p);
}

bool rope_valid(const jd_rope_t& r, int head_dim) { return rope_ok(r, head_dim); }

}  // namespace jd

using namespace jd;

extern "C" {

jd_status_t jd_rope_frequencies(int32_t rot_dim, double base, int32_t scaling, double factor, double original_len,
                                double low, double high, float* inv_freq, float* amplitude) {
  if (!inv_freq || rot_dim < 2 || rot_dim % 2 != 0 || rot_dim > 2 * kMaxHalf || !(base > 1.0) || !std::isfinite(base)) return JD_ERR_INVALID_ARG;
  if (scaling < JD_ROPE_SCALE_NONE || scaling > JD_ROPE_SCALE_YARN) return JD_ERR_INVALID_ARG;
  if (scaling != JD_ROPE_SCALE_NONE && !(factor >= 1.0 && std::isfinite(factor))) return JD_ERR_INVALID_ARG;
  const bool blend = scaling == JD_ROPE_SCALE_BANDS || scaling == JD_ROPE_SCALE_YARN;
  if (blend && !(original_len >= 1.0 && std::isfinite(original_len) && low > 0.0 && high > low && std::isfinite(high)))
    return JD_ERR_INVALID_ARG;
  const double two_pi = 6.28318530717958647692;
  const int half = rot_dim / 2;
  // index (a real number) whose frequency makes `turns` turns in original_len
  auto index_of = [&](double turns) { return rot_dim * std::log(original_len / (turns * two_pi)) / (2.0 * std::log(base)); };
  double first = 0.0, last = 0.0;
  if (scaling == JD_ROPE_SCALE_YARN) {
    first = std::fmax(std::floor(index_of(high)), 0.0);
    last = std::fmin(std::ceil(index_of(low)), rot_dim - 1.0);   // may lie behind the last index, half - 1: the blend then ends part of the way
    if (last <= first) last = first + 0.001;
  }
  for (int i = 0; i < half; ++i) {
    const double f = std::pow(base, -2.0 * i / rot_dim);
    double keep = 1.0;    // weight of the unscaled frequency
    if (scaling == JD_ROPE_SCALE_LINEAR) keep = 0.0;
    if (scaling == JD_ROPE_SCALE_BANDS) keep = std::fmin(1.0, std::fmax(0.0, (original_len * f / two_pi - low) / (high - low)));
    if (scaling == JD_ROPE_SCALE_YARN) keep = 1.0 - std::fmin(1.0, std::fmax(0.0, (i - first) / (last - first)));
    inv_freq[i] = (float)(scaling == JD_ROPE_SCALE_NONE ? f : f * (keep + (1.0 - keep) / factor));
  }
  if (amplitude) *amplitude = scaling == JD_ROPE_SCALE_YARN ? (float)(0.1 * std::log(factor) + 1.0) : 1.f;
  return JD_OK;
}

jd_status_t jd_rope(const jd_rope_args_t* a, void* cuda_stream) {
  if (!a || a->tokens < 0 || a->tokens > 0x7FFFFFFF || a->heads < 1 || a->head_dim < 1 || a->head_dim > 256) return JD_ERR_INVALID_ARG;
  if (a->dtype != JD_DTYPE_F32 && a->dtype != JD_DTYPE_BF16) return JD_ERR_INVALID_ARG;
  if (!rope_ok(a->rope, a->head_dim) || a->x_stride < 0 || a->out_stride < 0) return JD_ERR_INVALID_ARG;
  const int64_t dense = (int64_t)a->heads * a->head_dim;
  const int64_t xs = a->x_stride ? a->x_stride : dense, os = a->out_stride ? a->out_stride : dense;
  if (xs < dense || os < dense || dense > 0x7FFFFFFF / 8) return JD_ERR_INVALID_ARG;
  if (a->tokens == 0) return JD_OK;
  const uintptr_t e = a->dtype == JD_DTYPE_F32 ? 4 : 2;
  if (!a->x || !a->out || !a->positions) return JD_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(a->x) % e || reinterpret_cast<uintptr_t>(a->out) % e ||
      reinterpret_cast<uintptr_t>(a->positions) % 4)
    return JD_ERR_INVALID_ARG;
  if (a->x == a->out && xs != os) return JD_ERR_INVALID_ARG;
  const cudaError_t err = a->dtype == JD_DTYPE_F32 ? launch_rope<float>(*a, xs, os, (cudaStream_t)cuda_stream)
                                                   : launch_rope<__nv_bfloat16>(*a, xs, os, (cudaStream_t)cuda_stream);
  if (err != cudaSuccess) { cudaGetLastError(); return JD_ERR_CUDA; }
  return JD_OK;
}

}  // extern "C"
