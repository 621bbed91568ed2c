// Windowed attention: formulas, arguments, and single rows.  A warp computes a row of a result in float32, whatever the
// sizes, strides and types; the kernels do this for rows that hidden places have spoiled.
//
// Query i sees key j iff j <= i and (i - j < window or j < sinks), both below the sequence's length n.
//   s_ij = scale q_i.k_j,  lse_i = log sum_j exp s_ij,  p_ij = exp(s_ij - lse_i),  o_i = sum_j p_ij v_j
//   dp_ij = do_i.v_j,  delta_i = do_i.o_i,  ds_ij = p_ij (dp_ij - delta_i)
//   dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum_{i,h} ds_ij q_i,  dv_j = sum_{i,h} p_ij do_i
// The lanes take 32 keys (queries) at a time for the products over the head's dimension, then the dimensions for the sums
// over those keys.  Only what is seen is read into a sum, so what a hidden place holds has no effect.
#pragma once

#include "elements.cuh"
#include "sm100.cuh"

namespace brace {

constexpr int kHeadMost = 256;             // longest head dimension
constexpr int kHeadLane = kHeadMost / 32;  // of a lane
// delta_i = do_i.o_i has the rounding of o_i in it, which a row of few keys does not average out.  Queries that see at most so
// many keys sum it anew, in float32, from p and dp.  2 x 4096 tokens, 4 heads of 64, error of dq before and after, and the time
// of the gradient: window 2, bfloat16 4.4e-3 -> 2.3e-3 (30 -> 33 us), float16 5.1e-4 -> 2.1e-4 (41 -> 46); window 512, bfloat16
// 2.52e-3 -> 2.40e-3 (48 -> 57); window 4096, where only the first queries see so few, 2.53e-3 -> 2.42e-3 (170 -> 171).
constexpr int kExactKeys = 640;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kTinyScale = 1.4e-45f;      // for a scale of 0: a score times it is less than 2^-20, a hidden one's -inf stays so

struct HeadRef {                           // element (b, t, h, d) lies at b * stride + t * ld + h * head + d
  void* p;
  int64_t ld, head, stride;
};

struct AttnArgs {
  HeadRef q, k, v, out, dout, dq, dk, dv;
  float* lse;                              // (b, h, t) at b * stride_lse + h * head_lse + t
  int64_t stride_lse, head_lse;
  float *delta, *shift;                    // [b][h][padded]: delta_i, and -log2(e) lse_i
  uint32_t* range;                         // [b][kv head][2]: bits of the largest |do| and |v|
  float* part;                             // float32 sums: of dv and dk [b][kv head][parts][dv, dk][rows][D], before that of dq
                                           // [b][head][tile][rows][D]
  int64_t padded;                          // tokens, rounded up to 64
  int first_tiles, pieces, parts;          // parts: the shared tiles' pieces, then (of long sums) one of each other tile
  const int32_t* lengths;
  int batch, tokens, heads, kv_heads, share, dim, window, sinks;
  float scale;
};

__device__ __forceinline__ int attn_length(const AttnArgs& p, int b) {
  return p.lengths ? max(0, min(p.lengths[b], p.tokens)) : p.tokens;
}
template <typename T>
__device__ __forceinline__ T* head_row(const HeadRef& r, int b, int t, int h) {
  return static_cast<T*>(r.p) + b * r.stride + t * r.ld + h * r.head;
}
__device__ __forceinline__ float& attn_lse(const AttnArgs& p, int b, int h, int t) {
  return p.lse[b * p.stride_lse + h * p.head_lse + t];
}
__device__ __forceinline__ int64_t attn_delta(const AttnArgs& p, int b, int h, int t) {
  return ((int64_t)b * p.heads + h) * p.padded + t;
}

template <typename T>
__device__ __forceinline__ float dot_row(const T* a, const T* b, int dim) {
  float s = 0.f;
#pragma unroll 8
  for (int d = 0; d < dim; ++d) s = fmaf(to_f32(a[d]), to_f32(b[d]), s);
  return s;
}
// acc[r] += x * row[lane + 32 r]
template <typename T>
__device__ __forceinline__ void add_row(float (&acc)[kHeadLane], float x, const T* row, int dim) {
#pragma unroll
  for (int r = 0; r < kHeadLane; ++r) {
    const int d = (int)(threadIdx.x & 31) + 32 * r;
    if (d < dim) acc[r] = fmaf(x, to_f32(row[d]), acc[r]);
  }
}
template <typename T>
__device__ __forceinline__ void put_row(T* row, const float (&acc)[kHeadLane], float factor, int dim) {
#pragma unroll
  for (int r = 0; r < kHeadLane; ++r) {
    const int d = (int)(threadIdx.x & 31) + 32 * r;
    if (d < dim) row[d] = from_f32<T>(acc[r] * factor);
  }
}

// The keys that query i sees: the first `first` ones and those from `lo` to i.
struct Seen {
  int first, lo, count;
  __device__ __forceinline__ Seen(const AttnArgs& p, int i) {
    lo = max(0, i - p.window + 1);
    first = min(p.sinks, lo);
    count = first + i - lo + 1;
  }
  __device__ __forceinline__ int key(int t) const { return t < first ? t : lo + t - first; }
};

template <typename T>
__device__ __forceinline__ void forward_row(const AttnArgs& p, int b, int h, int i, int n) {
  const int lane = threadIdx.x & 31, g = h / p.share;
  float acc[kHeadLane] = {};
  if (i >= n) {
    put_row(head_row<T>(p.out, b, i, h), acc, 0.f, p.dim);
    if (p.lse && lane == 0) attn_lse(p, b, h, i) = -INFINITY;
    return;
  }
  const Seen seen(p, i);
  const T* q = head_row<const T>(p.q, b, i, h);
  float top = -INFINITY, total = 0.f;
  for (int t0 = 0; t0 < seen.count; t0 += 32) {
    const int some = min(32, seen.count - t0);
    float s = -INFINITY;
    if (lane < some) s = p.scale * dot_row(q, head_row<const T>(p.k, b, seen.key(t0 + lane), g), p.dim);
    float m = s;
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    m = fmaxf(m, top);
    const float shift = m == -INFINITY ? 0.f : m, keep = expf(top - shift);
    const float x = lane < some ? expf(s - shift) : 0.f;
    top = m;
    total = total * keep + x;
#pragma unroll
    for (int r = 0; r < kHeadLane; ++r) acc[r] *= keep;
    for (int t = 0; t < some; ++t)
      add_row(acc, __shfl_sync(0xffffffffu, x, t), head_row<const T>(p.v, b, seen.key(t0 + t), g), p.dim);
  }
  for (int o = 16; o; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
  put_row(head_row<T>(p.out, b, i, h), acc, 1.f / total, p.dim);
  if (p.lse && lane == 0) attn_lse(p, b, h, i) = top + logf(total);
}

template <typename T>
__device__ __forceinline__ void dq_row(const AttnArgs& p, int b, int h, int i, int n) {
  const int lane = threadIdx.x & 31, g = h / p.share;
  float acc[kHeadLane] = {};
  if (i >= n) {
    put_row(head_row<T>(p.dq, b, i, h), acc, 0.f, p.dim);
    return;
  }
  const Seen seen(p, i);
  const T *q = head_row<const T>(p.q, b, i, h), *dout = head_row<const T>(p.dout, b, i, h);
  const float lse = attn_lse(p, b, h, i), delta = p.delta[attn_delta(p, b, h, i)];
  for (int t0 = 0; t0 < seen.count; t0 += 32) {
    const int some = min(32, seen.count - t0);
    float ds = 0.f;
    if (lane < some) {
      const int j = seen.key(t0 + lane);
      const float s = p.scale * dot_row(q, head_row<const T>(p.k, b, j, g), p.dim);
      ds = expf(s - lse) * (dot_row(dout, head_row<const T>(p.v, b, j, g), p.dim) - delta);
    }
    for (int t = 0; t < some; ++t)
      add_row(acc, __shfl_sync(0xffffffffu, ds, t), head_row<const T>(p.k, b, seen.key(t0 + t), g), p.dim);
  }
  put_row(head_row<T>(p.dq, b, i, h), acc, p.scale, p.dim);
}

template <typename T>
__device__ __forceinline__ void dkv_row(const AttnArgs& p, int b, int g, int j, int n, bool put_k = true, bool put_v = true) {
  const int lane = threadIdx.x & 31;
  float dk[kHeadLane] = {}, dv[kHeadLane] = {};
  const int end = j >= n ? j : j < p.sinks || p.window > n - j ? n : j + p.window;
  const T *k = head_row<const T>(p.k, b, j, g), *v = head_row<const T>(p.v, b, j, g);
  for (int h = g * p.share; h < (g + 1) * p.share; ++h)
    for (int i0 = j; i0 < end; i0 += 32) {
      const int some = min(32, end - i0), i = i0 + lane;
      float x = 0.f, ds = 0.f;
      if (lane < some) {
        x = expf(p.scale * dot_row(head_row<const T>(p.q, b, i, h), k, p.dim) - attn_lse(p, b, h, i));
        ds = x * (dot_row(head_row<const T>(p.dout, b, i, h), v, p.dim) - p.delta[attn_delta(p, b, h, i)]);
      }
      for (int t = 0; t < some; ++t) {
        add_row(dv, __shfl_sync(0xffffffffu, x, t), head_row<const T>(p.dout, b, i0 + t, h), p.dim);
        add_row(dk, __shfl_sync(0xffffffffu, ds, t), head_row<const T>(p.q, b, i0 + t, h), p.dim);
      }
    }
  if (put_k) put_row(head_row<T>(p.dk, b, j, g), dk, p.scale, p.dim);
  if (put_v) put_row(head_row<T>(p.dv, b, j, g), dv, 1.f, p.dim);
}

}  // namespace brace
