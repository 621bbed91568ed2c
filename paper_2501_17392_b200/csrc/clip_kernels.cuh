// Every client's gradient norm over many tensors, and the gradients clipped by it.
//
// norm_c = sqrt(sum over the client's tensors of sum x^2), f_c = min(1, max_norm / (norm_c + eps)), out = f_c x.
// Bound by memory.  A call is a chain of launches; each clips some clients (whose values the launch before it has just
// read, so that they come from L2) and sums the squares of the next ones.  A client's elements are shared out evenly over
// its CTAs, each of which leaves one sum; who clips adds them up, in one order.  Squares are summed in float32 over the 8
// or 16 values that a thread has at a time, and by this in float64; where a float32 sum leaves its comfortable range
// (overflow, squares lost to underflow) those values are squared in float64.
#pragma once

#include "elements.cuh"
#include "sm100.cuh"

namespace brace {

constexpr int kClipThreads = 256;
constexpr int kClipUnit = 2048;      // elements: what a client's elements are shared out by
constexpr int kClipNarrow = 1024;    // rows of a strided tensor shorter than this are walked element by element

struct ClipTensor {
  const void* in;
  void* out;
  int64_t rows, cols;                // rows is 1 where both sides are one run of elements
  int64_t ld_in, ld_out, stride_in, stride_out;
  int64_t unit0, row_units;          // first unit of this tensor; units of a row (0: rows are walked together)
  int32_t in_type, out_type;
};

struct ClipArgs {
  double* part;                      // [client][parts]
  float* norms;
  int64_t units, parts, part0;       // of this list; parts of all lists, and the first one of this list
  int32_t clip_first, clip_count, sum_first, count;
  float max_norm, eps;
  int32_t zero_bad;                  // a client whose norm is not finite gets zeros
};

template <int CAP>
struct ClipList {
  ClipTensor t[CAP];
};

// What the 256 threads do with a run of n elements: sum of squares of this thread's (CLIP = false), or out = factor x.
template <typename TI, typename TO, int V, bool CLIP>
__device__ __forceinline__ double clip_run(const TI* in, TO* out, int64_t n, float factor, bool zero) {
  constexpr int U = 16 / V < 2 ? 2 : 16 / V;      // loads under way in a thread: 16 elements
  double acc = 0.0;
  for (int64_t i0 = 0; i0 < n; i0 += kClipThreads * V * U) {
    Pack<TI, V> x[U];
    const int64_t at = i0 + threadIdx.x * V;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (at + u * kClipThreads * V < n) x[u].load(in + at + u * kClipThreads * V);
    if (CLIP) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        Pack<TO, V> y;
#pragma unroll
        for (int k = 0; k < V; ++k) y.t[k] = from_f32<TO>(zero ? 0.f : to_f32(x[u].t[k]) * factor);
        if (at + u * kClipThreads * V < n) y.store_stream(out + at + u * kClipThreads * V);
      }
    } else {
      float q = 0.f;
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (at + u * kClipThreads * V < n)
#pragma unroll
          for (int k = 0; k < V; ++k) q = fmaf(to_f32(x[u].t[k]), to_f32(x[u].t[k]), q);
      if (q >= 1e-20f && q <= 1e37f) {
        acc += q;
      } else {
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (at + u * kClipThreads * V < n)
#pragma unroll
            for (int k = 0; k < V; ++k) {
              const double d = to_f32(x[u].t[k]);
              acc = fma(d, d, acc);
            }
      }
    }
  }
  return acc;
}

// A run whose ends may lie anywhere: wide words where the addresses of both sides allow it, after the elements before the
// first boundary.
template <typename TI, typename TO, bool CLIP>
__device__ __forceinline__ double clip_span(const TI* in, TO* out, int64_t n, float factor, bool zero) {
  constexpr int V = sizeof(TI) == 4 && (!CLIP || sizeof(TO) == 4) ? 4 : 8;
  constexpr int kAlignIn = V * sizeof(TI) < 16 ? V * sizeof(TI) : 16, kAlignOut = V * sizeof(TO) < 16 ? V * sizeof(TO) : 16;
  int64_t head = ((kAlignIn - ((uintptr_t)in & (kAlignIn - 1))) & (kAlignIn - 1)) / sizeof(TI);
  if (head > n) head = n;
  if (CLIP && ((uintptr_t)(out + head) & (kAlignOut - 1))) return clip_run<TI, TO, 1, CLIP>(in, out, n, factor, zero);
  const int64_t body = (n - head) / V * V, tail = n - head - body;
  double acc = 0.0;
  if (threadIdx.x < head) acc += clip_run<TI, TO, 1, CLIP>(in, out, head, factor, zero);
  acc += clip_run<TI, TO, V, CLIP>(in + head, out + head, body, factor, zero);
  if (threadIdx.x < tail) acc += clip_run<TI, TO, 1, CLIP>(in + head + body, out + head + body, tail, factor, zero);
  return acc;
}

// Units [u0, u1) of one tensor of client c.  Calls, not copies: the kernel has one for each pair of types.
template <typename TI, typename TO, bool CLIP>
__device__ __noinline__ double clip_units(const ClipTensor& t, int64_t c, int64_t u0, int64_t u1, float factor, bool zero) {
  const TI* in = static_cast<const TI*>(t.in) + c * t.stride_in;
  TO* out = CLIP ? static_cast<TO*>(t.out) + c * t.stride_out : nullptr;
  double acc = 0.0;
  if (t.row_units) {
    for (int64_t u = u0; u < u1;) {
      const int64_t row = u / t.row_units, k = u - row * t.row_units;
      const int64_t stop = u1 - u < t.row_units - k ? k + u1 - u : t.row_units;   // of this row
      const int64_t a = k * kClipUnit, b = stop * kClipUnit < t.cols ? stop * kClipUnit : t.cols;
      acc += clip_span<TI, TO, CLIP>(in + row * t.ld_in + a, CLIP ? out + row * t.ld_out + a : nullptr, b - a, factor, zero);
      u += stop - k;
    }
    return acc;
  }
  const int64_t n = t.rows * t.cols, end = u1 * kClipUnit < n ? u1 * kClipUnit : n;
  for (int64_t e = u0 * kClipUnit + threadIdx.x; e < end; e += kClipThreads) {
    const int64_t row = e / t.cols, col = e - row * t.cols;
    const float x = to_f32(in[row * t.ld_in + col]);
    if (CLIP)
      out[row * t.ld_out + col] = from_f32<TO>(zero ? 0.f : x * factor);
    else
      acc = fma((double)x, (double)x, acc);
  }
  return acc;
}

template <bool CLIP>
__device__ __forceinline__ double clip_tensor(const ClipTensor& t, int64_t c, int64_t u0, int64_t u1, float factor, bool zero) {
  auto in_as = [&](auto to) {
    using TO = decltype(to);
    if (t.in_type == kTypeF32) return clip_units<float, TO, CLIP>(t, c, u0, u1, factor, zero);
    if (t.in_type == kTypeBF16) return clip_units<__nv_bfloat16, TO, CLIP>(t, c, u0, u1, factor, zero);
    return clip_units<__half, TO, CLIP>(t, c, u0, u1, factor, zero);
  };
  if (!CLIP || t.out_type == kTypeF32) return in_as(float{});
  if (t.out_type == kTypeBF16) return in_as(__nv_bfloat16{});
  return in_as(__half{});
}

// Sum over the CTA, in every thread.
__device__ __forceinline__ double clip_block_sum(double v, double* cell) {
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if ((threadIdx.x & 31) == 0) cell[threadIdx.x >> 5] = v;
  __syncthreads();
  v = 0.0;
  for (int w = 0; w < kClipThreads / 32; ++w) v += cell[w];
  return v;
}

__device__ __forceinline__ double clip_total(const ClipArgs& p, int64_t c, double* cell) {
  double v = 0.0;
  for (int64_t k = threadIdx.x; k < p.parts; k += kClipThreads) v += p.part[c * p.parts + k];
  return clip_block_sum(v, cell);
}

// CTAs (x, y): y below clip_count clips client clip_first + y, the others sum client sum_first + y - clip_count.
template <int CAP>
__global__ void __launch_bounds__(kClipThreads) clip_kernel(const ClipArgs p, const __grid_constant__ ClipList<CAP> list) {
  __shared__ double cell[kClipThreads / 32];
  grid_trigger();
  grid_wait();
  const bool clip = (int)blockIdx.y < p.clip_count;
  const int64_t c = clip ? p.clip_first + (int)blockIdx.y : p.sum_first + (int)blockIdx.y - p.clip_count;
  float factor = 1.f;
  bool zero = false;
  if (clip) {
    const double norm = sqrt(clip_total(p, c, cell));
    const double f = norm == 0.0 ? 1.0 : (double)p.max_norm / (norm + (double)p.eps);
    factor = f > 1.0 ? 1.f : (float)f;
    zero = p.zero_bad && !isfinite(norm);
    if (p.norms && threadIdx.x == 0 && blockIdx.x == 0 && p.part0 == 0) p.norms[c] = (float)norm;
  }
  int64_t u = p.units * blockIdx.x / gridDim.x;
  const int64_t end = p.units * (blockIdx.x + 1) / gridDim.x;
  int i = 0;
  constexpr int kFirst = CAP >= 256 ? 256 : CAP >= 32 ? 32 : 8;
  static_assert(CAP <= 2 * kFirst, "the steps reach every tensor");
  for (int step = kFirst; step; step >>= 1)          // the last tensor that begins at u or before
    if (i + step < p.count && list.t[i + step].unit0 <= u) i += step;
  double acc = 0.0;
  for (; u < end; ++i) {
    const int64_t stop = i + 1 < p.count && list.t[i + 1].unit0 < end ? list.t[i + 1].unit0 : end;
    if (stop <= u) continue;                         // a tensor without elements
    const ClipTensor& t = list.t[i];
    if (!clip)
      acc += clip_tensor<false>(t, c, u - t.unit0, stop - t.unit0, 1.f, false);
    else if (factor != 1.f || zero || t.in != t.out)
      clip_tensor<true>(t, c, u - t.unit0, stop - t.unit0, factor, zero);
    u = stop;
  }
  if (!clip) {
    acc = clip_block_sum(acc, cell);
    if (threadIdx.x == 0) p.part[c * p.parts + p.part0 + blockIdx.x] = acc;
  }
}

__global__ void __launch_bounds__(kClipThreads) clip_norms_kernel(const ClipArgs p) {
  __shared__ double cell[kClipThreads / 32];
  grid_trigger();
  grid_wait();
  const double total = clip_total(p, blockIdx.x, cell);
  if (threadIdx.x == 0) p.norms[blockIdx.x] = (float)sqrt(total);
}

}  // namespace brace
