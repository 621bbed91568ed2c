// Every client's gradient norm over many tensors, and the gradients clipped by it.
//
// norm_c = sqrt(sum over the client's tensors of sum x^2), f_c = min(1, max_norm / (norm_c + eps)), out = f_c x.
// Bound by memory where values are not 0: every value is read for its square, and read again once the norm is known.  A launch sums (a client's
// elements shared out evenly over CTAs, each of which leaves one sum), a second one clips, the other way round, so that it
// begins with what is still in L2.
// 50 clients of 11.7 M float32 values (2.3 GB): 327 us to sum (7.2 TB/s) and 1092 in all (6.4 TB/s on what is read twice
// and written once; a copy moves 6.6).  Tried and not kept: chains of launches that clip the clients which the launch before
// summed, from L2 (1117 us where two passes took 1113: 4 to 5 us a launch are lost, and clients of 47 MB do not stay there); one cooperative launch
// that holds 224 KB an SM in shared memory between its sum and its clipping (1496 us from registers, 1668 by bulk copies:
// all CTAs wait for one another once a client).
// Squares are summed in float32 over at most 16 values that a thread has at a time, and beyond that in float64, in one
// order; where a float32 sum leaves its comfortable range (overflow, squares lost to underflow) those values are squared
// in float64.  So are 16 zeros, at the price of instructions: the norms of 8 clients' tables of 50,000 x 768 take 176 us dense, 235
// with all rows but 8192 zero and 306 all zero (bfloat16 96, 227, 274), clipping into float32 rows 572, 624 and 694 (422, 541, 586).
#pragma once

#include "elements.cuh"
#include "sm100.cuh"

namespace brace {

constexpr int kClipThreads = 256, kClipResident = 2;   // of a CTA that only sums or only clips; CTAs of an SM
constexpr int kClusterMost = 8;                        // CTAs of a cluster that has a client of few elements
constexpr int kClipUnit = 2048;      // elements: what a client's elements are shared out by
constexpr int kClipNarrow = 1024;    // rows of a strided tensor shorter than this are walked element by element

struct ClipTensor {
  const void* in;
  void* out;
  int64_t rows, cols;                // rows is 1 where both sides are one run of elements
  int64_t ld_in, ld_out, stride_in, stride_out;
  int64_t unit0, row_units;          // first unit of this tensor; units of a row (0: rows are walked together)
};

struct ClipArgs {
  double* part;                      // [client][parts]
  float* norms;
  int64_t units, parts, part0;       // of this list; parts of all lists, and the first one of this list
  int32_t count;                     // tensors of this list
  float max_norm, eps;
  int32_t zero_bad;                  // a client whose norm is not finite gets zeros
};

template <int CAP>
struct ClipList {
  ClipTensor t[CAP];
};

// A thread's values whose float32 sum of squares left its comfortable range, once more: `pieces` pieces of `width` values.
template <typename T>
__device__ __noinline__ double squares64(const T* x, int pieces, int width, int distance) {
  double acc = 0.0;
  for (int u = 0; u < pieces; ++u)
    for (int k = 0; k < width; ++k) {
      const double d = to_f32(x[u * distance + k]);
      acc = fma(d, d, acc);
    }
  return acc;
}

// What is done with the elements: their squares are summed, or they are clipped.
template <bool CLIP_>
struct ClipPass {
  static constexpr bool CLIP = CLIP_;
  float factor, rest;                // what a value is multiplied by, one after the other (clip_factor)
  bool zero;
  double acc;
};

// U pieces of V values of this thread, the pieces kThreads * V apart, those from piece `count` on not there (ALL: all are).
template <typename TI, typename TO, int V, int U, bool ALL, typename P>
__device__ __forceinline__ void clip_pieces(P& p, const TI* in, TO* out, int count) {
  constexpr int kApart = kClipThreads * V;
  Pack<TI, V> x[U];
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (ALL || u < count) x[u].load(in + u * kApart);
  if (P::CLIP) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      Pack<TO, V> y;
#pragma unroll
      for (int k = 0; k < V; ++k) y.t[k] = from_f32<TO>(p.zero ? 0.f : to_f32(x[u].t[k]) * p.factor * p.rest);
      if (ALL || u < count) y.store_stream(out + u * kApart);
    }
  } else {
    constexpr int kGroup = 16 / V < U ? 16 / V : U;      // pieces of a float32 sum
#pragma unroll
    for (int u0 = 0; u0 < U; u0 += kGroup) {
      float q = 0.f;
#pragma unroll
      for (int u = u0; u < u0 + kGroup; ++u)
        if (ALL || u < count)
#pragma unroll
          for (int k = 0; k < V; ++k) q = fmaf(to_f32(x[u].t[k]), to_f32(x[u].t[k]), q);
      if (q >= 1e-20f && q <= 1e37f)
        p.acc += q;
      else if (ALL || u0 < count)
        p.acc += squares64(in + u0 * kApart, ALL ? kGroup : min(kGroup, count - u0), V, kApart);
    }
  }
}

// A run of n elements (a multiple of V).
template <typename TI, typename TO, int V, typename P>
__device__ __forceinline__ void clip_run(P& p, const TI* in, TO* out, int64_t n) {
  constexpr int U = V == 1 ? 8 : 128 / (V * (int)sizeof(TI));     // 128 bytes under way in a thread
  constexpr int kStep = kClipThreads * V * U;
  in += threadIdx.x * V;
  out += threadIdx.x * V;
  for (; n >= kStep; n -= kStep, in += kStep, out += kStep) clip_pieces<TI, TO, V, U, true>(p, in, out, U);
  const int rest = (int)n - (int)threadIdx.x * V;
  if (rest > 0) clip_pieces<TI, TO, V, U, false>(p, in, out, (rest + kClipThreads * V - 1) / (kClipThreads * V));
}

// A run whose ends may lie anywhere: wide words where the addresses of both sides allow it, after the elements before the
// first boundary.
template <typename TI, typename TO, typename P>
__device__ __forceinline__ void clip_span(P& p, const TI* in, TO* out, int64_t n) {
  // neighbouring threads take neighbouring words of the wider type, so that a warp's access is one run of memory
  constexpr int V = sizeof(TI) == 4 || sizeof(TO) == 4 ? 4 : 8;
  constexpr uintptr_t kIn = V * sizeof(TI) - 1, kOut = V * sizeof(TO) - 1;
  int head = (int)(((kIn + 1 - ((uintptr_t)in & kIn)) & kIn) / sizeof(TI));
  if (head > n) head = (int)n;
  if (P::CLIP && ((uintptr_t)(out + head) & kOut)) {
    clip_run<TI, TO, 1>(p, in, out, n);
    return;
  }
  const int64_t body = (n - head) / V * V;
  const int tail = (int)(n - head - body), t = (int)threadIdx.x;
  clip_run<TI, TO, V>(p, in + head, out + head, body);
  if (t < head + tail) {     // fewer than 16 elements: one a thread
    const int64_t at = t < head ? t : body + t;
    clip_pieces<TI, TO, 1, 1, true>(p, in + at, out + at, 1);
  }
}

// Units [u0, u1) of one tensor of client c.
template <typename TI, typename TO, typename P>
__device__ __forceinline__ void clip_units(P& p, const ClipTensor& t, int64_t c, int64_t u0, int64_t u1) {
  const TI* in = static_cast<const TI*>(t.in) + c * t.stride_in;
  TO* out = static_cast<TO*>(t.out) + c * t.stride_out;     // summing does not look at it
  if (t.row_units) {
    while (u0 < u1) {
      const int64_t row = t.rows > 1 ? u0 / t.row_units : 0, k = u0 - row * t.row_units;
      const int64_t stop = u1 - u0 < t.row_units - k ? k + u1 - u0 : t.row_units;   // of this row
      const int64_t a = k * kClipUnit, b = stop * kClipUnit < t.cols ? stop * kClipUnit : t.cols;
      clip_span(p, in + row * t.ld_in + a, out + row * t.ld_out + a, b - a);
      u0 += stop - k;
    }
    return;
  }
  const int64_t n = t.rows * t.cols, end = u1 * kClipUnit < n ? u1 * kClipUnit : n;
  for (int64_t e = u0 * kClipUnit + threadIdx.x; e < end; e += kClipThreads) {
    const int64_t row = e / t.cols, col = e - row * t.cols;
    clip_pieces<TI, TO, 1, 1, true>(p, in + row * t.ld_in + col, out + row * t.ld_out + col, 1);
  }
}

// f(tensor, first unit of it, end) for each of the list's tensors that has some of the units [u, end).
template <int CAP, typename F>
__device__ __forceinline__ void clip_walk(const ClipList<CAP>& list, int count, int64_t u, int64_t end, F&& f) {
  int i = 0;
  constexpr int kFirst = CAP >= 256 ? 256 : CAP >= 32 ? 32 : 8;
  static_assert(CAP <= 2 * kFirst, "the steps reach every tensor");
  for (int step = kFirst; step; step >>= 1)          // the last tensor that begins at u or before
    if (i + step < count && list.t[i + step].unit0 <= u) i += step;
  for (; u < end; ++i) {
    const int64_t stop = i + 1 < count && list.t[i + 1].unit0 < end ? list.t[i + 1].unit0 : end;
    const ClipTensor& t = list.t[i];
    f(t, u - t.unit0, stop - t.unit0);
    u = stop;
  }
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

// Sum of client c's parts, in every thread.
__device__ __forceinline__ double clip_total(const ClipArgs& a, int64_t c, double* cell) {
  double v = 0.0;
  for (int64_t k = threadIdx.x; k < a.parts; k += kClipThreads) v += a.part[c * a.parts + k];
  return clip_block_sum(v, cell);
}

__device__ __forceinline__ void clip_factor(const ClipArgs& a, double norm, ClipPass<true>& p) {
  double f = norm == 0.0 ? 1.0 : (double)a.max_norm / (norm + (double)a.eps);
  // float32 has fewer bits below 2^-126, where the norm of values near its largest ones takes the factor: half of its exponent
  // then goes into a power of two.  What the first product loses below 2^-126 is less than the result can hold.
  const int half = f < 0x1p-100 && f > 0.0 ? ilogb(f) / 2 : 0;
  f = ldexp(f, -half);
  p.rest = (float)ldexp(1.0, half);
  p.factor = f > 1.0 ? 1.f : (float)f;      // NaN stays
  p.zero = a.zero_bad && !isfinite(norm);
}

// All tensors of a launch are of the types TI and TO.  grid: (CTAs of a client, clients)
template <typename TI, int CAP>
__global__ void __launch_bounds__(kClipThreads, kClipResident) clip_sum_kernel(const ClipArgs a, const __grid_constant__ ClipList<CAP> list) {
  __shared__ double cell[kClipThreads / 32];
  grid_trigger();
  grid_wait();
  const int64_t c = blockIdx.y;
  ClipPass<false> p = {};
  clip_walk(list, a.count, a.units * blockIdx.x / gridDim.x, a.units * (blockIdx.x + 1) / gridDim.x,
            [&](const ClipTensor& t, int64_t u0, int64_t u1) { clip_units<TI, TI>(p, t, c, u0, u1); });
  const double sum = clip_block_sum(p.acc, cell);
  if (threadIdx.x == 0) a.part[c * a.parts + a.part0 + blockIdx.x] = sum;
}

template <typename TI, typename TO, int CAP>
__global__ void __launch_bounds__(kClipThreads, kClipResident) clip_apply_kernel(const ClipArgs a, const __grid_constant__ ClipList<CAP> list) {
  __shared__ double cell[kClipThreads / 32];
  grid_trigger();
  grid_wait();
  const int64_t c = gridDim.y - 1 - blockIdx.y, x = gridDim.x - 1 - blockIdx.x;
  const double norm = sqrt(clip_total(a, c, cell));
  ClipPass<true> p = {};
  clip_factor(a, norm, p);
  if (a.norms && threadIdx.x == 0 && x == 0 && a.part0 == 0) a.norms[c] = (float)norm;
  clip_walk(list, a.count, a.units * x / gridDim.x, a.units * (x + 1) / gridDim.x, [&](const ClipTensor& t, int64_t u0, int64_t u1) {
    if (p.factor != 1.f || p.zero || t.in != t.out) clip_units<TI, TO>(p, t, c, u0, u1);
  });
}

// Clients of few elements in one launch: a cluster has a client, its CTAs tell one another their sums.  What a CTA reads twice
// is its own.  grid: (CTAs of a cluster, clients)
template <typename TI, typename TO, int CAP>
__global__ void __launch_bounds__(kClipThreads, kClipResident) clip_cluster_kernel(const ClipArgs a, const __grid_constant__ ClipList<CAP> list) {
  __shared__ double cell[kClipThreads / 32];
  __shared__ double sums[kClusterMost];
  cluster_arrive();
  grid_trigger();
  grid_wait();
  const int64_t c = blockIdx.y, from = a.units * blockIdx.x / gridDim.x, to = a.units * (blockIdx.x + 1) / gridDim.x;
  ClipPass<false> s = {};
  clip_walk(list, a.count, from, to, [&](const ClipTensor& t, int64_t u0, int64_t u1) { clip_units<TI, TI>(s, t, c, u0, u1); });
  const double sum = clip_block_sum(s.acc, cell);
  cluster_wait();     // all CTAs have begun: their shared memory is theirs
  if (threadIdx.x < gridDim.x) st_cluster_f64(map_to_rank(smem_addr(sums + cluster_rank()), threadIdx.x), sum);
  cluster_sync();
  double total = 0.0;
  for (int k = 0; k < (int)gridDim.x; ++k) total += sums[k];
  const double norm = sqrt(total);
  ClipPass<true> p = {};
  clip_factor(a, norm, p);
  if (a.norms && threadIdx.x == 0 && blockIdx.x == 0) a.norms[c] = (float)norm;
  clip_walk(list, a.count, from, to, [&](const ClipTensor& t, int64_t u0, int64_t u1) {
    if (p.factor != 1.f || p.zero || t.in != t.out) clip_units<TI, TO>(p, t, c, u0, u1);
  });
}

__global__ void __launch_bounds__(kClipThreads) clip_norms_kernel(const ClipArgs a) {
  __shared__ double cell[kClipThreads / 32];
  grid_trigger();
  grid_wait();
  const double total = clip_total(a, blockIdx.x, cell);
  if (threadIdx.x == 0) a.norms[blockIdx.x] = (float)sqrt(total);
}

}  // namespace brace
