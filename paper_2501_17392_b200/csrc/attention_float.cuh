// Windowed attention in float32 arithmetic, for float32 tensors and for those that the tensor cores' kernels do not take
// (rows that are not aligned, head dimensions above 128 or not a multiple of 8, broadcast tensors).  Formulas and the
// treatment of single rows are in attention_rows.cuh, blocks and pieces as in attention_tiles.cuh.
//
// A CTA has 64 rows (queries, or keys in the pass that makes dk and dv) and walks blocks of columns.  Tiles lie in shared
// memory as float32, rows padded by 4 so that 8 rows' words of 16 bytes lie in different banks; of each product of two
// tiles a thread has 4 rows x 4 columns.  Bound by the multiply-adds and their reads of shared memory: 8192 tokens, 12 heads
// of 64, window 1024, 0.86 ms forward (28 TFLOP/s) and 3.2 ms backward (19).  A row whose result is not finite is computed
// again, key by key, from what it sees.
#pragma once

#include "attention_blocks.cuh"
#include "attention_host.cuh"

namespace brace {

constexpr int kFloatThreads = 256;

template <int D>
struct FloatShape {
  static constexpr int kLd = D + 4;
  static constexpr int kForward = (3 * kFloatRows * kLd + kFloatRows * (kFloatRows + 4)) * 4;
  static constexpr int kBlock = D > 128 ? 32 : 64;       // columns of a block of the backward pass
  static constexpr int kGrad = (2 * kFloatRows * kLd + 2 * kBlock * kLd + 2 * kFloatRows * (kBlock + 4) + 2 * kBlock) * 4;
};

// Rows t .. t + ROWS of one or two heads as float32; 0 from the sequence's end and from the head's dimension on.  A warp reads
// some rows of both before it writes any: the reads are under way together.
template <typename T, int D, int ROWS, bool TWO>
__device__ __forceinline__ void float_tiles(float* to, const HeadRef& x, float* to2, const HeadRef& x2, int b, int h, int t, int n, int dim) {
  constexpr int W = kFloatThreads / 32, P = D / 32, G = D == 256 ? 2 : 4;      // warps; values of a lane and row; rows at a time
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll 1
  for (int r0 = warp; r0 < ROWS; r0 += W * G) {
    float v[TWO ? 2 : 1][G][P];
#pragma unroll
    for (int i = 0; i < G; ++i) {
      const int row = t + r0 + i * W;
#pragma unroll
      for (int k = 0; k < P; ++k) {
        const int d = lane + 32 * k;
        const bool here = row < n && d < dim;
        v[0][i][k] = here ? to_f32(head_row<const T>(x, b, row, h)[d]) : 0.f;
        if (TWO) v[TWO][i][k] = here ? to_f32(head_row<const T>(x2, b, row, h)[d]) : 0.f;
      }
    }
#pragma unroll
    for (int i = 0; i < G; ++i)
#pragma unroll
      for (int k = 0; k < P; ++k) {
        to[(r0 + i * W) * (D + 4) + lane + 32 * k] = v[0][i][k];
        if (TWO) to2[(r0 + i * W) * (D + 4) + lane + 32 * k] = v[TWO][i][k];
      }
  }
}

// acc[i][c] = a[4 ty + i] . b[tx + 16 c]
template <int D, int C>
__device__ __forceinline__ void float_scores(const float* a, const float* b, int dim, float (&acc)[4][C]) {
  const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int c = 0; c < C; ++c) acc[i][c] = 0.f;
#pragma unroll 2
  for (int d = 0; d < dim; d += 4) {
    float4 x[4], y[C];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = *reinterpret_cast<const float4*>(a + (4 * ty + i) * (D + 4) + d);
#pragma unroll
    for (int c = 0; c < C; ++c) y[c] = *reinterpret_cast<const float4*>(b + (tx + 16 * c) * (D + 4) + d);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int c = 0; c < C; ++c)
        acc[i][c] = fmaf(x[i].w, y[c].w, fmaf(x[i].z, y[c].z, fmaf(x[i].y, y[c].y, fmaf(x[i].x, y[c].x, acc[i][c]))));
  }
}

// acc[i][4 c + e] += sum_j p[4 ty + i][j] x[j][64 c + 4 tx + e]
template <int D, int J>
__device__ __forceinline__ void float_sums(const float* p, const float* x, float (&acc)[4][D / 16]) {
  const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
#pragma unroll 2
  for (int j = 0; j < J; j += 4) {
    float w[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) *reinterpret_cast<float4*>(w[i]) = *reinterpret_cast<const float4*>(p + (4 * ty + i) * (J + 4) + j);
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int c = 0; c < D / 64; ++c) {
        const float4 y = *reinterpret_cast<const float4*>(x + (j + k) * (D + 4) + 64 * c + 4 * tx);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          acc[i][4 * c] = fmaf(w[i][k], y.x, acc[i][4 * c]);
          acc[i][4 * c + 1] = fmaf(w[i][k], y.y, acc[i][4 * c + 1]);
          acc[i][4 * c + 2] = fmaf(w[i][k], y.z, acc[i][4 * c + 2]);
          acc[i][4 * c + 3] = fmaf(w[i][k], y.w, acc[i][4 * c + 3]);
        }
      }
  }
}

// A row of results: stores acc * factor, says whether it is finite.
template <typename T, int D>
__device__ __forceinline__ bool float_put(T* row, const float (&acc)[D / 16], float factor, int dim) {
  const int tx = threadIdx.x & 15;
  bool fine = true;
#pragma unroll
  for (int c = 0; c < D / 64; ++c)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int d = 64 * c + 4 * tx + e;
      if (d < dim) {
        const float v = acc[4 * c + e] * factor;
        fine = fine && isfinite(v);
        row[d] = from_f32<T>(v);
      }
    }
  return fine;
}

__device__ __forceinline__ bool attn_sees(const AttnArgs& p, int i, int j) {
  return j <= i && (i - j < p.window || j < p.sinks);
}

// grid: (tiles of queries, heads, sequences)
template <typename T, int D>
__global__ void __launch_bounds__(kFloatThreads, D == 64 ? 3 : 1) attn_forward_float_kernel(const AttnArgs p) {
  constexpr int LD = D + 4, N = kFloatRows;
  extern __shared__ float tiles[];
  __shared__ int again[N];
  float *sq = tiles, *sk = sq + N * LD, *sv = sk + N * LD, *sp = sv + N * LD;
  grid_trigger();
  grid_wait();
  const int b = blockIdx.z, h = blockIdx.y, g = h / p.share, n = attn_length(p, b), q0 = N * (int)(gridDim.x - 1 - blockIdx.x);
  const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
  const float c = fmaxf(fabsf(p.scale) * kLog2e, kTinyScale), sign = p.scale < 0.f ? -1.f : 1.f;
  float acc[4][D / 16] = {}, top[4], total[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    top[i] = -INFINITY;
    total[i] = 0.f;
  }
  if (threadIdx.x < N) again[threadIdx.x] = 0;
  const KeyBlocks keys(p, q0, min(n, q0 + N), N);
  const int count = q0 < n ? keys.count : 0;
  if (count) float_tiles<T, D, N, false>(sq, p.q, nullptr, p.q, b, h, q0, n, p.dim);
  for (int k = 0; k < count; ++k) {
    const int j0 = keys.key(k, N), end = k < keys.nfirst ? keys.first : n;
    __syncthreads();
    float_tiles<T, D, N, true>(sk, p.k, sv, p.v, b, g, j0, n, p.dim);
    __syncthreads();
    float s[4][4];
    float_scores<D, 4>(sq, sk, p.dim, s);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int at = q0 + 4 * ty + i;
      float most = -INFINITY;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int j = j0 + tx + 16 * e;
        s[i][e] = j < end && attn_sees(p, at, j) ? s[i][e] * sign : -INFINITY;
        most = fmaxf(most, s[i][e]);
      }
      for (int o = 8; o; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
      most = fmaxf(most, top[i]);
      const float keep = top[i] == -INFINITY ? 1.f : exp2f((top[i] - most) * c);
      top[i] = most;
      const float shift = most == -INFINITY ? 0.f : -most * c;
      total[i] *= keep;
#pragma unroll
      for (int d = 0; d < D / 16; ++d) acc[i][d] *= keep;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = exp2f(fmaf(s[i][e], c, shift));
        total[i] += x;
        sp[(4 * ty + i) * (N + 4) + tx + 16 * e] = x;
      }
    }
    __syncthreads();
    float_sums<D, N>(sp, sv, acc);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    for (int o = 8; o; o >>= 1) total[i] += __shfl_xor_sync(0xffffffffu, total[i], o);
    const int at = q0 + 4 * ty + i;
    if (at >= p.tokens) continue;
    const bool real = at < n;
    const bool fine = float_put<T, D>(head_row<T>(p.out, b, at, h), acc[i], real ? 1.f / total[i] : 0.f, p.dim);
    if (p.lse && tx == 0) attn_lse(p, b, h, at) = real ? (top[i] * c + log2f(total[i])) * kLn2 : -INFINITY;
    if (real && (!fine || !isfinite(total[i]))) again[4 * ty + i] = 1;
  }
  __syncthreads();
  for (int r = threadIdx.x >> 5; r < N; r += kFloatThreads / 32)
    if (again[r]) forward_row<T>(p, b, h, q0 + r, n);
}

// delta and -log2(e) lse of every query, a warp a row.  grid: (padded / 8, heads, sequences)
template <typename T>
__global__ void __launch_bounds__(256) attn_prepare_float_kernel(const AttnArgs p) {
  grid_trigger();
  grid_wait();
  const int i = blockIdx.x * 8 + (threadIdx.x >> 5), h = blockIdx.y, b = blockIdx.z, n = attn_length(p, b);
  float s = 0.f;
  if (i < n) {
    const T *o = head_row<const T>(p.out, b, i, h), *dout = head_row<const T>(p.dout, b, i, h);
    for (int d = threadIdx.x & 31; d < p.dim; d += 32) s = fmaf(to_f32(o[d]), to_f32(dout[d]), s);
  }
  for (int o2 = 16; o2; o2 >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o2);
  if ((threadIdx.x & 31) == 0) {
    p.delta[attn_delta(p, b, h, i)] = i < n ? s : 0.f;
    p.shift[attn_delta(p, b, h, i)] = i < n ? -kLog2e * attn_lse(p, b, h, i) : 0.f;
  }
}

// grid: that of GradWork
template <typename T, int D, bool DKV>
__global__ void __launch_bounds__(kFloatThreads, 1) attn_grad_float_kernel(const AttnArgs p) {
  constexpr int LD = D + 4, N = kFloatRows, BLOCK = FloatShape<D>::kBlock, C = BLOCK / 16;
  extern __shared__ float tiles[];
  __shared__ int again[N];
  float *a1 = tiles, *a2 = a1 + N * LD, *b1 = a2 + N * LD, *b2 = b1 + BLOCK * LD, *sp = b2 + BLOCK * LD, *sds = sp + N * (BLOCK + 4);
  float* numbers = sds + N * (BLOCK + 4);          // of the block's queries: shifts, deltas
  grid_trigger();
  grid_wait();
  const int b = blockIdx.z, n = attn_length(p, b), ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
  const GradWork w(p, n, DKV, N, BLOCK);
  const float c = p.scale * kLog2e;
  // dv; dk or dq.  A sum over many columns is made of sums over 256: one float32 sum over the queries of 8 heads of 501 tokens
  // left dk and dv off by 1.2e-6, these leave 5e-7 (head dimensions above 128 keep them out of registers: 649 -> 718 us at
  // 1024 tokens, 8 heads of 200 on one).  One CTA an SM: of D = 64, two with 128 registers a thread are faster where there are many
  // (8192 tokens, 12 heads, window 1024: 2760 us for 3160) and slower where there are few (1000 tokens, 8 heads: 459 for 297).
  constexpr int kSome = 256 / BLOCK, K0 = DKV ? D / 16 : 1;
  float r0[4][K0] = {}, r1[4][D / 16] = {}, all0[4][K0] = {}, all1[4][D / 16] = {};
  if (threadIdx.x < N) again[threadIdx.x] = 0;
  float shift[4] = {}, delta[4] = {};
  if (w.count) {
    float_tiles<T, D, N, true>(a1, DKV ? p.k : p.q, a2, DKV ? p.v : p.dout, b, w.head, w.row0, n, p.dim);
    if (!DKV)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int at = w.row0 + 4 * ty + i;
        if (at < n) {
          shift[i] = p.shift[attn_delta(p, b, w.head, at)];
          delta[i] = p.delta[attn_delta(p, b, w.head, at)];
        }
      }
  }
  // the pass that makes dq walks few blocks twice: first for delta, then for ds
  const int first_pass = !DKV && sizeof(T) == 2 && w.count * BLOCK <= kExactKeys ? w.count : 0;
  float sum[4] = {};                                          // of p dp
  for (int step = 0; step < w.count + first_pass; ++step) {
    const int k = step < first_pass ? step : step - first_pass;
    const int t = w.first(k), h = w.head_of(k, p), end = DKV || k >= w.keys.nfirst ? n : w.keys.first;
    if (first_pass && step == first_pass)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        for (int o = 8; o; o >>= 1) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], o);
        delta[i] = sum[i];
        const int at = w.row0 + 4 * ty + i;
        if (tx == 0 && at < n) p.delta[attn_delta(p, b, w.head, at)] = delta[i];
      }
    __syncthreads();
    float_tiles<T, D, BLOCK, true>(b1, DKV ? p.q : p.k, b2, DKV ? p.dout : p.v, b, h, t, n, p.dim);
    if (DKV && threadIdx.x < 2 * BLOCK) {
      const int i = threadIdx.x % BLOCK;
      numbers[threadIdx.x] = t + i < n ? (threadIdx.x < BLOCK ? p.shift : p.delta)[attn_delta(p, b, h, t + i)] : 0.f;
    }
    __syncthreads();
    float s[4][C], y[4][C];
    float_scores<D, C>(a1, b1, p.dim, s);
    float_scores<D, C>(a2, b2, p.dim, y);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int at = w.row0 + 4 * ty + i;
#pragma unroll
      for (int e = 0; e < C; ++e) {
        const int col = tx + 16 * e, j = t + col;
        const bool seen = j < end && (DKV ? attn_sees(p, j, at) : attn_sees(p, at, j));
        const float x = exp2f(fmaf(s[i][e], c, DKV ? numbers[col] : shift[i]));
        const int cell = (4 * ty + i) * (BLOCK + 4) + col;
        if (DKV) sp[cell] = seen ? x : 0.f;
        if (step < first_pass)
          sum[i] += seen ? x * y[i][e] : 0.f;
        else
          sds[cell] = seen ? x * (y[i][e] - (DKV ? numbers[BLOCK + col] : delta[i])) : 0.f;
      }
    }
    if (step < first_pass) continue;
    __syncthreads();
    if constexpr (DKV) float_sums<D, BLOCK>(sp, b2, r0);
    float_sums<D, BLOCK>(sds, b1, r1);
    if ((k + 1) % kSome == 0 || k + 1 == w.count)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int d = 0; d < K0; ++d) {
          all0[i][d] += r0[i][d];
          r0[i][d] = 0.f;
        }
#pragma unroll
        for (int d = 0; d < D / 16; ++d) {
          all1[i][d] += r1[i][d];
          r1[i][d] = 0.f;
        }
      }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = 4 * ty + i, at = w.row0 + row;
    if constexpr (DKV) {
      if (w.piece >= 0) {
        float* part = p.part + w.part_of(p, b, 0, N, D) + (int64_t)row * D;
#pragma unroll
        for (int x = 0; x < D / 64; ++x) {
          *reinterpret_cast<float4*>(part + 64 * x + 4 * tx) = make_float4(all0[i][4 * x], all0[i][4 * x + 1], all0[i][4 * x + 2], all0[i][4 * x + 3]);
          *reinterpret_cast<float4*>(part + N * D + 64 * x + 4 * tx) =
              make_float4(all1[i][4 * x] * p.scale, all1[i][4 * x + 1] * p.scale, all1[i][4 * x + 2] * p.scale, all1[i][4 * x + 3] * p.scale);
        }
        continue;
      }
      if (at >= p.tokens) continue;
      bool fine = float_put<T, D>(head_row<T>(p.dv, b, at, w.head), all0[i], at < n ? 1.f : 0.f, p.dim);
      fine = float_put<T, D>(head_row<T>(p.dk, b, at, w.head), all1[i], at < n ? p.scale : 0.f, p.dim) && fine;
      if (!fine && at < n) again[row] = 1;
    } else {
      if (at >= p.tokens) continue;
      if (!float_put<T, D>(head_row<T>(p.dq, b, at, w.head), all1[i], at < n ? p.scale : 0.f, p.dim) && at < n) again[row] = 1;
    }
  }
  __syncthreads();
  for (int r = threadIdx.x >> 5; r < N; r += kFloatThreads / 32)
    if (again[r]) {
      if (DKV)
        dkv_row<T>(p, b, w.head, w.row0 + r, n);
      else
        dq_row<T>(p, b, w.head, w.row0 + r, n);
    }
}

}  // namespace brace
