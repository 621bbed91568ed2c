// Layer norm of the clients' activations, forward and backward.
//
// Row t of client c: mean = sum x / D, var = sum (x - mean)^2 / D, rstd = 1 / sqrt(var + eps), xh = (x - mean) rstd,
// y = xh w + b.  Backward, g = dy w: dx = rstd (g - sum g / D - xh sum(g xh) / D), dw = sum_t dy xh, db = sum_t dy.
// Every activation is read once and written once.  Bound by memory in float32; in 16 bits by instructions (16 x 8192 x 768 forward
// from float32 to bfloat16 108 us, 0.85 of the copy rate; 8 x 8192 x 768 from bfloat16 to bfloat16 52 us for 31).  G threads hold a row in registers (so that the
// variance is summed from differences, in a second pass that reads nothing), a thread always has the same columns, keeps
// their weights in registers for all of its rows and, backward, the sums of their gradients; the CTAs' sums are joined by
// a second launch, in one order.  Sums are float32.
// Rows of 256 columns or more that start on 16-byte boundaries come through shared memory: each group has a ring of rows
// that bulk copies fill ahead, so that what is under way does not depend on the registers.  Others are loaded by the threads.
#pragma once

#include "elements.cuh"
#include "sm100.cuh"

namespace brace {

constexpr int kNormThreads = 256;
// CTAs of an SM whose threads have so many columns of rows that come through rings; bytes of such a CTA's rings
__host__ __device__ constexpr int ring_resident(int columns) { return columns <= 16 ? 3 : 2; }
__host__ __device__ constexpr int ring_bytes(int columns) { return columns <= 16 ? 62 * 1024 : 96 * 1024; }
constexpr int kRingMost = 8;            // rows of a ring
constexpr int kNormShort = 8192;     // longest row that a CTA's registers hold, its weights and its gradients' sums beside it

// CTAs of an SM that hold so many columns a thread in their registers.
__host__ __device__ constexpr int norm_resident(int columns) { return columns > 12 ? 1 : columns > 8 ? 2 : 4; }

struct NormArgs {
  const void *x, *weight, *bias;
  void* y;                           // forward: written; backward: the gradient of y, read
  float *mean, *rstd;
  void *dx, *dweight, *dbias;
  float* part;                       // [client][part][2][dim]
  int64_t ld_x, stride_x, stride_weight, stride_bias, ld_y, stride_y, stride_stats, ld_dx, stride_dx, stride_dweight, stride_dbias;
  int64_t rows;
  int dim, weight_type, grad_type, group, parts, accumulate;
  int stages, row_bytes;             // of a ring
  float eps;
};

// Element i of an array of any element type.
__device__ __forceinline__ float load_any(const void* p, int type, int64_t i) {
  if (type == kTypeF32) return static_cast<const float*>(p)[i];
  if (type == kTypeBF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
  return __half2float(static_cast<const __half*>(p)[i]);
}
__device__ __forceinline__ void store_any(void* p, int type, int64_t i, float v) {
  if (type == kTypeF32)
    static_cast<float*>(p)[i] = v;
  else if (type == kTypeBF16)
    static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v);
  else
    static_cast<__half*>(p)[i] = __float2half_rn(v);
}

// Sums over the `group` threads of a row.  Groups of more than a warp are the whole CTA; `cell` is then used by turns.
template <int N>
__device__ __forceinline__ void group_sum(float (&v)[N], int group, float (*cell)[kNormThreads / 32][2], int& turn) {
  const int first = group < 32 ? group : 32;
  for (int o = first >> 1; o; o >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
  if (group <= 32) return;
  turn ^= 1;
  if ((threadIdx.x & 31) == 0)
#pragma unroll
    for (int i = 0; i < N; ++i) cell[turn][threadIdx.x >> 5][i] = v[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = 0.f;
  for (int w = 0; w < (group >> 5); ++w)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += cell[turn][w][i];
}

// Forward.  Thread g of a row's G has the NV groups of V columns (i G + g) V .. + V.
template <typename TX, typename TY, int V, int NV>
__global__ void __launch_bounds__(kNormThreads, norm_resident(NV * V)) norm_forward_kernel(const NormArgs p) {
  __shared__ float cell[2][kNormThreads / 32][2];
  grid_trigger();
  grid_wait();
  const int G = p.group, slot = threadIdx.x / G, g = threadIdx.x % G, slots = blockDim.x / G;
  const int64_t c = blockIdx.y;
  const float inv = 1.f / (float)p.dim;
  float w[NV * V], b[NV * V];
#pragma unroll
  for (int i = 0; i < NV * V; ++i) {
    const int col = (i / V * G + g) * V + i % V;
    w[i] = p.weight && col < p.dim ? load_any(p.weight, p.weight_type, c * p.stride_weight + col) : 1.f;
    b[i] = p.bias && col < p.dim ? load_any(p.bias, p.weight_type, c * p.stride_bias + col) : 0.f;
  }
  const TX* x = static_cast<const TX*>(p.x) + c * p.stride_x;
  TY* y = static_cast<TY*>(p.y) + c * p.stride_y;
  int turn = 0;
  for (int64_t r0 = (int64_t)blockIdx.x * slots; r0 < p.rows; r0 += (int64_t)gridDim.x * slots) {
    const int64_t row = r0 + slot;
    const bool live = row < p.rows;
    Pack<TX, V> raw[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int col = (i * G + g) * V;
      if (live && col < p.dim) raw[i].load(x + row * p.ld_x + col);
    }
    float v[NV * V], s[1] = {0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const bool here = live && (i * G + g) * V < p.dim;
#pragma unroll
      for (int k = 0; k < V; ++k) {
        v[i * V + k] = here ? to_f32(raw[i].t[k]) : 0.f;
        s[0] += v[i * V + k];
      }
    }
    group_sum(s, G, cell, turn);
    const float mean = s[0] * inv;
    s[0] = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const bool here = live && (i * G + g) * V < p.dim;
#pragma unroll
      for (int k = 0; k < V; ++k) {
        v[i * V + k] -= mean;
        if (here) s[0] = fmaf(v[i * V + k], v[i * V + k], s[0]);
      }
    }
    group_sum(s, G, cell, turn);
    const float rstd = 1.f / sqrtf(fmaf(s[0], inv, p.eps));
    if (!live) continue;
    if (g == 0) {
      if (p.mean) p.mean[c * p.stride_stats + row] = mean;
      if (p.rstd) p.rstd[c * p.stride_stats + row] = rstd;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int col = (i * G + g) * V;
      Pack<TY, V> o;
#pragma unroll
      for (int k = 0; k < V; ++k) o.t[k] = from_f32<TY>(fmaf(v[i * V + k] * rstd, w[i * V + k], b[i * V + k]));
      if (col < p.dim) o.store_plain(y + row * p.ld_y + col);
    }
  }
}

// This CTA's sums of dweight and dbias: to its part, or to the gradients where it is a client's only CTA.
template <int V, int NV>
__device__ __forceinline__ void norm_put_sums(const NormArgs& p, float (&dw)[NV * V], float (&db)[NV * V], float (*sums)[1024]) {
  const int G = p.group, g = threadIdx.x % G;
  const int64_t c = blockIdx.y;
  // rows of one warp first, then the warps one after the other
  for (int o = G; o < 32; o <<= 1)
#pragma unroll
    for (int i = 0; i < NV * V; ++i) {
      dw[i] += __shfl_xor_sync(0xffffffffu, dw[i], o);
      db[i] += __shfl_xor_sync(0xffffffffu, db[i], o);
    }
  const int warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  if (G <= 32 && warps > 1) {
    for (int t = 0; t < warps; ++t) {
      if (warp == t && (threadIdx.x & 31) < G) {
#pragma unroll
        for (int i = 0; i < NV * V; ++i) {
          const int col = (i / V * G + g) * V + i % V;
          if (col < p.dim) {
            if (t > 0) {
              dw[i] += sums[0][col];
              db[i] += sums[1][col];
            }
            sums[0][col] = dw[i];
            sums[1][col] = db[i];
          }
        }
      }
      __syncthreads();
    }
    if (warp != warps - 1) return;
  }
  if ((threadIdx.x & 31) >= G) return;
#pragma unroll
  for (int i = 0; i < NV * V; ++i) {
    const int col = (i / V * G + g) * V + i % V;
    if (col >= p.dim) continue;
    if (p.parts > 1) {
      float* to = p.part + (c * p.parts + blockIdx.x) * 2 * (int64_t)p.dim + col;
      to[0] = dw[i];
      to[p.dim] = db[i];
    } else {
      const int64_t at_w = c * p.stride_dweight + col, at_b = c * p.stride_dbias + col;
      if (p.dweight) store_any(p.dweight, p.grad_type, at_w, p.accumulate ? load_any(p.dweight, p.grad_type, at_w) + dw[i] : dw[i]);
      if (p.dbias) store_any(p.dbias, p.grad_type, at_b, p.accumulate ? load_any(p.dbias, p.grad_type, at_b) + db[i] : db[i]);
    }
  }
}

// Backward: dx, and this CTA's part of dweight and dbias (the whole of it where there is one CTA for a client).
template <typename TX, typename TY, int V, int NV>
__global__ void __launch_bounds__(kNormThreads, norm_resident(NV * V)) norm_grad_kernel(const NormArgs p) {
  __shared__ float cell[2][kNormThreads / 32][2];
  __shared__ float sums[2][1024];    // rows of a warp or less have at most 1024 columns
  grid_trigger();
  grid_wait();
  const int G = p.group, slot = threadIdx.x / G, g = threadIdx.x % G, slots = blockDim.x / G;
  const int64_t c = blockIdx.y;
  const float inv = 1.f / (float)p.dim;
  const bool params = p.dweight || p.dbias;
  float w[NV * V], dw[NV * V], db[NV * V];
#pragma unroll
  for (int i = 0; i < NV * V; ++i) {
    const int col = (i / V * G + g) * V + i % V;
    w[i] = p.weight && col < p.dim ? load_any(p.weight, p.weight_type, c * p.stride_weight + col) : 1.f;
    dw[i] = db[i] = 0.f;
  }
  const TX* x = static_cast<const TX*>(p.x) + c * p.stride_x;
  const TY* dy = static_cast<const TY*>(p.y) + c * p.stride_y;
  TX* dx = static_cast<TX*>(p.dx) + c * p.stride_dx;
  int turn = 0;
  for (int64_t r0 = (int64_t)blockIdx.x * slots; r0 < p.rows; r0 += (int64_t)gridDim.x * slots) {
    const int64_t row = r0 + slot;
    const bool live = row < p.rows;
    Pack<TX, V> xr[NV];
    Pack<TY, V> yr[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int col = (i * G + g) * V;
      if (live && col < p.dim) {
        xr[i].load(x + row * p.ld_x + col);
        yr[i].load(dy + row * p.ld_y + col);
      }
    }
    const float mean = live ? p.mean[c * p.stride_stats + row] : 0.f, rstd = live ? p.rstd[c * p.stride_stats + row] : 0.f;
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (live && (i * G + g) * V < p.dim) {
#pragma unroll
        for (int k = 0; k < V; ++k) {
          const int e = i * V + k;
          const float xh = (to_f32(xr[i].t[k]) - mean) * rstd, d = to_f32(yr[i].t[k]), gr = d * w[e];
          s[0] += gr;
          s[1] = fmaf(gr, xh, s[1]);
          dw[e] = fmaf(d, xh, dw[e]);
          db[e] += d;
        }
      }
    }
    group_sum(s, G, cell, turn);
    const float m1 = s[0] * inv, m2 = s[1] * inv;
    if (!live) continue;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int col = (i * G + g) * V;
      Pack<TX, V> o;
      if (col >= p.dim) continue;
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const float xh = (to_f32(xr[i].t[k]) - mean) * rstd;
        o.t[k] = from_f32<TX>(rstd * (fmaf(-xh, m2, to_f32(yr[i].t[k]) * w[i * V + k]) - m1));
      }
      o.store_plain(dx + row * p.ld_dx + col);
    }
  }
  if (params) norm_put_sums<V, NV>(p, dw, db, sums);
}

// ---- rows through shared memory.  A group is a warp, or the whole CTA.

struct Ring {
  uint32_t rows, bars;      // addresses in shared memory
  int stages, bytes;        // of the ring, of a row (of both tensors, backward)
  volatile int* dead;
};

// The CTA's shared memory: the groups' barriers, then their rings.
__device__ __forceinline__ Ring ring_of_group(const NormArgs& p, uint8_t* smem, int* dead) {
  const int G = p.group, slot = threadIdx.x / G;
  Ring r;
  r.stages = p.stages;
  r.bytes = p.row_bytes;
  r.bars = smem_addr(smem) + slot * kRingMost * 8;
  r.rows = smem_addr(smem) + 1024 + slot * p.stages * p.row_bytes;
  r.dead = dead;
  if (threadIdx.x == 0) *dead = 0;
  if (threadIdx.x % G == 0)
    for (int s = 0; s < p.stages; ++s) mbar_init(r.bars + 8 * s, 1);
  if (threadIdx.x % G == 0) mbar_init_visible();
  __syncthreads();
  return r;
}
constexpr uint32_t kGaveUp = 2;      // beside the parity of a thread's phase: a wait ran out, and it waits no more
// A wait ran out at stage `s`: lets the rows that are under way land (or the limit run out again) before the CTA's memory goes.
// For the thread that fetches, which then fetches no more; stages that nothing is on its way to end at the limit.
__device__ __forceinline__ void ring_give_up(const Ring& ring, int s, uint32_t phase) {
#pragma unroll 1
  for (int i = 0; i < ring.stages; ++i) {
    mbar_wait(ring.bars + 8 * s, phase, ring.dead);
    if (++s == ring.stages) {
      s = 0;
      phase ^= 1u;
    }
  }
}
__device__ __forceinline__ void group_barrier(int G) {
  if (G > 32)
    __syncthreads();
  else
    __syncwarp();
}

// V columns of a row in shared memory.
template <typename T, int V>
__device__ __forceinline__ void ring_piece(Pack<T, V>& x, uint32_t addr) {
  using W = typename Pack<T, V>::W;
#pragma unroll
  for (int i = 0; i < Pack<T, V>::kWords; ++i) {
    if constexpr (sizeof(W) == 16)
      asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                   : "=r"(reinterpret_cast<uint4*>(x.t)[i].x), "=r"(reinterpret_cast<uint4*>(x.t)[i].y),
                     "=r"(reinterpret_cast<uint4*>(x.t)[i].z), "=r"(reinterpret_cast<uint4*>(x.t)[i].w)
                   : "r"(addr + 16 * i));
    else
      asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];"
                   : "=r"(reinterpret_cast<uint2*>(x.t)[i].x), "=r"(reinterpret_cast<uint2*>(x.t)[i].y)
                   : "r"(addr + 8 * i));
  }
}

template <typename TX, typename TY, int V, int NV>
__global__ void __launch_bounds__(kNormThreads, ring_resident(NV * V)) norm_forward_ring_kernel(const NormArgs p) {
  extern __shared__ __align__(1024) uint8_t smem[];
  __shared__ float cell[2][kNormThreads / 32][2];
  __shared__ int dead;
  const Ring ring = ring_of_group(p, smem, &dead);
  grid_trigger();
  grid_wait();
  const int G = p.group, slot = threadIdx.x / G, g = threadIdx.x % G, slots = blockDim.x / G;
  const int64_t c = blockIdx.y, step = (int64_t)gridDim.x * slots, first = (int64_t)blockIdx.x * slots + slot;
  const float inv = 1.f / (float)p.dim;
  const TX* x = static_cast<const TX*>(p.x) + c * p.stride_x;
  TY* y = static_cast<TY*>(p.y) + c * p.stride_y;
  auto fetch = [&](int64_t row, int s) {
    mbar_expect_tx(ring.bars + 8 * s, ring.bytes);
    bulk_load(ring.rows + s * ring.bytes, x + row * p.ld_x, ring.bytes, ring.bars + 8 * s);
  };
  if (g == 0) {
    fence_async_global();
    for (int s = 0; s < ring.stages; ++s)
      if (first + s * step < p.rows) fetch(first + s * step, s);
  }
  float w[NV * V], b[NV * V];
#pragma unroll
  for (int i = 0; i < NV * V; ++i) {
    const int col = (i / V * G + g) * V + i % V;
    w[i] = p.weight && col < p.dim ? load_any(p.weight, p.weight_type, c * p.stride_weight + col) : 1.f;
    b[i] = p.bias && col < p.dim ? load_any(p.bias, p.weight_type, c * p.stride_bias + col) : 0.f;
  }
  int turn = 0, s = 0;
  uint32_t phase = 0;
  int64_t limit = p.rows;      // of rows that are fetched: 0 once a wait ran out
  for (int64_t row = first; row < p.rows; row += step) {
    if (!mbar_wait(ring.bars + 8 * s, phase, ring.dead)) {
      if (g == 0 && limit) ring_give_up(ring, s, phase);
      limit = 0;
    }
    float v[NV * V], sum[1] = {0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int col = (i * G + g) * V;
      Pack<TX, V> raw;
      if (col < p.dim) ring_piece(raw, ring.rows + s * ring.bytes + col * (int)sizeof(TX));
#pragma unroll
      for (int k = 0; k < V; ++k) {
        v[i * V + k] = col < p.dim ? to_f32(raw.t[k]) : 0.f;
        sum[0] += v[i * V + k];
      }
    }
    group_barrier(G);      // all have read the row
    if (g == 0 && row + ring.stages * step < limit) fetch(row + ring.stages * step, s);
    if (++s == ring.stages) {
      s = 0;
      phase ^= 1u;
    }
    group_sum(sum, G, cell, turn);
    const float mean = limit ? sum[0] * inv : NAN;      // a wait that ran out shows in the result
    sum[0] = 0.f;
#pragma unroll
    for (int i = 0; i < NV * V; ++i) {
      v[i] -= mean;
      if ((i / V * G + g) * V < p.dim) sum[0] = fmaf(v[i], v[i], sum[0]);
    }
    group_sum(sum, G, cell, turn);
    const float rstd = 1.f / sqrtf(fmaf(sum[0], inv, p.eps));
    if (g == 0) {
      if (p.mean) p.mean[c * p.stride_stats + row] = mean;
      if (p.rstd) p.rstd[c * p.stride_stats + row] = rstd;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int col = (i * G + g) * V;
      Pack<TY, V> o;
#pragma unroll
      for (int k = 0; k < V; ++k) o.t[k] = from_f32<TY>(fmaf(v[i * V + k] * rstd, w[i * V + k], b[i * V + k]));
      if (col < p.dim) o.store_plain(y + row * p.ld_y + col);
    }
  }
}

template <typename TX, typename TY, int V, int NV>
__global__ void __launch_bounds__(kNormThreads, ring_resident(NV * V)) norm_grad_ring_kernel(const NormArgs p) {
  extern __shared__ __align__(1024) uint8_t smem[];
  __shared__ float cell[2][kNormThreads / 32][2];
  __shared__ float sums[2][1024];
  __shared__ int dead;
  const Ring ring = ring_of_group(p, smem, &dead);
  grid_trigger();
  grid_wait();
  const int G = p.group, slot = threadIdx.x / G, g = threadIdx.x % G, slots = blockDim.x / G;
  const int64_t c = blockIdx.y, step = (int64_t)gridDim.x * slots, first = (int64_t)blockIdx.x * slots + slot;
  const float inv = 1.f / (float)p.dim;
  const TX* x = static_cast<const TX*>(p.x) + c * p.stride_x;
  const TY* dy = static_cast<const TY*>(p.y) + c * p.stride_y;
  TX* dx = static_cast<TX*>(p.dx) + c * p.stride_dx;
  const int x_bytes = p.dim * (int)sizeof(TX);
  auto fetch = [&](int64_t row, int s) {
    mbar_expect_tx(ring.bars + 8 * s, ring.bytes);
    bulk_load(ring.rows + s * ring.bytes, x + row * p.ld_x, x_bytes, ring.bars + 8 * s);
    bulk_load(ring.rows + s * ring.bytes + x_bytes, dy + row * p.ld_y, ring.bytes - x_bytes, ring.bars + 8 * s);
  };
  if (g == 0) {
    fence_async_global();
    for (int s = 0; s < ring.stages; ++s)
      if (first + s * step < p.rows) fetch(first + s * step, s);
  }
  float w[NV * V], dw[NV * V], db[NV * V];
#pragma unroll
  for (int i = 0; i < NV * V; ++i) {
    const int col = (i / V * G + g) * V + i % V;
    w[i] = p.weight && col < p.dim ? load_any(p.weight, p.weight_type, c * p.stride_weight + col) : 1.f;
    dw[i] = db[i] = 0.f;
  }
  int turn = 0, s = 0;
  uint32_t phase = 0;      // and kGaveUp
  for (int64_t row = first; row < p.rows; row += step) {
    const float mean = p.mean[c * p.stride_stats + row], rstd = p.rstd[c * p.stride_stats + row];
    if (phase < kGaveUp && !mbar_wait(ring.bars + 8 * s, phase, ring.dead)) phase |= kGaveUp;
    const uint32_t at = ring.rows + s * ring.bytes;
    float t[2] = {phase < kGaveUp ? 0.f : NAN, 0.f};      // a wait that ran out shows in the results
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int col = (i * G + g) * V;
      if (col >= p.dim) continue;
      Pack<TX, V> xr;
      Pack<TY, V> yr;
      ring_piece(xr, at + col * (int)sizeof(TX));
      ring_piece(yr, at + x_bytes + col * (int)sizeof(TY));
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const int e = i * V + k;
        const float xh = (to_f32(xr.t[k]) - mean) * rstd, d = to_f32(yr.t[k]), gr = d * w[e];
        t[0] += gr;
        t[1] = fmaf(gr, xh, t[1]);
        dw[e] = fmaf(d, xh, dw[e]);
        db[e] += d;
      }
    }
    group_sum(t, G, cell, turn);
    const float m1 = t[0] * inv, m2 = t[1] * inv;
#pragma unroll
    for (int i = 0; i < NV; ++i) {      // the row once more: it is still there
      const int col = (i * G + g) * V;
      if (col >= p.dim) continue;
      Pack<TX, V> xr, o;
      Pack<TY, V> yr;
      ring_piece(xr, at + col * (int)sizeof(TX));
      ring_piece(yr, at + x_bytes + col * (int)sizeof(TY));
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const float xh = (to_f32(xr.t[k]) - mean) * rstd;
        o.t[k] = from_f32<TX>(rstd * (fmaf(-xh, m2, to_f32(yr.t[k]) * w[i * V + k]) - m1));
      }
      o.store_plain(dx + row * p.ld_dx + col);
    }
    group_barrier(G);      // all have read the row
    if (g == 0 && phase < kGaveUp && row + ring.stages * step < p.rows) fetch(row + ring.stages * step, s);
    if (phase < kGaveUp && ++s == ring.stages) {
      s = 0;
      phase ^= 1u;
    }
  }
  if (phase >= kGaveUp)
#pragma unroll
    for (int i = 0; i < NV * V; ++i) dw[i] = db[i] = NAN;
  if (phase >= kGaveUp && g == 0) ring_give_up(ring, s, phase & 1u);
  if (p.dweight || p.dbias) norm_put_sums<V, NV>(p, dw, db, sums);
}

// dweight and dbias from the CTAs' parts: 32 columns a CTA, a warp takes every 8th part.
__global__ void __launch_bounds__(256) norm_join_kernel(const NormArgs p) {
  __shared__ float cell[8][32];
  grid_trigger();
  grid_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, at = blockIdx.x * 32 + lane;   // of both vectors
  const int64_t c = blockIdx.y;
  float sum = 0.f;
  if (at < 2 * p.dim) {
    const float* from = p.part + c * p.parts * 2 * (int64_t)p.dim + at;
#pragma unroll 4
    for (int k = warp; k < p.parts; k += 8) sum += from[(int64_t)k * 2 * p.dim];
  }
  cell[warp][lane] = sum;
  __syncthreads();
  if (warp || at >= 2 * p.dim) return;
  for (int k = 1; k < 8; ++k) sum += cell[k][lane];
  void* to = at < p.dim ? p.dweight : p.dbias;
  if (!to) return;
  const int64_t i = at < p.dim ? c * p.stride_dweight + at : c * p.stride_dbias + at - p.dim;
  store_any(to, p.grad_type, i, p.accumulate ? load_any(to, p.grad_type, i) + sum : sum);
}

// ---- rows longer than kNormShort: a CTA walks a row more than once (the later passes find it in L1 or L2), and the
// weights' gradients take a pass of their own.

// V weights from index i, by words of 16 bytes where they lie so.  Read one by one, by lanes that are V columns apart, they
// bound these kernels: 2000 x 16384 in bfloat16 takes 51 us forward and 118 us back with the one, 95 and 160 with the other.
template <int V>
__device__ __forceinline__ bool even_weights(const void* p, int type, int64_t i) {
  return V == 8 && ((reinterpret_cast<uintptr_t>(p) + i * (type == kTypeF32 ? 4 : 2)) & 15) == 0;
}
template <int V>
__device__ __forceinline__ void load_weights(const void* p, int type, int64_t i, bool even, float none, float (&to)[V]) {
  if (!p) {
#pragma unroll
    for (int k = 0; k < V; ++k) to[k] = none;
  } else if (!even) {
#pragma unroll
    for (int k = 0; k < V; ++k) to[k] = load_any(p, type, i + k);
  } else if (type == kTypeF32) {
    Pack<float, V> a;
    a.load(static_cast<const float*>(p) + i);
#pragma unroll
    for (int k = 0; k < V; ++k) to[k] = a.t[k];
  } else if (type == kTypeBF16) {
    Pack<__nv_bfloat16, V> a;
    a.load(static_cast<const __nv_bfloat16*>(p) + i);
#pragma unroll
    for (int k = 0; k < V; ++k) to[k] = to_f32(a.t[k]);
  } else {
    Pack<__half, V> a;
    a.load(static_cast<const __half*>(p) + i);
#pragma unroll
    for (int k = 0; k < V; ++k) to[k] = to_f32(a.t[k]);
  }
}

// f(first column, the V values of x there, those of y) for this thread's pieces of a row.
template <typename TX, typename TY, int V, typename F>
__device__ __forceinline__ void norm_pieces(const TX* x, const TY* y, int dim, F&& f) {
  constexpr int U = V == 1 ? 8 : 2;      // pieces under way
  for (int i0 = threadIdx.x * V; i0 < dim; i0 += kNormThreads * V * U) {
    Pack<TX, V> a[U];
    Pack<TY, V> b[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * kNormThreads * V;
      if (i < dim) {
        a[u].load(x + i);
        if (y) b[u].load(y + i);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i0 + u * kNormThreads * V < dim) f(i0 + u * kNormThreads * V, a[u], b[u]);
  }
}

template <typename TX, typename TY, int V>
__global__ void __launch_bounds__(kNormThreads) norm_forward_long_kernel(const NormArgs p) {
  __shared__ float cell[2][kNormThreads / 32][2];
  grid_trigger();
  grid_wait();
  const int64_t c = blockIdx.y;
  const float inv = 1.f / (float)p.dim;
  const bool even_w = even_weights<V>(p.weight, p.weight_type, c * p.stride_weight);
  const bool even_b = even_weights<V>(p.bias, p.weight_type, c * p.stride_bias);
  int turn = 0;
  for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
    const TX* x = static_cast<const TX*>(p.x) + c * p.stride_x + row * p.ld_x;
    TY* y = static_cast<TY*>(p.y) + c * p.stride_y + row * p.ld_y;
    const TY* none = nullptr;
    float s[1] = {0.f};
    norm_pieces<TX, TY, V>(x, none, p.dim, [&](int, const Pack<TX, V>& a, const Pack<TY, V>&) {
#pragma unroll
      for (int k = 0; k < V; ++k) s[0] += to_f32(a.t[k]);
    });
    group_sum(s, kNormThreads, cell, turn);
    const float mean = s[0] * inv;
    s[0] = 0.f;
    norm_pieces<TX, TY, V>(x, none, p.dim, [&](int, const Pack<TX, V>& a, const Pack<TY, V>&) {
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const float d = to_f32(a.t[k]) - mean;
        s[0] = fmaf(d, d, s[0]);
      }
    });
    group_sum(s, kNormThreads, cell, turn);
    const float rstd = 1.f / sqrtf(fmaf(s[0], inv, p.eps));
    if (threadIdx.x == 0) {
      if (p.mean) p.mean[c * p.stride_stats + row] = mean;
      if (p.rstd) p.rstd[c * p.stride_stats + row] = rstd;
    }
    norm_pieces<TX, TY, V>(x, none, p.dim, [&](int i, const Pack<TX, V>& a, const Pack<TY, V>&) {
      Pack<TY, V> o;
      float w[V], b[V];
      load_weights<V>(p.weight, p.weight_type, c * p.stride_weight + i, even_w, 1.f, w);
      load_weights<V>(p.bias, p.weight_type, c * p.stride_bias + i, even_b, 0.f, b);
#pragma unroll
      for (int k = 0; k < V; ++k) o.t[k] = from_f32<TY>(fmaf((to_f32(a.t[k]) - mean) * rstd, w[k], b[k]));
      o.store_plain(y + i);
    });
  }
}

template <typename TX, typename TY, int V>
__global__ void __launch_bounds__(kNormThreads) norm_grad_long_kernel(const NormArgs p) {
  __shared__ float cell[2][kNormThreads / 32][2];
  grid_trigger();
  grid_wait();
  const int64_t c = blockIdx.y;
  const float inv = 1.f / (float)p.dim;
  const bool even = even_weights<V>(p.weight, p.weight_type, c * p.stride_weight);
  int turn = 0;
  for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
    const TX* x = static_cast<const TX*>(p.x) + c * p.stride_x + row * p.ld_x;
    const TY* dy = static_cast<const TY*>(p.y) + c * p.stride_y + row * p.ld_y;
    TX* dx = static_cast<TX*>(p.dx) + c * p.stride_dx + row * p.ld_dx;
    const float mean = p.mean[c * p.stride_stats + row], rstd = p.rstd[c * p.stride_stats + row];
    float s[2] = {0.f, 0.f};
    norm_pieces<TX, TY, V>(x, dy, p.dim, [&](int i, const Pack<TX, V>& a, const Pack<TY, V>& d) {
      float w[V];
      load_weights<V>(p.weight, p.weight_type, c * p.stride_weight + i, even, 1.f, w);
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const float gr = to_f32(d.t[k]) * w[k];
        s[0] += gr;
        s[1] = fmaf(gr, (to_f32(a.t[k]) - mean) * rstd, s[1]);
      }
    });
    group_sum(s, kNormThreads, cell, turn);
    const float m1 = s[0] * inv, m2 = s[1] * inv;
    norm_pieces<TX, TY, V>(x, dy, p.dim, [&](int i, const Pack<TX, V>& a, const Pack<TY, V>& d) {
      Pack<TX, V> o;
      float w[V];
      load_weights<V>(p.weight, p.weight_type, c * p.stride_weight + i, even, 1.f, w);
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const float xh = (to_f32(a.t[k]) - mean) * rstd;
        o.t[k] = from_f32<TX>(rstd * (fmaf(-xh, m2, to_f32(d.t[k]) * w[k]) - m1));
      }
      o.store_plain(dx + i);
    });
  }
}

// Part blockIdx.y (every parts-th row) of dweight and dbias, V columns a thread.
template <typename TX, typename TY, int V>
__global__ void __launch_bounds__(kNormThreads) norm_columns_kernel(const NormArgs p) {
  grid_trigger();
  grid_wait();
  const int64_t c = blockIdx.z;
  const int col = (blockIdx.x * kNormThreads + threadIdx.x) * V;
  if (col >= p.dim) return;
  const TX* x = static_cast<const TX*>(p.x) + c * p.stride_x + col;
  const TY* dy = static_cast<const TY*>(p.y) + c * p.stride_y + col;
  float dw[V] = {}, db[V] = {};
#pragma unroll 4
  for (int64_t row = blockIdx.y; row < p.rows; row += p.parts) {
    Pack<TX, V> a;
    Pack<TY, V> d;
    a.load(x + row * p.ld_x);
    d.load(dy + row * p.ld_y);
    const float mean = p.mean[c * p.stride_stats + row], rstd = p.rstd[c * p.stride_stats + row];
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const float g = to_f32(d.t[k]);
      dw[k] = fmaf(g, (to_f32(a.t[k]) - mean) * rstd, dw[k]);
      db[k] += g;
    }
  }
  float* to = p.part + (c * p.parts + blockIdx.y) * 2 * (int64_t)p.dim + col;
#pragma unroll
  for (int k = 0; k < V; ++k) {
    to[k] = dw[k];
    to[p.dim + k] = db[k];
  }
}

}  // namespace brace
