// Kernels of the orthogonalised update (Newton-Schulz) and of the momentum step around it (sm_100a).
//
// The iteration.  For a matrix G (rows x cols), X_0 = G / (||G||_F + eps) and
//     S = X X^T  (X^T X when rows > cols: the Gram matrix of the short side, m x m)
//     P = b S + c S^2
//     X <- a X + P X  (a X + X P)
// `steps` times.  All singular vectors stay, every singular value s goes to a s + b s^3 + c s^5, so the values are
// pushed towards 1 and X towards the nearest matrix with orthonormal rows (columns).
//
// Number format.  The operands of all products are float16 times a power of two, with float32 accumulators.  That is
// possible because the iteration's values are bounded (the host checks the coefficients: singular values below 2,
// |b s^2 + c s^4| below 8), so X 2^14, S 2^14 and P 2^13 cannot overflow and entries down to 4e-9 stay normal; it
// keeps 11 bits where bfloat16, at the same rate, keeps 8.  For a 16-bit result one float16 holds an operand.  Where
// float32 accuracy is asked for, an operand is the sum of two float16 planes (hi + lo, 22 bits) and a product is
// hi*hi + hi*lo + lo*hi: three times the matrix instructions.
//
// Symmetry.  S and P are symmetric: only tiles on and below the diagonal are computed, the others are written as
// their mirror images.  That takes a step from 2 m^2 k + 2 m^3 + 2 m^2 k operations to m^2 k + m^3 + 2 m^2 k.
#pragma once

#include "elements.cuh"
#include "sm100.cuh"

namespace brace {

constexpr float kScaleX = 16384.f;                  // stored X = X * 2^14
constexpr float kScaleSInv = 1.f / 16384.f;         // X X^T * 2^28 -> S * 2^14
constexpr float kPolyB = 0.5f;                      // S * 2^14 -> P * 2^13
constexpr float kPolyC = 1.f / 32768.f;             // S S * 2^28 -> P * 2^13
constexpr float kStepAcc = 1.f / 8192.f;            // P X * 2^27 -> X * 2^14

// A matrix of a user's: `type`, rows `ld` elements apart, matrices of a batch `batch` elements apart.
struct MatRef {
  const void* p;
  int64_t ld, batch;
  int type;
  int vec;   // 8 consecutive elements of a row, from a multiple of 8, can be read as whole 16-byte words
  int64_t bit0;
};

// 8 elements of a row from column `col`; `n` of them exist (the others read as 0).
template <typename T>
__device__ __forceinline__ void load8(const T* p, int vec, int n, float (&v)[8]) {
  if (vec && n == 8) {
    alignas(16) T t[8];
#pragma unroll
    for (int i = 0; i < (int)(8 * sizeof(T) / 16); ++i)
      reinterpret_cast<uint4*>(t)[i] = reinterpret_cast<const uint4*>(p)[i];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = to_f32(t[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? to_f32(p[i]) : 0.f;
  }
}
template <typename T>
__device__ __forceinline__ void store8(T* p, int vec, int n, const float (&v)[8]) {
  if (vec && n == 8) {
    alignas(16) T t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = from_f32<T>(v[i]);
#pragma unroll
    for (int i = 0; i < (int)(8 * sizeof(T) / 16); ++i) reinterpret_cast<uint4*>(p)[i] = reinterpret_cast<uint4*>(t)[i];
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = from_f32<T>(v[i]);
  }
}
// +1 / -1 from packed bits, least significant first (the rows that an aggregation round leaves).
__device__ __forceinline__ void load_bits8(const uint32_t* words, int64_t k, int n, float (&v)[8]) {
  const int64_t w = k >> 5;
  const int sh = (int)(k & 31);
  uint32_t x = __ldg(words + w) >> sh;
  if (sh + n > 32) x |= __ldg(words + w + 1) << (32 - sh);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = i < n ? ((x >> i) & 1u ? 1.f : -1.f) : 0.f;
}

struct PrepArgs {
  MatRef g;             // the new update (or the matrix to orthogonalise)
  const float* m_in;    // momentum, or null
  float* m_out;
  int64_t ld_m_in, batch_m_in, ld_m_out, batch_m_out;
  int vec_m_in, vec_m_out;
  float beta;
  int nesterov;
  int rows, cols;
  int units_row;        // ceil(cols / 8)
  int norm_blocks;      // partial sums per matrix
  double* partial;      // [batch][norm_blocks]
  float eps;
  __half* x;            // X_0: [batch][planes][rows][ld_x]
  int64_t ld_x;
  int planes;
  int* status;
};

template <int TYPE>
__device__ __forceinline__ void load_g(const PrepArgs& p, int64_t b, int row, int col, int n, float (&g)[8]) {
  if (TYPE == kTypeBits) {
    load_bits8((const uint32_t*)p.g.p, p.g.bit0 + b * p.g.batch + (int64_t)row * p.g.ld + col, n, g);
  } else {
    using T = typename Elem<TYPE>::T;
    load8((const T*)p.g.p + b * p.g.batch + (int64_t)row * p.g.ld + col, p.g.vec, n, g);
  }
}

__device__ __forceinline__ double block_sum(double v, double* scratch) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
  __syncthreads();
  double t = 0;
  for (int w = 0; w < (int)(blockDim.x >> 5); ++w) t += scratch[w];
  return t;
}

// Pass 1: the momentum (if any) and the partial sums of squares of the matrix that is orthogonalised.  Bytes: the
// update once, the momentum once in and once out.  The squares are summed in float64, so that no finite float32
// update overflows and the order of a sum does not matter for the result's bits in practice; each block's sum has a
// place of its own, so the result is the same every time.
template <int TYPE>
__global__ void __launch_bounds__(256) ortho_norm_kernel(const PrepArgs p) {
  __shared__ double scratch[8];
  grid_wait();
  grid_trigger();
  const int64_t b = blockIdx.y;
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *p.status = 0;
  const uint32_t units = (uint32_t)p.rows * (uint32_t)p.units_row;
  double sum = 0;
  for (uint32_t u = blockIdx.x * 256u + threadIdx.x; u < units; u += gridDim.x * 256u) {
    const int row = (int)(u / (uint32_t)p.units_row), col = (int)(u % (uint32_t)p.units_row) * 8;
    const int n = min(8, p.cols - col);
    float g[8];
    load_g<TYPE>(p, b, row, col, n, g);
    if (p.m_in) {
      float m[8];
      load8(p.m_in + b * p.batch_m_in + (int64_t)row * p.ld_m_in + col, p.vec_m_in, n, m);
#pragma unroll
      for (int i = 0; i < 8; ++i) m[i] = fmaf(p.beta, m[i], g[i]);
      store8(p.m_out + b * p.batch_m_out + (int64_t)row * p.ld_m_out + col, p.vec_m_out, n, m);
#pragma unroll
      for (int i = 0; i < 8; ++i) g[i] = p.nesterov ? fmaf(p.beta, m[i], g[i]) : m[i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) sum = fma((double)g[i], (double)g[i], sum);
  }
  const double t = block_sum(sum, scratch);
  if (threadIdx.x == 0) p.partial[b * p.norm_blocks + blockIdx.x] = t;
}

__device__ __forceinline__ void split_store8(__half* hi, int64_t plane, int planes, const float (&v)[8]) {
  alignas(16) __half h[8], l[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    h[i] = __float2half_rn(v[i]);
    l[i] = __float2half_rn(v[i] - __half2float(h[i]));
  }
  *reinterpret_cast<uint4*>(hi) = *reinterpret_cast<uint4*>(h);
  if (planes == 2) *reinterpret_cast<uint4*>(hi + plane) = *reinterpret_cast<uint4*>(l);
}

// Pass 2: X_0, scaled and rounded to one or two float16 planes.
template <int TYPE>
__global__ void __launch_bounds__(256) ortho_scale_kernel(const PrepArgs p) {
  __shared__ double scratch[8];
  grid_wait();
  grid_trigger();
  const int64_t b = blockIdx.y;
  double part = 0;
  for (int i = threadIdx.x; i < p.norm_blocks; i += 256) part += p.partial[b * p.norm_blocks + i];
  const double norm = sqrt(block_sum(part, scratch));
  const float inv = (float)((double)kScaleX / (norm + (double)p.eps));
  const int64_t plane = (int64_t)p.rows * p.ld_x;
  const uint32_t units_x = (uint32_t)(p.ld_x >> 3);   // rows of X are padded: the pad is written as zeros
  const uint32_t units = (uint32_t)p.rows * units_x;
  for (uint32_t u = blockIdx.x * 256u + threadIdx.x; u < units; u += gridDim.x * 256u) {
    const int row = (int)(u / units_x), col = (int)(u % units_x) * 8;
    const int n = max(0, min(8, p.cols - col));
    float g[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) g[i] = 0.f;
    if (n > 0) {
      if (!p.m_in || p.nesterov) load_g<TYPE>(p, b, row, col, n, g);
      if (p.m_in) {
        float m[8];
        load8((const float*)p.m_out + b * p.batch_m_out + (int64_t)row * p.ld_m_out + col, p.vec_m_out, n, m);
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] = p.nesterov ? fmaf(p.beta, m[i], g[i]) : m[i];
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) g[i] *= inv;
    split_store8(p.x + b * p.planes * plane + (int64_t)row * p.ld_x + col, plane, p.planes, g);
  }
  fence_async_global();
}

// ---------------------------------------------------------------------------------------------------------------
// The products.
// ---------------------------------------------------------------------------------------------------------------

enum { kModeGram = 0, kModePoly = 1, kModeStep = 2, kModeLast = 3 };

struct GemmArgs {
  int M, N, K;                  // result M x N, contraction K
  int tiles_n, tiles;           // tile columns, tiles per matrix
  int total;                    // tiles of all matrices
  float alpha;                  // times the source (S or X)
  float beta;                   // times the product
  const __half* src;            // [batch][planes][M][ld_src]
  int64_t ld_src;
  __half* dst;                  // [batch][planes][M][ld_dst]
  int64_t ld_dst;
  // kModeLast: the result O, or the weights W_out = keep * W_in - rate * O for `replicas` copies
  void* out;
  const void* w_in;
  int64_t ld_out, batch_out, rep_out, ld_in, batch_in, rep_in;
  int out_type, vec_out, vec_in, replicas;
  float keep, rate;
  int* status;
};

constexpr int kTileK = 64;                       // contraction per stage: one 128-byte swizzle row
constexpr int kOperandBytes = 128 * kTileK * 2;  // an operand of a stage in one CTA: 128 rows (or columns)

template <int CG, int NP>
struct GemmShape {
  static constexpr int kTile = 128 * CG;                     // square tiles
  static constexpr int kStageBytes = 2 * NP * kOperandBytes;
  static constexpr int kStages = NP == 1 ? 6 : 3;            // 192 KB either way
  static constexpr int kThreads = CG == 1 ? 256 : 384;       // warps 0-3: loads, MMAs, tensor memory, -; then epilogue
  static constexpr int kTmemCols = 2 * kTile;                // two accumulators: one is filled while one is read
  static constexpr int kSmem = kStages * kStageBytes + 1024 + 256;
};

// Column blocks of the lower triangle in rows: t -> (row, col), col <= row.
__device__ __forceinline__ void triangle(int t, int& row, int& col) {
  row = (int)((sqrtf(8.f * (float)t + 1.f) - 1.f) * 0.5f);
  while ((row + 1) * (row + 2) / 2 <= t) ++row;
  while (row * (row + 1) / 2 > t) --row;
  col = t - row * (row + 1) / 2;
}

template <typename T>
__device__ __forceinline__ void last_chunk(const GemmArgs& p, int64_t b, int row, int col, int n, const float (&o)[32]) {
  for (int r = 0; r < p.replicas; ++r) {
    T* out = (T*)p.out + b * p.batch_out + r * p.rep_out + (int64_t)row * p.ld_out + col;
    const T* in = p.w_in ? (const T*)p.w_in + b * p.batch_in + r * p.rep_in + (int64_t)row * p.ld_in + col : nullptr;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int nq = min(8, n - 8 * q);
      if (nq <= 0) break;
      float v[8];
      if (in) {
        // a plain load: in and out may be the same buffer
        if (p.vec_in && nq == 8) {
          alignas(16) T t[8];
#pragma unroll
          for (int i = 0; i < (int)(8 * sizeof(T) / 16); ++i)
            reinterpret_cast<uint4*>(t)[i] = *(reinterpret_cast<const uint4*>(in + 8 * q) + i);
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] = to_f32(t[i]);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] = i < nq ? to_f32(in[8 * q + i]) : 0.f;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = p.keep * v[i] - p.rate * o[8 * q + i];
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = o[8 * q + i];
      }
      store8(out + 8 * q, p.vec_out, nq, v);
    }
  }
}

// One product of the iteration over tiles of 128 x 128 (CG = 1) or, by a pair of CTAs, 256 x 256 (CG = 2); NP planes
// per operand; A_MN / B_MN: the operand lies with the contraction along its rows (the other axis contiguous).
// Warp 0 loads, warp 1 issues the matrix instructions, warp 2 owns the tensor memory, warps 4.. read the
// accumulators and write the results; persistent over tiles, so that the epilogue of a tile runs under the products
// of the next.
template <int CG, int NP, bool A_MN, bool B_MN, int MODE>
__global__ void __launch_bounds__(GemmShape<CG, NP>::kThreads, 1)
    ortho_gemm_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                      const GemmArgs p) {
  using Shape = GemmShape<CG, NP>;
  constexpr int T = Shape::kTile, STAGES = Shape::kStages;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_addr(smem_raw) + 1023u) & ~1023u;
  const uint32_t bars = base + STAGES * Shape::kStageBytes;
  const uint32_t full = bars, empty = bars + 8 * STAGES, tm_full = empty + 8 * STAGES, tm_empty = tm_full + 16;
  volatile int* dead = (volatile int*)(smem_raw + (tm_empty + 16 - smem_addr(smem_raw)));
  uint32_t* tmem_slot = (uint32_t*)(smem_raw + (tm_empty + 24 - smem_addr(smem_raw)));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = CG == 1 ? 0u : cluster_rank();
  constexpr int kEpiWarps = Shape::kThreads / 32 - 4;

  if (threadIdx.x == 0) {
    *dead = 0;
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(full + 8 * s, 1);
      mbar_init(empty + 8 * s, 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(tm_full + 8 * i, 1);
      mbar_init(tm_empty + 8 * i, CG * kEpiWarps);
    }
    mbar_init_visible();
    tma_prefetch(&map_a);
    tma_prefetch(&map_b);
  }
  if (warp == 2) tmem_alloc<CG>(smem_addr(tmem_slot), Shape::kTmemCols);
  tc_fence_before();
  __syncthreads();
  if (CG == 2) cluster_sync();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  grid_trigger();   // the next kernel of the chain may set itself up; it reads nothing before this one is complete
  grid_wait();
  fence_async_global();

  const int cluster = blockIdx.x / CG, clusters = gridDim.x / CG;
  const int kblocks = (p.K + kTileK - 1) / kTileK;
  auto place = [&](int tile, int& b, int& ti, int& tj) {
    b = tile / p.tiles;
    const int t = tile - b * p.tiles;
    if (MODE == kModeGram || MODE == kModePoly) {
      triangle(t, ti, tj);
    } else {
      ti = t / p.tiles_n;
      tj = t - ti * p.tiles_n;
    }
  };

  if (warp == 0) {
    if (lane == 0) {
      const uint32_t full0 = CG == 1 ? full : map_to_rank(full, 0);
      int s = 0;
      uint32_t ph = 0, issued = 0;
      bool ok = true;
      for (int tile = cluster; ok && tile < p.total; tile += clusters) {
        int b, ti, tj;
        place(tile, b, ti, tj);
        const int ra = ti * T + (int)rank * 128, rb = tj * T + (int)rank * 128;
        for (int kb = 0; kb < kblocks; ++kb) {
          if (!mbar_wait(empty + 8 * s, ph ^ 1u, dead)) {
            ok = false;
            break;
          }
          if (rank == 0) mbar_expect_tx(full + 8 * s, CG * Shape::kStageBytes);
          const uint32_t st = base + s * Shape::kStageBytes;
#pragma unroll
          for (int pl = 0; pl < NP; ++pl) {
            const int z = b * NP + pl;
#pragma unroll
            for (int h = 0; h < 2; ++h) {   // boxes of 64 x 64: two make an operand, whichever way it lies
              const uint32_t da = st + pl * kOperandBytes + h * (kOperandBytes / 2), db = da + NP * kOperandBytes;
              if (A_MN)
                tma_load<CG>(da, &map_a, ra + 64 * h, kb * kTileK, z, full0 + 8 * s);
              else
                tma_load<CG>(da, &map_a, kb * kTileK, ra + 64 * h, z, full0 + 8 * s);
              if (B_MN)
                tma_load<CG>(db, &map_b, rb + 64 * h, kb * kTileK, z, full0 + 8 * s);
              else
                tma_load<CG>(db, &map_b, kb * kTileK, rb + 64 * h, z, full0 + 8 * s);
            }
          }
          ++issued;
          if (++s == STAGES) {
            s = 0;
            ph ^= 1u;
          }
        }
      }
      if (!ok && rank == 0) {   // gave up: let the copies in flight land before the memory goes
        for (uint32_t i = issued > (uint32_t)STAGES ? issued - STAGES : 0; i < issued; ++i)
          mbar_wait(full + 8 * (i % STAGES), (i / STAGES) & 1u, dead);
      }
    }
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {
      constexpr uint32_t idesc = f16_idesc(128 * CG, 128 * CG, A_MN, B_MN);
      // per 16 of the contraction: 32 bytes along a swizzled row, or 16 rows of 128 bytes
      constexpr uint64_t step_a = (A_MN ? 2048 : 32) >> 4, step_b = (B_MN ? 2048 : 32) >> 4;
      int s = 0, buf = 0;
      uint32_t ph = 0, tph = 0;
      bool ok = true;
      for (int tile = cluster; ok && tile < p.total; tile += clusters) {
        if (!mbar_wait(tm_empty + 8 * buf, tph ^ 1u, dead)) break;
        tc_fence_after();
        const uint32_t d = tmem + buf * T;
        for (int kb = 0; kb < kblocks; ++kb) {
          if (!mbar_wait(full + 8 * s, ph, dead)) {
            ok = false;
            break;
          }
          tc_fence_after();
          const uint32_t st = base + s * Shape::kStageBytes;
          uint64_t da[NP], db[NP];
#pragma unroll
          for (int pl = 0; pl < NP; ++pl) {
            da[pl] = operand_desc(st + pl * kOperandBytes, kOperandBytes / 2);
            db[pl] = operand_desc(st + (NP + pl) * kOperandBytes, kOperandBytes / 2);
          }
#pragma unroll
          for (int k = 0; k < kTileK / 16; ++k) {
            if (NP == 2) {   // the small terms first
              mma_f16<CG>(d, da[NP - 1] + k * step_a, db[0] + k * step_b, idesc, kb | k);
              mma_f16<CG>(d, da[0] + k * step_a, db[NP - 1] + k * step_b, idesc, 1);
              mma_f16<CG>(d, da[0] + k * step_a, db[0] + k * step_b, idesc, 1);
            } else {
              mma_f16<CG>(d, da[0] + k * step_a, db[0] + k * step_b, idesc, kb | k);
            }
          }
          mma_commit<CG>(empty + 8 * s);
          if (++s == STAGES) {
            s = 0;
            ph ^= 1u;
          }
        }
        if (!ok) break;
        mma_commit<CG>(tm_full + 8 * buf);
        if (++buf == 2) {
          buf = 0;
          tph ^= 1u;
        }
      }
    }
  } else if (warp >= 4) {
    const uint32_t tm_empty0 = CG == 1 ? tm_empty : map_to_rank(tm_empty, 0);
    const int quarter = warp & 3;                          // the 32 lanes of tensor memory this warp can read
    const int col0 = CG == 1 ? 0 : ((warp - 4) >> 2) * 128;
    int buf = 0;
    uint32_t tph = 0;
    for (int tile = cluster; tile < p.total; tile += clusters) {
      int b, ti, tj;
      place(tile, b, ti, tj);
      if (!mbar_wait(tm_full + 8 * buf, tph, dead)) break;
      tc_fence_after();
      const int row = ti * T + (int)rank * 128 + quarter * 32 + lane;
      const bool mirror = (MODE == kModeGram || MODE == kModePoly) && ti != tj;
      const int64_t plane_s = (int64_t)p.M * p.ld_src, plane_d = (int64_t)p.M * p.ld_dst;
      const __half* src = p.src + b * NP * plane_s + (int64_t)row * p.ld_src;
      __half* dst = p.dst + b * NP * plane_d;
#pragma unroll 1
      for (int c = 0; c < 4; ++c) {
        const int col = tj * T + col0 + 32 * c;
        float v[32];
        tmem_load32(tmem + ((uint32_t)(quarter * 32) << 16) + buf * T + col0 + 32 * c, v);
        if (row < p.M && col < p.N) {
          if (MODE == kModeGram) {
  #pragma unroll
            for (int i = 0; i < 32; ++i) v[i] *= p.beta;
          } else {
  #pragma unroll
            for (int q = 0; q < 4; ++q) {   // rows are padded to 64, so a chunk of 32 columns never leaves its row
              alignas(16) __half h[8], l[8];
              *reinterpret_cast<uint4*>(h) = *reinterpret_cast<const uint4*>(src + col + 8 * q);
              if (NP == 2) *reinterpret_cast<uint4*>(l) = *reinterpret_cast<const uint4*>(src + plane_s + col + 8 * q);
  #pragma unroll
              for (int i = 0; i < 8; ++i) {
                float x = __half2float(h[i]);
                if (NP == 2) x += __half2float(l[i]);
                v[8 * q + i] = fmaf(p.alpha, x, p.beta * v[8 * q + i]);
              }
            }
          }
          if (MODE == kModeLast) {
  #pragma unroll
            for (int i = 0; i < 32; ++i) v[i] *= 1.f / kScaleX;
            const int n = min(32, p.N - col);
            if (p.out_type == kTypeF32)
              last_chunk<float>(p, b, row, col, n, v);
            else if (p.out_type == kTypeBF16)
              last_chunk<__nv_bfloat16>(p, b, row, col, n, v);
            else
              last_chunk<__half>(p, b, row, col, n, v);
          } else {
            alignas(16) __half h[32], l[32];
  #pragma unroll
            for (int i = 0; i < 32; ++i) {
              h[i] = __float2half_rn(v[i]);
              if (NP == 2) l[i] = __float2half_rn(v[i] - __half2float(h[i]));
            }
            __half* to = dst + (int64_t)row * p.ld_dst + col;
  #pragma unroll
            for (int q = 0; q < 4; ++q) {
              reinterpret_cast<uint4*>(to)[q] = reinterpret_cast<uint4*>(h)[q];
              if (NP == 2) reinterpret_cast<uint4*>(to + plane_d)[q] = reinterpret_cast<uint4*>(l)[q];
            }
            if (mirror) {   // 32 lanes write 32 neighbours of a row
  #pragma unroll
              for (int i = 0; i < 32; ++i) {
                if (col + i < p.N) {
                  dst[(int64_t)(col + i) * p.ld_dst + row] = h[i];
                  if (NP == 2) dst[plane_d + (int64_t)(col + i) * p.ld_dst + row] = l[i];
                }
              }
            }
          }
        }
        __syncwarp();
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        if (CG == 1)
          mbar_arrive(tm_empty + 8 * buf);
        else
          mbar_arrive_cluster(tm_empty0 + 8 * buf);
      }
      if (++buf == 2) {
        buf = 0;
        tph ^= 1u;
      }
    }
    fence_async_global();
  }
  __syncthreads();
  if (*dead) {   // a wait ran out: matrix instructions and the other CTA's copies may still be under way
    if (threadIdx.x == 0) atomicExch(p.status, 1);
    for (int i = 0; i < 200; ++i) __nanosleep(1000);
  }
  tc_fence_before();
  __syncthreads();
  if (CG == 2) cluster_sync();
  if (warp == 2) {
    tc_fence_after();
    tmem_free<CG>(tmem, Shape::kTmemCols);
  }
}

}  // namespace brace
