// Kernels of the orthogonalised update (Newton-Schulz) and of the momentum step around it (sm_100a).
//
// The iteration.  For a matrix G (rows x cols), X_0 = G / (||G||_F + eps) and
//     S = X X^T  (X^T X when rows > cols: the Gram matrix of the short side, m x m)
//     X <- a X + (b S + c S^2) X  (a X + X (b S + c S^2))
// `steps` times, computed as
//     S = X X^T;   P = a I + b S + c S S   or   T = b I + c S, P = a I + S T;   X <- P X  (X P)
// so that a product's epilogue scales, adds a constant on the diagonal and stores.  With two planes the form with T is
// taken: its epilogues read nothing.  With one plane T's own rounding would show (2.9e-3 against 2.2e-3 of the result
// at 512 x 2048), and S is read while the product still runs.  All singular vectors stay, every singular value s goes
// to a s + b s^3 + c s^5, so the values are pushed towards 1 and X towards the nearest matrix with orthonormal rows
// (columns).
//
// Number format.  The operands of all products are float16 times a power of two, with float32 accumulators.  That is
// possible because the iteration's values are bounded (the host checks the coefficients: singular values below 1.9,
// eigenvalues of T and P below 7.5), so X 2^14, S 2^14, T 2^13 and P 2^13 cannot overflow and entries down to 8e-9 stay
// normal; it keeps 11 bits where bfloat16, at the same rate, keeps 8.  An operand is the sum of two such planes (hi + lo,
// 22 bits) and a product is hi*hi + hi*lo + lo*hi: three times the matrix instructions.  One plane alone is there for
// callers who ask for it: 11 bits are enough for updates of full rank only, since an error outside the matrix's range
// grows by a a step.
//
// Symmetry.  S and P are symmetric: only tiles on and below the diagonal are computed and stored.  Where a product
// needs one above it, the stored tile is loaded instead and the matrix instruction reads it the other way (the
// descriptors allow either axis to be the contiguous one).  That takes a step from 2 m^2 k + 2 m^3 + 2 m^2 k
// operations to m^2 k + m^3 + 2 m^2 k, and nothing is written twice.
#pragma once

#include "elements.cuh"
#include "sm100.cuh"

namespace brace {

constexpr float kScaleX = 16384.f;                  // stored X = X * 2^14
constexpr float kGramScale = 1.f / 16384.f;         // X X^T * 2^28 -> S * 2^14
constexpr float kSquareScale = 8192.f;              // T, P -> T * 2^13, P * 2^13
constexpr float kFromGram = 0.5f;                   // S * 2^14 -> S * 2^13
constexpr float kPolyScale = 1.f / 16384.f;         // S T * 2^27 -> P * 2^13
constexpr float kStepScale = 1.f / 8192.f;          // P X * 2^27 -> X * 2^14

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
  uint32_t x = words[w] >> sh;
  if (sh + n > 32) x |= words[w + 1] << (32 - sh);
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
// place of its own, so the result is the same every time.  2048 x 2048 float32 with momentum: 10 us, 5 TB/s.
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
// How an operand lies in memory: with the contraction along its rows (contiguous), across them, or symmetric with the
// tiles on and below the diagonal stored.
enum { kAlong = 0, kAcross = 1, kSymmetric = 2 };

struct GemmArgs {
  int M, N, K;                  // result M x N, contraction K
  int tiles_n, tiles;           // tile columns, tiles per matrix
  int total;                    // tiles of all matrices
  int chunk;                    // stages per accumulator (two planes)
  float scale, diagonal;        // of the product, and added on its diagonal
  __half* dst;                  // [batch][planes][M][ld_dst]
  int64_t ld_dst;
  __half* dst2;                 // two planes, kModeGram: T beside S, scale2 * S + diagonal2 on the diagonal
  float scale2, diagonal2;      // one plane, kModePoly: scale2 * src is added
  const __half* src;            // S, laid out as dst
  // kModeLast: the result O, or the weights W_out = keep * W_in - rate * O for `replicas` copies
  void* out;
  const void* w_in;
  int64_t ld_out, batch_out, rep_out, ld_in, batch_in, rep_in;
  int vec_out, vec_in, replicas;
  float keep, rate;
  int* status;
};

constexpr int kTileK = 64;                       // contraction per stage: one 128-byte swizzle row
constexpr int kOperandBytes = 128 * kTileK * 2;  // an operand of a stage in one CTA: 128 rows (or columns)
// The tensor cores' float32 accumulation cuts off what does not fit, an error that no sign cancels: over a long
// contraction it adds up (2.4e-5 of the result at 512 x 2048, five steps).  With two planes the accumulators therefore
// hold `chunk` stages only and are added in registers, rounded to nearest.  One stage (K = 64) leaves no more error than
// products in plain float32 arithmetic from a short side of about 500 on (768 x 768: full rank 1.7e-6 against 2.7e-6, rank 4
// 5.6e-5 against 7.3e-5), and below that up to 1.7 times as much (64 x 64: 2.0e-6 against 1.2e-6).  Two stages leave up
// to twice one's (768 x 768: 3.0e-6, rank 4 9.9e-5) but take less time (4096 x 4096: 3.5 ms against 4.3): they are used
// where that is not seen, for bfloat16 results (rounded to 1.7e-3) and from the short side on where plain float32 is
// worse on every spectrum tried, full rank, 1 / i^2 and ranks 1, 4, 33 and 128: at 1600 x 1600 full rank 3.2e-6 against
// 3.5e-6, rank 4 1.12e-4 against 1.14e-4; at 1400 x 1400 rank 4 has 1.12e-4 against 1.05e-4.
constexpr int kLongChunkFrom = 1600;
constexpr int kCellBytes = 2048;                 // a warp's staging of the epilogue: 32 rows of 64 bytes

// An operand's tensor map(s), each with boxes that fill a stage's operand, all planes, in one load: the cost of a
// load is some 46 clocks and 2 for each 128 bytes (measured: 59 bytes a clock with 256 rows, 48 with 64).
//   along: 128 (64) rows of one block of 64 columns;  across: 64 rows of two blocks (one).
// A symmetric operand has both.
struct GemmMaps {
  CUtensorMap a[2], b[2];
};

// Tiles of 128 CG rows and TN columns by CG CTAs.
template <int CG, int TN, int NP>
struct GemmShape {
  static constexpr int kRows = 128 * CG;
  static constexpr int kColumns = TN / 4;                    // an epilogue warp takes 32 rows of so many columns
  static constexpr int kEpiWarps = 16;
  static constexpr int kThreads = 128 + 32 * kEpiWarps;      // warps 0-3: loads, MMAs, tensor memory, -; then epilogue
  static constexpr int kBytesB = TN / CG * kTileK * 2;       // each CTA of a pair loads half of the columns' operand
  static constexpr int kStageBytes = NP * (kOperandBytes + kBytesB);
  static constexpr int kStages = 192 * 1024 / kStageBytes;
  static constexpr int kBuffers = 512 / TN;                  // accumulators in tensor memory: all of its 512 columns
  static constexpr int kSmem = kStages * kStageBytes + kEpiWarps * kCellBytes + 1024 + 256;
};

// Tiles on and below the diagonal, row by row, `per` columns of tiles to a row of tiles: t -> (row, col).
__device__ __forceinline__ void triangle(int t, int per, int& row, int& col) {
  const int u = t / per;
  row = (int)((sqrtf(8.f * (float)u + 1.f) - 1.f) * 0.5f);
  while ((row + 1) * (row + 2) / 2 <= u) ++row;
  while (row * (row + 1) / 2 > u) --row;
  col = t - per * (row * (row + 1) / 2);
}

// A warp's cell: 32 rows of four 16-byte words.  A lane writes (reads) its own row, and reads (writes) rows of 4
// neighbouring lanes: word w of row r lies at w ^ ((r >> 1) & 3), so that neither way has bank conflicts.
__device__ __forceinline__ uint32_t cell_at(uint32_t cell, int r, int w) {
  return cell + (uint32_t)(r * 64 + ((w ^ ((r >> 1) & 3)) << 4));
}
__device__ __forceinline__ void sts16(uint32_t a, uint4 v) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ uint4 lds16(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
  return v;
}

// A 32 x 32 block to a padded float16 matrix: the lane's own row goes through the cell, 8 rows of 64 bytes per store.
__device__ __forceinline__ void block_store(uint32_t cell, const uint4 (&own)[4], __half* p, int64_t ld, int rows) {
  const int lane = threadIdx.x & 31;
  __syncwarp();
#pragma unroll
  for (int w = 0; w < 4; ++w) sts16(cell_at(cell, lane, w), own[w]);
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = i * 8 + (lane >> 2);
    const uint4 t = lds16(cell_at(cell, r, lane & 3));
    if (r < rows) *reinterpret_cast<uint4*>(p + r * ld + (lane & 3) * 8) = t;
  }
}

__device__ __forceinline__ uint4 pack8(const float* v) {
  uint4 t;
  __half2* h = reinterpret_cast<__half2*>(&t);
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
  return t;
}
// what 8 values lose in pack8
__device__ __forceinline__ uint4 pack8_rest(const float* v, const uint4& hi) {
  const __half* h = reinterpret_cast<const __half*>(&hi);
  float r[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = v[i] - __half2float(h[i]);
  return pack8(r);
}

// ... and back: fetched 8 rows at a time, the lane's own row times `scale` added to v.
__device__ __forceinline__ void block_fetch(const __half* p, int64_t ld, int rows, uint4 (&x)[4]) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = i * 8 + (lane >> 2);
    x[i] = r < rows ? *reinterpret_cast<const uint4*>(p + r * ld + (lane & 3) * 8) : make_uint4(0, 0, 0, 0);
  }
}
__device__ __forceinline__ void block_add(uint32_t cell, const uint4 (&x)[4], float scale, float* v) {
  const int lane = threadIdx.x & 31;
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 4; ++i) sts16(cell_at(cell, i * 8 + (lane >> 2), lane & 3), x[i]);
  __syncwarp();
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const uint4 t = lds16(cell_at(cell, lane, w));
    const __half* h = reinterpret_cast<const __half*>(&t);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[8 * w + j] = fmaf(scale, __half2float(h[j]), v[8 * w + j]);
  }
}

template <int NP>
__device__ __forceinline__ void store_planes(uint32_t cell, const float* v, __half* p, int64_t plane, int64_t ld, int rows) {
  uint4 o[4];
#pragma unroll
  for (int w = 0; w < 4; ++w) o[w] = pack8(v + 8 * w);
  block_store(cell, o, p, ld, rows);
  if (NP == 2) {
#pragma unroll
    for (int w = 0; w < 4; ++w) o[w] = pack8_rest(v + 8 * w, o[w]);
    block_store(cell, o, p + plane, ld, rows);
  }
}

// 32 x 16 results, staged as float32, to the caller's tensor: four neighbouring elements a lane.
template <typename T>
__device__ __forceinline__ void last_cell(const GemmArgs& p, uint32_t cell, int64_t b, int row0, int col0, const float* own) {
  const int lane = threadIdx.x & 31;
  __syncwarp();
#pragma unroll
  for (int w = 0; w < 4; ++w) sts16(cell_at(cell, lane, w), make_uint4(__float_as_uint(own[4 * w]), __float_as_uint(own[4 * w + 1]),
                                             __float_as_uint(own[4 * w + 2]), __float_as_uint(own[4 * w + 3])));
  __syncwarp();
  const int col = col0 + (lane & 3) * 4, n = min(4, p.N - col);
  if (n <= 0) return;
  const int r0 = lane >> 2;
  if (p.vec_out && p.vec_in && n == 4 && row0 + 32 <= p.M) {
    for (int k = 0; k < p.replicas; ++k) {
      T* out = (T*)p.out + b * p.batch_out + k * p.rep_out + (int64_t)(row0 + r0) * p.ld_out + col;
      Pack<T, 4> y[4];
      if (p.w_in) {
        const T* in = (const T*)p.w_in + b * p.batch_in + k * p.rep_in + (int64_t)(row0 + r0) * p.ld_in + col;
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i].load(in + i * 8 * p.ld_in);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint4 t = lds16(cell_at(cell, i * 8 + r0, lane & 3));
        const float o[4] = {__uint_as_float(t.x), __uint_as_float(t.y), __uint_as_float(t.z), __uint_as_float(t.w)};
#pragma unroll
        for (int j = 0; j < 4; ++j) y[i].t[j] = from_f32<T>(p.w_in ? p.keep * to_f32(y[i].t[j]) - p.rate * o[j] : o[j]);
        y[i].store_plain(out + i * 8 * p.ld_out);
      }
    }
    return;
  }
#pragma unroll 1
  for (int i = 0; i < 4; ++i) {
    const int r = i * 8 + r0, row = row0 + r;
    if (row >= p.M) break;
    const uint4 t = lds16(cell_at(cell, r, lane & 3));
    const float o[4] = {__uint_as_float(t.x), __uint_as_float(t.y), __uint_as_float(t.z), __uint_as_float(t.w)};
    for (int k = 0; k < p.replicas; ++k) {
      T* out = (T*)p.out + b * p.batch_out + k * p.rep_out + (int64_t)row * p.ld_out + col;
      const T* in = (const T*)p.w_in + b * p.batch_in + k * p.rep_in + (int64_t)row * p.ld_in + col;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (j < n) out[j] = from_f32<T>(p.w_in ? p.keep * to_f32(in[j]) - p.rate * o[j] : o[j]);
    }
  }
}

// Asks for the weights that a lane's row of `cols` columns will be added to, while the products still run.
template <typename T>
__device__ __forceinline__ void prefetch_weights(const GemmArgs& p, int64_t b, int row, int col, int cols) {
  const int n = min(cols, p.N - col);
  if (!p.w_in || row >= p.M || n <= 0) return;
  for (int k = 0; k < p.replicas; ++k) {
    const T* in = (const T*)p.w_in + b * p.batch_in + k * p.rep_in + (int64_t)row * p.ld_in + col;
    for (int j = 0; j < n; j += 128 / (int)sizeof(T)) asm volatile("prefetch.global.L2 [%0];" ::"l"(in + j));
    asm volatile("prefetch.global.L2 [%0];" ::"l"(in + n - 1));
  }
}

// Where there are too few tiles for the GPU, a cluster of KS CTAs shares the contraction of one (CG = 1): each sums its
// part of it, hands every other one its share of the columns, and finishes its own.  The shares go as bulk copies from
// shared memory to shared memory (the same as 16-byte stores of the lanes took 5 us for 2).  In both places the share
// of 32 / KS 16-byte words a row is swizzled by the row.
template <int KS>
struct Exchange {
  static constexpr int kWords = 32 / KS, kBytes = 128 * kWords * 16;   // of a share: 128 rows
  // what goes to CTA `to`, and what came from CTA `from`: where the stages were
  static __device__ __forceinline__ uint32_t out(uint32_t base, int to) { return base + (uint32_t)(to * kBytes); }
  static __device__ __forceinline__ uint32_t in(uint32_t base, int from) { return base + (uint32_t)((KS + from) * kBytes); }
  static __device__ __forceinline__ uint32_t word(uint32_t share, int row, int w) {
    return share + (uint32_t)((row * kWords + (w ^ (row & (kWords - 1)))) << 4);
  }
};

// 32 rows x 32 columns of a finished product: scaled, and stored as operand planes or as the caller's result.
template <int NP, int MODE, typename TOUT>
__device__ __forceinline__ void finish_block(const GemmArgs& p, uint32_t cell, int64_t b, int row0, int col0, int rows,
                                             const uint4 (&source)[4], float* v) {
  const int64_t plane = (int64_t)p.M * p.ld_dst, at = b * NP * plane + (int64_t)row0 * p.ld_dst + col0;
  const int own = row0 + (int)(threadIdx.x & 31) - col0;   // the diagonal's column in this lane's row
  if (MODE == kModeLast) {
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] *= kStepScale / kScaleX;
#pragma unroll
    for (int q = 0; q < 2; ++q) last_cell<TOUT>(p, cell, b, row0, col0 + 16 * q, v + 16 * q);
  } else {
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = fmaf(v[i], p.scale, MODE == kModePoly && i == own ? p.diagonal : 0.f);
    if (MODE == kModePoly && NP == 1) block_add(cell, source, p.scale2, v);
    store_planes<NP>(cell, v, p.dst + at, plane, p.ld_dst, rows);
    if (MODE == kModeGram && NP == 2) {
#pragma unroll
      for (int i = 0; i < 32; ++i) v[i] = fmaf(v[i], p.scale2, i == own ? p.diagonal2 : 0.f);
      store_planes<NP>(cell, v, p.dst2 + at, plane, p.ld_dst, rows);
    }
  }
}

// One product of the iteration over tiles of 128 x 128 (CG = 1) or, by a pair of CTAs, 256 x TN (CG = 2), NP planes
// per operand.  Warp 0 loads, warp 1 issues the matrix instructions, warp 2 owns the tensor memory, warps 4.. read the
// accumulators and write the results; persistent over tiles, so that the epilogue of a tile runs under the products
// of the next.  Bound by the matrix rate at large sizes: 4096 x 4096, five steps, one plane 1.03 ms, 1.33 PFLOP/s, in a
// short loop and 1.23 ms in one of seconds, where the power cap sustains 1.37 PFLOP/s of a library product; two planes
// 3.4 ms, 1.20 PFLOP/s, and 3.7; by launches, first loads and epilogues (some 4.5 us a product, 7 with two planes) below
// 1000.
template <int CG, int TN, int NP, int OP_A, int OP_B, int MODE, typename TOUT, int KS>
__global__ void __launch_bounds__(GemmShape<CG, TN, NP>::kThreads, 1)
    ortho_gemm_kernel(const __grid_constant__ GemmMaps maps, const GemmArgs p) {
  using Shape = GemmShape<CG, TN, NP>;
  constexpr int TM = Shape::kRows, STAGES = Shape::kStages, BUFS = Shape::kBuffers;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_addr(smem_raw) + 1023u) & ~1023u;
  const uint32_t cells = base + STAGES * Shape::kStageBytes;
  const uint32_t full = cells + Shape::kEpiWarps * kCellBytes, empty = full + 8 * STAGES;
  const uint32_t tm_full = empty + 8 * STAGES, tm_empty = tm_full + 8 * BUFS, shared_bar = tm_empty + 8 * BUFS;
  const uint32_t tail = shared_bar + 8;
  volatile int* dead = (volatile int*)(smem_raw + (tail - smem_addr(smem_raw)));
  uint32_t* tmem_slot = (uint32_t*)(smem_raw + (tail + 8 - smem_addr(smem_raw)));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  static_assert(KS == 1 || CG == 1, "a pair of CTAs does not share a contraction");
  const uint32_t rank = CG == 1 ? 0u : cluster_rank();
  const int part = KS == 1 ? 0 : (int)cluster_rank();

  if (threadIdx.x == 0) {
    *dead = 0;
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(full + 8 * s, 1);
      mbar_init(empty + 8 * s, 1);
    }
    for (int i = 0; i < BUFS; ++i) {
      mbar_init(tm_full + 8 * i, 1);
      mbar_init(tm_empty + 8 * i, CG * Shape::kEpiWarps);
    }
    if (KS > 1) {
      mbar_init(shared_bar, 1);
      mbar_expect_tx(shared_bar, (KS - 1) * Exchange<KS>::kBytes);
    }
    mbar_init_visible();
    tma_prefetch(&maps.a[0]);
    tma_prefetch(&maps.b[0]);
    if (OP_A == kSymmetric) tma_prefetch(&maps.a[1]);
    if (OP_B == kSymmetric) tma_prefetch(&maps.b[1]);
  }
  if (warp == 2) tmem_alloc<CG>(smem_addr(tmem_slot), 512);
  tc_fence_before();
  __syncthreads();
  if (CG == 2) cluster_sync();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  grid_trigger();   // the next kernel of the chain may set itself up; it reads nothing before this one is complete
  grid_wait();
  fence_async_global();

  const int cluster = blockIdx.x / (CG * KS), clusters = gridDim.x / (CG * KS);
  const int kall = (p.K + kTileK - 1) / kTileK, kfirst = kall * part / KS, kblocks = kall * (part + 1) / KS;
  auto place = [&](int tile, int& b, int& ti, int& tj) {
    b = tile / p.tiles;
    const int t = tile - b * p.tiles;
    if (MODE == kModeGram || MODE == kModePoly) {
      triangle(t, TM / TN, ti, tj);
    } else {
      ti = t / p.tiles_n;
      tj = t - ti * p.tiles_n;
    }
  };
  // whether the operand from row `row` on lies across the contraction in stage kb: of a symmetric one the blocks of TM
  // rows up to the diagonal block are stored
  auto across = [](int op, int row, int kb) { return op == kAcross || (op == kSymmetric && kb * kTileK >= (row / TM + 1) * TM); };

  // the launch's registers (640 threads x 96) go to the warps that hold accumulators: 4 x 32 x 32 + 16 x 32 x 112
  if (TN == 256 && warp < 4) asm volatile("setmaxnreg.dec.sync.aligned.u32 32;");
  constexpr int kAcc = NP == 1 ? 32 : Shape::kColumns;
  float acc[kAcc];
  if (warp == 0) {
    const bool lead = elect_one();
    const uint32_t full0 = CG == 1 ? full : map_to_rank(full, 0);
    int s = 0;
    uint32_t ph = 0, issued = 0;
    bool ok = true;
    for (int tile = cluster; ok && tile < p.total; tile += clusters) {
      int b, ti, tj;
      place(tile, b, ti, tj);
      const int ra = ti * TM + (int)rank * 128, rb = tj * TN + (int)rank * (TN / CG);
      for (int kb = kfirst; kb < kblocks; ++kb) {
        if (!mbar_wait(empty + 8 * s, ph ^ 1u, dead)) {
          ok = false;
          break;
        }
        const uint32_t st = base + s * Shape::kStageBytes, bar = full0 + 8 * s;
        const bool a_across = across(OP_A, ti * TM, kb), b_across = across(OP_B, tj * TN, kb);
        // the tensors as blocks of 64 columns: (column in the block, row, block, plane)
        const CUtensorMap* ma = &maps.a[OP_A == kSymmetric && a_across ? 1 : 0];
        const CUtensorMap* mb = &maps.b[OP_B == kSymmetric && b_across ? 1 : 0];
        if (lead) {
          if (rank == 0) mbar_expect_tx(full + 8 * s, CG * Shape::kStageBytes);
          tma_load<CG>(st, ma, 0, a_across ? kb * kTileK : ra, a_across ? ra / 64 : kb, b * NP, bar);
          tma_load<CG>(st + NP * kOperandBytes, mb, 0, b_across ? kb * kTileK : rb, b_across ? rb / 64 : kb, b * NP, bar);
        }
        __syncwarp();
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
  } else if (warp == 1) {
    if (rank == 0) {
      const bool lead = elect_one();
      const uint64_t desc0 = operand_desc(base, kOperandBytes / 2);
      int s = 0, buf = 0;
      uint32_t ph = 0, tph = 0;
      bool ok = true;
      for (int tile = cluster; ok && tile < p.total; tile += clusters) {
        int b, ti, tj;
        place(tile, b, ti, tj);
        for (int kb = kfirst; ok && kb < kblocks;) {
          if (!mbar_wait(tm_empty + 8 * buf, tph ^ 1u, dead)) {
            ok = false;
            break;
          }
          tc_fence_after();
          const uint32_t d = tmem + buf * TN;
          const int kend = NP == 1 ? kblocks : min(kblocks, kb + p.chunk);
          for (uint32_t add = 0; kb < kend; ++kb) {
            if (!mbar_wait(full + 8 * s, ph, dead)) {
              ok = false;
              break;
            }
            tc_fence_after();
            const bool a_across = across(OP_A, ti * TM, kb), b_across = across(OP_B, tj * TN, kb);
            const uint32_t idesc = f16_idesc(TM, TN, a_across, b_across);
            // per 16 of the contraction: 32 bytes along a swizzled row, or 16 rows of 128 bytes
            const uint64_t step_a = (a_across ? 2048 : 32) >> 4, step_b = (b_across ? 2048 : 32) >> 4;
            const uint64_t da = desc0 + (uint64_t)(s * Shape::kStageBytes >> 4), db = da + (NP * kOperandBytes >> 4);
            constexpr uint64_t lo_a = kOperandBytes >> 4, lo_b = Shape::kBytesB >> 4;   // the second plane
            if (lead) {
              if (kb + 1 < kall) {
#pragma unroll
                for (int k = 0; k < kTileK / 16; ++k) {
                  if (NP == 2) {   // the small terms first: what is cut off goes by the accumulators' size
                    mma_f16<CG>(d, da + lo_a + k * step_a, db + k * step_b, idesc, k ? 1 : add);
                    mma_f16<CG>(d, da + k * step_a, db + lo_b + k * step_b, idesc, 1);
                  }
                }
#pragma unroll
                for (int k = 0; k < kTileK / 16; ++k)
                  mma_f16<CG>(d, da + k * step_a, db + k * step_b, idesc, NP == 2 || k ? 1 : add);
              } else {             // past K the stage holds zeros: only as many as are needed
                const int steps = (p.K - kb * kTileK + 15) / 16;
#pragma unroll 1
                for (int k = 0; k < steps; ++k) {
                  if (NP == 2) {
                    mma_f16<CG>(d, da + lo_a + k * step_a, db + k * step_b, idesc, k ? 1 : add);
                    mma_f16<CG>(d, da + k * step_a, db + lo_b + k * step_b, idesc, 1);
                  }
                }
#pragma unroll 1
                for (int k = 0; k < steps; ++k)
                  mma_f16<CG>(d, da + k * step_a, db + k * step_b, idesc, NP == 2 || k ? 1 : add);
              }
              mma_commit<CG>(empty + 8 * s);
            }
            __syncwarp();
            add = 1;
            if (++s == STAGES) {
              s = 0;
              ph ^= 1u;
            }
          }
          if (!ok) break;
          if (lead) mma_commit<CG>(tm_full + 8 * buf);
          __syncwarp();
          if (++buf == BUFS) {
            buf = 0;
            tph ^= 1u;
          }
        }
      }
    }
  } else if (warp >= 4) {
    if (TN == 256) asm volatile("setmaxnreg.inc.sync.aligned.u32 112;");
    const uint32_t tm_empty0 = CG == 1 ? tm_empty : map_to_rank(tm_empty, 0);
    const int quarter = warp & 3;                          // the 32 lanes of tensor memory this warp can read
    const int cols0 = ((warp - 4) >> 2) * Shape::kColumns;
    const uint32_t cell = cells + (warp - 4) * kCellBytes;
    const uint32_t tm_mine = tmem + ((uint32_t)(quarter * 32) << 16) + cols0;
    int buf = 0;
    uint32_t tph = 0;
    bool ok = true;
    auto release = [&] {
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        if (CG == 1)
          mbar_arrive(tm_empty + 8 * buf);
        else
          mbar_arrive_cluster(tm_empty0 + 8 * buf);
      }
      if (++buf == BUFS) {
        buf = 0;
        tph ^= 1u;
      }
    };
    for (int tile = cluster; ok && tile < p.total; tile += clusters) {
      int b, ti, tj;
      place(tile, b, ti, tj);
      const int row0 = ti * TM + (int)rank * 128 + quarter * 32, col0 = tj * TN + cols0;
      const int rows = min(32, p.M - row0);   // may be none: the accumulators are then read for nothing
      // Rows are padded to 64 columns.  Of the pad this writes what shares 32 (with 256 columns a tile, 64) columns with the
      // matrix: zeros, since the operands' are; the rest holds what the workspace held.  Those columns are never contracted
      // (the last stage stops at the next multiple of 16), and as rows or columns of a result they end in pads alone.
      const bool live = rows > 0 && col0 < p.N;
      if (MODE == kModeLast) prefetch_weights<TOUT>(p, b, row0 + lane, col0, Shape::kColumns);
      uint4 x0[4], x1[4];
      if (MODE == kModePoly && NP == 1 && KS == 1 && live) {
        const __half* src = p.src + b * p.M * p.ld_dst + (int64_t)row0 * p.ld_dst + col0;
        block_fetch(src, p.ld_dst, rows, x0);
        if (Shape::kColumns == 64) block_fetch(src + 32, p.ld_dst, rows, x1);
      }
      if (NP == 2) {
        for (int kb = kfirst; kb < kblocks; kb += p.chunk) {
          if (!mbar_wait(tm_full + 8 * buf, tph, dead)) {
            ok = false;
            break;
          }
          tc_fence_after();
#pragma unroll
          for (int q = 0; q < Shape::kColumns / 16; ++q) {
            float v[16];
            tmem_load16(tm_mine + buf * TN + 16 * q, v);
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[(16 * q + i) % kAcc] = (kb > kfirst ? acc[(16 * q + i) % kAcc] : 0.f) + v[i];
          }
          release();
        }
      } else if (!mbar_wait(tm_full + 8 * buf, tph, dead)) {
        ok = false;
      } else {
        tc_fence_after();
      }
      if (!ok) break;
      if constexpr (KS > 1) {
        if (NP == 1) tmem_load32(tm_mine + buf * TN, *reinterpret_cast<float(*)[32]>(acc));
        break;   // one tile; it is finished below
      } else {
#pragma unroll
        for (int h = 0; h < Shape::kColumns / 32; ++h) {
          float* v = acc + (NP == 1 ? 0 : 32 * h);
          if (NP == 1) {
            tmem_load32(tm_mine + buf * TN + 32 * h, *reinterpret_cast<float(*)[32]>(v));
            if (h + 1 == Shape::kColumns / 32) release();
          }
          if (live) finish_block<NP, MODE, TOUT>(p, cell, b, row0, col0 + 32 * h, rows, h == 0 ? x0 : x1, v);
        }
      }
    }
    if (KS == 1) fence_async_global();
  }
  if constexpr (KS > 1) {
    using E = Exchange<KS>;
    int b, ti, tj;
    place(cluster, b, ti, tj);
    const int quarter = warp & 3, cols0 = ((warp - 4) >> 2) * 32, owner = cols0 / (128 / KS);   // of this warp's columns
    cluster_arrive();   // once all are here, no matrix instruction or load uses the stages any more
    if (warp >= 4) {
#pragma unroll
      for (int w = 0; w < 8; ++w)
        sts16(E::word(E::out(base, owner), quarter * 32 + lane, cols0 / 4 + w - owner * E::kWords),
              make_uint4(__float_as_uint(acc[4 * w]), __float_as_uint(acc[4 * w + 1]), __float_as_uint(acc[4 * w + 2]),
                         __float_as_uint(acc[4 * w + 3])));
      fence_async();
      // 32 rows of an owner's share are one piece: KS == 2 has two warps' words in each row
      if (KS == 2) asm volatile("bar.sync %0, 64;" ::"r"(2 + quarter * 2 + owner) : "memory");
    }
    __syncwarp();
    cluster_wait();
    if (warp >= 4) {
      if (lane == 0 && owner != part && (KS == 4 || ((warp - 4) >> 2) % 2 == 0))
        copy_to_cta(map_to_rank(E::in(base, part) + quarter * (E::kBytes / 4), (uint32_t)owner),
                    E::out(base, owner) + quarter * (E::kBytes / 4), E::kBytes / 4, map_to_rank(shared_bar, (uint32_t)owner));
      asm volatile("bar.sync 1, 512;" ::: "memory");   // this CTA's own share is there
      mbar_wait(shared_bar, 0, dead);
    }
    constexpr int kBlocks = 4 / KS;   // blocks of 32 columns of this CTA's share
    const int block = (warp - 4) >> 2;
    if (warp >= 4 && block < kBlocks) {
      const int row0 = ti * TM + quarter * 32, col0 = tj * TN + (part * kBlocks + block) * 32, rows = min(32, p.M - row0);
      if (rows > 0 && col0 < ((p.N + 63) & ~63)) {
        uint4 x0[4];
        if (MODE == kModePoly && NP == 1)
          block_fetch(p.src + b * p.M * p.ld_dst + (int64_t)row0 * p.ld_dst + col0, p.ld_dst, rows, x0);
#pragma unroll
        for (int i = 0; i < 32; ++i) acc[i] = 0.f;
        for (int q = 0; q < KS; ++q) {
          const uint32_t share = q == part ? E::out(base, q) : E::in(base, q);
#pragma unroll
          for (int w = 0; w < 8; ++w) {
            const uint4 t = lds16(E::word(share, quarter * 32 + lane, block * 8 + w));
            acc[4 * w] += __uint_as_float(t.x);
            acc[4 * w + 1] += __uint_as_float(t.y);
            acc[4 * w + 2] += __uint_as_float(t.z);
            acc[4 * w + 3] += __uint_as_float(t.w);
          }
        }
        finish_block<NP, MODE, TOUT>(p, cells + (warp - 4) * kCellBytes, b, row0, col0, rows, x0, acc);
      }
    }
    fence_async_global();
    __syncwarp();
    cluster_sync();   // the others have what was copied to them from here
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
    tmem_free<CG>(tmem, 512);
  }
}

// ---------------------------------------------------------------------------------------------------------------
// Matrices with a short side of at most 128: the whole iteration in one launch, on chip.
//
// A cluster of CTAs holds one matrix; each keeps a slice of the long side as float16 operand planes in shared memory
// for all steps.  Per step a CTA forms its slice's share of S, the
// cluster adds the shares through distributed shared memory (each CTA adds the rows that it owns and hands them to
// all), and every CTA forms P itself and takes its slice to P X.
// At these sizes nothing is bound by bandwidth or by the products (a 128 x 128 product is some 0.3 us); what counts is
// the chain of dependent steps, which as separate launches costs a launch and a round trip through L2 each: with one plane
// 128 x 128 takes 23 us (a step 4.2: products 0.6 each, epilogues 0.7 to 0.9) against 68 in launches of tiles, with two
// 38; 40 x 40 15 and 21.  Several CTAs spend 4 to 7 us a step on the exchange of S: one plane 128 x 512 takes 49 us against
// 78, two planes 67, 128 x 1024 72 against 154 and 128 x 2048, by 16 CTAs, 83.
// ---------------------------------------------------------------------------------------------------------------

struct ResidentArgs {
  PrepArgs prep;
  GemmArgs last;
  int m;              // short side
  int slice;          // long side per CTA, a multiple of 64
  int tall;           // the long side are the rows
  int steps;
  int out_type;
  float a, b, c;
};

constexpr int kResidentThreads = 512;
constexpr int kSquareBytes = 128 * 128 * 2;   // one plane of S or P
constexpr int kResidentSmem = 226 * 1024;     // at most

// The operand planes of X, of S / P, and (several CTAs) the shares of S.
inline int64_t resident_smem(int planes, int slice, int ctas) {
  return (int64_t)planes * (128 * slice * 2 + kSquareBytes) + (ctas > 1 ? (128 + ctas) * 512 : 0) + 1024;
}

// A 16-byte word of a swizzled operand: `word` of row `row` of a block of 64 columns.
__device__ __forceinline__ uint32_t swizzled(uint32_t block, int row, int word) {
  return block + (uint32_t)(row * 128 + ((word ^ (row & 7)) << 4));
}

// 32 columns of the accumulators of a tall matrix: the lanes hold neighbours of a row of the result.
template <typename T>
__device__ __forceinline__ void last_columns(const GemmArgs& p, int64_t b, int row0, int rows, int col, const float (&o)[32]) {
  if (col >= p.N) return;
  for (int k = 0; k < p.replicas; ++k) {
    T* out = (T*)p.out + b * p.batch_out + k * p.rep_out + (int64_t)row0 * p.ld_out + col;
    const T* in = p.w_in ? (const T*)p.w_in + b * p.batch_in + k * p.rep_in + (int64_t)row0 * p.ld_in + col : nullptr;
    T w[32];
    if (in) {
#pragma unroll
      for (int j = 0; j < 32; ++j) w[j] = j < rows ? in[j * p.ld_in] : from_f32<T>(0.f);
    }
#pragma unroll
    for (int j = 0; j < 32; ++j)
      if (j < rows) out[j * p.ld_out] = from_f32<T>(in ? p.keep * to_f32(w[j]) - p.rate * o[j] : o[j]);
  }
}

template <int NP, int TYPE>
__global__ void __launch_bounds__(kResidentThreads, 1) ortho_resident_kernel(const __grid_constant__ ResidentArgs p) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ double s_sum[16], s_part[16];
  __shared__ alignas(8) uint64_t s_bar;
  __shared__ uint32_t s_tmem;
  __shared__ int s_dead;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  uint32_t ctas;
  asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(ctas));
  const int rank = ctas > 1 ? (int)cluster_rank() : 0;
  const int64_t b = blockIdx.x / ctas;
  const uint32_t base = (smem_addr(smem_raw) + 1023u) & ~1023u;
  const uint32_t x_plane = 128u * (uint32_t)p.slice * 2u;
  const uint32_t sm_x = base, sm_s = sm_x + NP * x_plane, sm_share = sm_s + NP * kSquareBytes;
  const uint32_t x_block = p.tall ? (uint32_t)p.slice * 128u : 128u * 128u;   // 64 columns of all rows
  const uint32_t bar = smem_addr(&s_bar);
  volatile int* dead = &s_dead;
  const int m = p.m;
  // this CTA's part of the matrix
  const int long_side = p.tall ? p.prep.rows : p.prep.cols;
  const int at = rank * p.slice, width = min(p.slice, long_side - at);   // never empty
  const int row0 = p.tall ? at : 0, col0 = p.tall ? 0 : at;
  const int rows = p.tall ? width : m, cols = p.tall ? m : width;

  if (tid == 0) {
    s_dead = 0;
    mbar_init(bar, 1);
    mbar_init_visible();
  }
  const uint32_t tmem_cols = NP == 1 && p.slice <= 128 ? 256 : 512;
  if (warp == 0) tmem_alloc<1>(smem_addr(&s_tmem), tmem_cols);
  // pads of the operands are zeros: rows and columns past the matrix take part in the products
  for (uint32_t i = tid * 16; i < NP * (x_plane + kSquareBytes); i += kResidentThreads * 16)
    sts16(sm_x + i, make_uint4(0, 0, 0, 0));
  __syncthreads();
  grid_trigger();   // after the allocation of tensor memory: what is launched next cannot take it first
  grid_wait();
  if (blockIdx.x == 0 && tid == 0) *p.prep.status = 0;

  // momentum and sum of squares, as in ortho_norm_kernel; what is orthogonalised stays in registers (at most 128 x 256
  // elements, 8 groups of 8 a thread), all loads of four groups first
  const int units_row = (cols + 7) / 8, units = rows * units_row;
  const bool whole = cols % 8 == 0;
  float held[8][8];
  double sum = 0;
#pragma unroll
  for (int h = 0; h < 8; h += 4) {
    if (h * kResidentThreads >= units) break;
    float mo[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int u = tid + (h + i) * kResidentThreads, at_u = min(u, units - 1);   // past the end: read again, not used
      const int r = at_u / units_row, c = (at_u - r * units_row) * 8, row = row0 + r, col = col0 + c, n = min(8, cols - c);
      load_g<TYPE>(p.prep, b, row, col, whole ? 8 : n, held[h + i]);
      if (p.prep.m_in && u < units)   // in place, another thread's elements may be written at any time
        load8(p.prep.m_in + b * p.prep.batch_m_in + (int64_t)row * p.prep.ld_m_in + col, p.prep.vec_m_in, whole ? 8 : n, mo[i]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int u = tid + (h + i) * kResidentThreads;
      if (u >= units) continue;
      const int r = u / units_row, c = (u - r * units_row) * 8, n = min(8, cols - c);
      float(&g)[8] = held[h + i];
      if (p.prep.m_in) {
#pragma unroll
        for (int j = 0; j < 8; ++j) mo[i][j] = fmaf(p.prep.beta, mo[i][j], g[j]);
        store8(p.prep.m_out + b * p.prep.batch_m_out + (int64_t)(row0 + r) * p.prep.ld_m_out + col0 + c, p.prep.vec_m_out, n, mo[i]);
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] = p.prep.nesterov ? fmaf(p.prep.beta, mo[i][j], g[j]) : mo[i][j];
      }
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < n) sum = fma((double)g[j], (double)g[j], sum);
    }
  }
  sum = block_sum(sum, s_sum);
  if (ctas > 1) {
    cluster_sync();   // every CTA runs before its memory is written
    if (tid < (int)ctas) st_cluster_f64(map_to_rank(smem_addr(&s_part[rank]), (uint32_t)tid), sum);
    cluster_sync();
    sum = 0;
    for (uint32_t i = 0; i < ctas; ++i) sum += s_part[i];
  }
  const float inv = (float)((double)kScaleX / (sqrt(sum) + (double)p.prep.eps));

  // X_0: the operand planes
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int u = tid + i * kResidentThreads;
    if (u >= units) break;
    const int r = u / units_row, c8 = u - r * units_row;
#pragma unroll
    for (int j = 0; j < 8; ++j) held[i][j] *= inv;
    const uint32_t to = swizzled(sm_x + (uint32_t)(c8 >> 3) * x_block, r, c8 & 7);
    const uint4 hi = pack8(held[i]);
    sts16(to, hi);
    if (NP == 2) sts16(to + x_plane, pack8_rest(held[i], hi));
  }
  fence_async();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = s_tmem;
  const int quarter = warp & 3, group = warp >> 2;   // lanes of tensor memory, and which 32 columns of every 128
  const uint32_t tm_s = tmem + ((uint32_t)(quarter * 32) << 16);
  const int mrow = quarter * 32 + lane;              // this thread's row of the short side
  const int k_long = (width + 15) / 16, k_short = (m + 15) / 16;
  const uint32_t n_short = (uint32_t)k_short * 16, n_long = (uint32_t)k_long * 16;
  const int x_groups = (width + 31) / 32;            // groups of 32 columns of the accumulators of X
  uint32_t ph = 0;

  // One product, issued by one lane of warp 0 and waited for by all: D = A B, with two planes in parts of 64 of the
  // contraction in accumulators of their own (d_part columns apart), which are added in registers: see kLongChunkFrom.
  // Operands: A B over `ks` steps of 16, operands at
  // desc + k * step (within a block of 64 of the contraction: `fold` steps) + block steps.
  auto product = [&](uint32_t d, uint32_t d_part, uint32_t a, uint32_t a_lo, uint32_t a_blocks, bool a_across, uint32_t bb, uint32_t b_lo,
                     uint32_t b_blocks, bool b_across, int ks, uint32_t n) {
    if (warp == 0) {
      tc_fence_after();
      const bool lead = elect_one();
      const uint32_t idesc = f16_idesc(128, (int)n, a_across, b_across);
      const uint64_t da0 = operand_desc(a, a_blocks), db0 = operand_desc(bb, b_blocks);
      for (int k0 = 0; k0 < ks; k0 += 4) {
        // the small terms first: what is cut off goes by the accumulators' size
        for (int pass = NP == 2 ? 0 : 1; pass < 2; ++pass) {
          for (int k = k0; k < min(ks, k0 + 4); ++k) {
            const uint64_t da = da0 + (a_across ? (uint32_t)k * 128u : (uint32_t)(k >> 2) * (a_blocks >> 4) + (uint32_t)(k & 3) * 2u);
            const uint64_t db = db0 + (b_across ? (uint32_t)k * 128u : (uint32_t)(k >> 2) * (b_blocks >> 4) + (uint32_t)(k & 3) * 2u);
            if (lead) {
              if (pass == 0) {
                mma_f16<1>(d, da + (a_lo >> 4), db, idesc, k > k0);
                mma_f16<1>(d, da, db + (b_lo >> 4), idesc, 1);
              } else {
                mma_f16<1>(d, da, db, idesc, NP == 2 || k);
              }
            }
          }
        }
        if (NP == 2) d += d_part;
      }
      if (lead) mma_commit<1>(bar);
      __syncwarp();
    }
    mbar_wait(bar, ph, dead);   // where it runs out the results are not valid, but every CTA goes the same way
    ph ^= 1u;
    tc_fence_after();
  };

  // 32 columns of a product
  auto result = [&](uint32_t at, uint32_t part, int ks, float (&v)[32]) {
    tmem_load32(at, v);
    if (NP == 2) {
      for (int k = 4; k < ks; k += 4) {
        at += part;
        float y[16];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          tmem_load16(at + 16 * h, y);
#pragma unroll
          for (int j = 0; j < 16; ++j) v[16 * h + j] += y[j];
        }
      }
    }
  };
  const uint32_t x_at = NP == 1 ? 128u : 0u, x_part = (uint32_t)p.slice;   // accumulators of P X

  for (int step = 0; step < p.steps; ++step) {
    // S = X X^T over this slice
    product(tmem, 128, sm_x, x_plane, x_block, p.tall, sm_x, x_plane, x_block, p.tall, k_long, n_short);
    const bool mine = 32 * group < m;   // this warp's 32 columns of S exist
    float v[32];
    if (mine) result(tm_s + 32 * group, 128, k_long, v);
    if (ctas == 1) {
      if (mine) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
#pragma unroll
          for (int j = 0; j < 8; ++j) v[8 * w + j] *= kGramScale;
          const uint32_t to = swizzled(sm_s + (uint32_t)(group >> 1) * 16384u, mrow, (group & 1) * 4 + w);
          const uint4 hi = pack8(v + 8 * w);
          sts16(to, hi);
          if (NP == 2) sts16(to + kSquareBytes, pack8_rest(v + 8 * w, hi));
        }
      }
    } else {
      // the shares to the rows' owners: [share][row of the owner][128], words swizzled by the row
      const int own = (m + (int)ctas - 1) / (int)ctas;
      if (mine && mrow < m) {
        const int owner = mrow / own, r = mrow - owner * own;
        const uint32_t to = map_to_rank(sm_share + (uint32_t)((rank * own + r) * 512 + group * 128), (uint32_t)owner);
#pragma unroll
        for (int w = 0; w < 8; ++w)
          st_cluster16(to + (uint32_t)((w ^ (r & 7)) << 4),
                       make_uint4(__float_as_uint(v[4 * w]), __float_as_uint(v[4 * w + 1]), __float_as_uint(v[4 * w + 2]),
                                  __float_as_uint(v[4 * w + 3])));
      }
      cluster_sync();
      // the owner adds its rows' shares, in the order of the CTAs, and hands 8 columns at a time to all
      const int words = (int)n_short / 8, first = rank * own, have = max(0, min(own, m - first));
      for (int u = tid; u < have * words; u += kResidentThreads) {
        const int r = u / words, c8 = u - r * words;
        float t[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) t[j] = 0.f;
        for (int q = 0; q < (int)ctas; ++q) {
          const uint32_t from = sm_share + (uint32_t)((q * own + r) * 512 + (c8 >> 2) * 128);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint4 x = lds16(from + (uint32_t)(((((c8 & 3) * 2) + h) ^ (r & 7)) << 4));
            t[4 * h] += __uint_as_float(x.x);
            t[4 * h + 1] += __uint_as_float(x.y);
            t[4 * h + 2] += __uint_as_float(x.z);
            t[4 * h + 3] += __uint_as_float(x.w);
          }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) t[j] *= kGramScale;
        const uint32_t to = swizzled(sm_s + (uint32_t)(c8 >> 3) * 16384u, first + r, c8 & 7);
        const uint4 hi = pack8(t), lo = NP == 2 ? pack8_rest(t, hi) : hi;
        for (uint32_t q = 0; q < ctas; ++q) {
          st_cluster16(map_to_rank(to, q), hi);
          if (NP == 2) st_cluster16(map_to_rank(to + kSquareBytes, q), lo);
        }
      }
      fence_async();
      cluster_sync();
    }
    fence_async();
    tc_fence_before();
    __syncthreads();

    // P = a I + b S + c S^2, in place of S
    product(tmem, 128, sm_s, kSquareBytes, 16384u, false, sm_s, kSquareBytes, 16384u, false, k_short, n_short);
    if (mine) {
      result(tm_s + 32 * group, 128, k_short, v);
      const int own = mrow - 32 * group;   // the diagonal's column in this lane's row
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const uint32_t at_s = swizzled(sm_s + (uint32_t)(group >> 1) * 16384u, mrow, (group & 1) * 4 + w);
#pragma unroll
        for (int j = 0; j < 8; ++j)
          v[8 * w + j] = fmaf(v[8 * w + j], p.c * kFromGram * kGramScale, own == 8 * w + j && mrow < m ? p.a * kSquareScale : 0.f);
#pragma unroll
        for (int pl = NP - 1; pl >= 0; --pl) {
          const uint4 x = lds16(at_s + pl * kSquareBytes);
          const __half* h = reinterpret_cast<const __half*>(&x);
#pragma unroll
          for (int j = 0; j < 8; ++j) v[8 * w + j] = fmaf(p.b * kFromGram, __half2float(h[j]), v[8 * w + j]);
        }
        const uint4 hi = pack8(v + 8 * w);
        sts16(at_s, hi);
        if (NP == 2) sts16(at_s + kSquareBytes, pack8_rest(v + 8 * w, hi));
      }
    }
    fence_async();
    tc_fence_before();
    __syncthreads();

    // X <- P X
    product(tmem + x_at, x_part, sm_s, kSquareBytes, 16384u, false, sm_x, x_plane, x_block, !p.tall, k_short, n_long);
    if (step + 1 == p.steps) break;
    for (int g = group; g < x_groups; g += 4) {
      result(tm_s + x_at + 32 * g, x_part, k_short, v);
#pragma unroll
      for (int w = 0; w < 4; ++w) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[8 * w + j] *= kStepScale;
        const uint4 hi = pack8(v + 8 * w), lo = NP == 2 ? pack8_rest(v + 8 * w, hi) : hi;
        if (p.tall) {   // neighbouring lanes are neighbours in memory: two bytes each
#pragma unroll
          for (int pl = 0; pl < NP; ++pl) {
            const unsigned short* h = reinterpret_cast<const unsigned short*>(pl ? &lo : &hi);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const uint32_t to = swizzled(sm_x + pl * x_plane + (uint32_t)(mrow >> 6) * x_block, 32 * g + 8 * w + j, (mrow & 63) >> 3);
              asm volatile("st.shared.u16 [%0], %1;" ::"r"(to + (uint32_t)(mrow & 7) * 2u), "h"(h[j]) : "memory");
            }
          }
        } else {
          const uint32_t to = swizzled(sm_x + (uint32_t)(g >> 1) * x_block, mrow, (g & 1) * 4 + w);
          sts16(to, hi);
          if (NP == 2) sts16(to + x_plane, lo);
        }
      }
    }
    fence_async();
    tc_fence_before();
    __syncthreads();
  }

  // the result, or the weights
  for (int g = group; g < x_groups; g += 4) {
    float v[32];
    result(tm_s + x_at + 32 * g, x_part, k_short, v);
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] *= kStepScale / kScaleX;
    if (p.tall) {
      const int first = at + 32 * g, n = min(32, long_side - first);
      if (p.out_type == kTypeF32)
        last_columns<float>(p.last, b, first, n, mrow, v);
      else if (p.out_type == kTypeBF16)
        last_columns<__nv_bfloat16>(p.last, b, first, n, mrow, v);
      else
        last_columns<__half>(p.last, b, first, n, mrow, v);
    } else {
      const uint32_t cell = sm_s + (uint32_t)warp * kCellBytes;   // P is used up
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        if (p.out_type == kTypeF32)
          last_cell<float>(p.last, cell, b, quarter * 32, at + 32 * g + 16 * q, v + 16 * q);
        else if (p.out_type == kTypeBF16)
          last_cell<__nv_bfloat16>(p.last, cell, b, quarter * 32, at + 32 * g + 16 * q, v + 16 * q);
        else
          last_cell<__half>(p.last, cell, b, quarter * 32, at + 32 * g + 16 * q, v + 16 * q);
      }
    }
  }
  __syncthreads();
  if (*dead) {   // a wait ran out: let what may still be under way end before the memory goes
    if (tid == 0) atomicExch(p.prep.status, 1);
    for (int i = 0; i < 200; ++i) __nanosleep(1000);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 0) {
    tc_fence_after();
    tmem_free<1>(tmem, tmem_cols);
  }
}

}  // namespace brace
