// Host side of the language-model operators: argument checks, workspaces, tensor maps and kernel launches.
// C ABI declared in brace.h.
#include "brace.h"

#include <algorithm>
#include <atomic>
#include <cmath>
#include <type_traits>

#include "embedding_kernels.cuh"
#include "host.cuh"
#include "ortho_kernels.cuh"

using namespace brace;

namespace {

// ---- the orthogonalisation --------------------------------------------------------------------------------------

constexpr int kMaxNormBlocks = 512;
constexpr int kPrepBlocks = 1184;   // CTAs of the element-wise passes that fill the GPU: 148 SMs x 8

bool coefficients_ok(const brace_ortho_params* p) {
  if (!p || p->steps < 1 || p->steps > 1000) return false;
  if (!std::isfinite(p->a) || !std::isfinite(p->b) || !std::isfinite(p->c)) return false;
  if (!std::isfinite(p->eps) || !(p->eps >= 1e-30f)) return false;
  if (p->precision < BRACE_ORTHO_AUTO || p->precision > BRACE_ORTHO_SINGLE) return false;
  // upper bound of the singular values, step by step: the extremes of s -> a s + b s^3 + c s^5 on [0, top]
  const double a = p->a, b = p->b, c = p->c;
  double top = 1.0;
  for (int k = 0; k < p->steps; ++k) {
    const double t_top = top * top;
    // eigenvalues of T = b + c t and of P = a + b t + c t^2, t up to top^2
    double q = std::fmax(std::fmax(std::fabs(a), std::fabs(a + b * t_top + c * t_top * t_top)),
                         std::fmax(std::fabs(b), std::fabs(b + c * t_top)));
    double next = std::fabs(top * (a + b * t_top + c * t_top * t_top));
    if (c != 0.0) {
      const double tq = -b / (2 * c);   // extreme of P
      if (tq > 0 && tq < t_top) q = std::fmax(q, std::fabs(a + b * tq + c * tq * tq));
      const double disc = 9 * b * b - 20 * a * c;
      if (disc >= 0)
        for (int sg = -1; sg <= 1; sg += 2) {
          const double t = (-3 * b + sg * std::sqrt(disc)) / (10 * c);
          if (t > 0 && t < t_top) next = std::fmax(next, std::fabs(std::sqrt(t) * (a + b * t + c * t * t)));
        }
    } else if (b != 0.0) {
      const double t = -a / (3 * b);
      if (t > 0 && t < t_top) next = std::fmax(next, std::fabs(std::sqrt(t) * (a + b * t)));
    }
    if (!(q <= 7.5) || !(next <= 1.9)) return false;
    if (k > 64 && next <= top) break;   // the bound has settled
    top = std::fmax(next, 0.0);
  }
  return true;
}

struct OrthoPlan {
  int batch, rows, cols, m;   // m: the short side
  int planes, chunk;          // chunk: stages per accumulator (two planes)
  int64_t ld_x, ld_s;
  int norm_blocks;
  size_t off_partial, off_x[2], off_s, off_t[2], off_p, bytes;   // T of even and of odd steps
};

OrthoPlan make_plan(int32_t batch, int32_t rows, int32_t cols, const brace_ortho_params* p, int out_type) {
  OrthoPlan q;
  q.batch = batch;
  q.rows = rows;
  q.cols = cols;
  q.m = rows < cols ? rows : cols;
  // One plane only where the caller asks for it, for bfloat16 results too: what the rounding of an operand puts outside
  // the matrix's range grows by a = 3.4445 a step, 485 times over five, which 11 bits have no room for (1024 x 4096 in
  // bfloat16: rank 1 1.5e-1, rank 33 2.7e-2, full rank 1.9e-3 in 186 us; with two planes 1.7e-3, the result's own
  // rounding, for all of them in 358 us).
  const bool single = p->precision != BRACE_ORTHO_HALF;
  q.planes = single ? 2 : 1;
  q.chunk = out_type == BRACE_TYPE_BF16 || q.m >= kLongChunkFrom ? 2 : 1;
  q.ld_x = round_up(cols, 64);
  q.ld_s = round_up(q.m, 64);
  const int64_t units = (int64_t)rows * ((cols + 7) / 8);
  int64_t nb = (units + 511) / 512;
  const int64_t per = (kPrepBlocks + batch - 1) / batch;
  if (nb > per) nb = per;
  if (nb > kMaxNormBlocks) nb = kMaxNormBlocks;
  q.norm_blocks = (int)(nb < 1 ? 1 : nb);
  size_t at = 256;   // status word
  auto take = [&at](int64_t bytes) {
    const size_t here = at;
    at += (size_t)round_up(bytes, 256);
    return here;
  };
  q.off_partial = take((int64_t)batch * q.norm_blocks * 8);
  const int64_t xb = (int64_t)batch * q.planes * rows * q.ld_x * 2, sb = (int64_t)batch * q.planes * q.m * q.ld_s * 2;
  q.off_x[0] = take(xb);
  q.off_x[1] = take(xb);
  q.off_s = take(sb);
  // Where bfloat16 is asked for, T lies where the step's X goes: that place is free until then, and the workspace stays
  // a fifth smaller than float32's.
  const bool in_x = out_type == BRACE_TYPE_BF16;
  const size_t apart = take(single && !in_x ? sb : 0);
  for (int k = 0; k < 2; ++k) q.off_t[k] = in_x ? q.off_x[k ^ 1] : apart;
  q.off_p = take(sb);
  q.bytes = at;
  return q;
}

bool sizes_ok(int32_t batch, int32_t rows, int32_t cols) { return batch >= 0 && rows >= 0 && cols >= 0; }
bool sizes_served(int32_t batch, int32_t rows, int32_t cols) {
  return batch <= 32767 && (int64_t)rows * (((int64_t)cols + 63) / 64 * 8) < (int64_t)1 << 31;
}

// A matrix of operand planes in the workspace and its tensor maps, made when a launch first needs them: [planes of all
// matrices][rows][ld] float16 as blocks of 64 columns; a box holds the planes of `span` rows of a block (along) or of
// 64 rows of span / 64 blocks (across); 128-byte swizzle, zeros outside.
struct Operand {
  void* base;
  int64_t rows, ld, z;
  int planes;
  CUtensorMap map[2][2];   // [across][span 64 or 128]
  bool made[2][2];
  const CUtensorMap* get(bool across, int span) {
    const int s = span == 128;
    if (!made[across][s]) {
      EncodeFn enc = encode_fn();
      if (!enc) return nullptr;
      const cuuint64_t dim[4] = {64, (cuuint64_t)rows, (cuuint64_t)(ld / 64), (cuuint64_t)z};
      const cuuint64_t stride[3] = {(cuuint64_t)ld * 2, 128, (cuuint64_t)ld * 2 * (cuuint64_t)rows};
      const cuuint32_t box[4] = {64, across ? 64u : (cuuint32_t)span, across ? (cuuint32_t)span / 64 : 1u, (cuuint32_t)planes};
      const cuuint32_t one[4] = {1, 1, 1, 1};
      if (enc(&map[across][s], CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, base, dim, stride, box, one,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return nullptr;
      made[across][s] = true;
    }
    return &map[across][s];
  }
};

template <int CG, int TN, int NP, int OP_A, int OP_B, int MODE, typename TOUT, int KS>
cudaError_t launch_gemm_as(Operand& a, Operand& b, const GemmArgs& g, cudaStream_t st) {
  using Shape = GemmShape<CG, TN, NP>;
  auto* kernel = ortho_gemm_kernel<CG, TN, NP, OP_A, OP_B, MODE, TOUT, KS>;
  GemmMaps maps = {};   // first the one that the operand needs (a symmetric one needs both)
  auto put = [](CUtensorMap* to, Operand& x, int op, int span) {
    const CUtensorMap* first = x.get(op == kAcross, span);
    const CUtensorMap* second = op == kSymmetric ? x.get(true, span) : first;
    if (!first || !second) return false;
    to[0] = *first;
    to[1] = *second;
    return true;
  };
  if (!put(maps.a, a, OP_A, 128) || !put(maps.b, b, OP_B, TN / CG)) return cudaErrorNotSupported;
  static std::atomic<uint64_t> granted{0};   // devices on which this kernel may use its shared memory
  int dev = 0;
  cudaError_t err = cudaGetDevice(&dev);
  if (err != cudaSuccess) return err;
  const uint64_t bit = 1ull << (dev & 63);
  if (!(granted.load(std::memory_order_relaxed) & bit)) {
    err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape::kSmem);
    if (err != cudaSuccess) return err;
    granted.fetch_or(bit, std::memory_order_relaxed);
  }
  int clusters = KS > 1 ? g.total : sm_count() / CG;
  if (clusters > g.total) clusters = g.total;
  return launch(kernel, dim3((unsigned)(clusters * CG * KS)), Shape::kThreads, Shape::kSmem, CG * KS, st, maps, g);
}

// CTAs that share the contraction of a tile, where the tiles alone leave SMs idle: sharing costs an exchange and saves
// its part of the stages (0.2 us each, 0.65 with two planes): 512 x 2048 in float32 259 -> 166 us.  The costs are the
// ones that choose best between 130 x 130 and 1500 x 1500: with 1 for one plane 512 x 512 takes 111 us for 89, with 2 for
// two planes 200 x 200 takes 128 us for 119.
// All clusters have to run at once, and one of 4 CTAs lies within a group of SMs that the hardware wires together: 28
// always find room, 36 did not (1024 x 1024 took 210 us for 119).
constexpr double kSplitCost[2] = {2.0, 1.0};
int split_of(int64_t tiles, int kblocks, int planes) {
  const double stage = planes == 1 ? 0.2 : 0.65;
  int best = 1;
  double least = kblocks * stage;
  for (int ks = 2; ks <= 4; ks *= 2) {
    if (tiles * ks > (ks == 2 ? sm_count() * 7 / 8 : sm_count() * 3 / 4) || kblocks < ks) break;
    const double t = (kblocks + ks - 1) / ks * stage + kSplitCost[planes - 1];
    if (t < least) {
      least = t;
      best = ks;
    }
  }
  return best;
}

template <int CG, int TN, int NP, int OP_A, int OP_B, int MODE, typename TOUT = __half>
cudaError_t launch_gemm(Operand& a, Operand& b, const GemmArgs& g, cudaStream_t st) {
  if constexpr (CG == 1) {
    switch (split_of(g.total, (g.K + kTileK - 1) / kTileK, NP)) {
      case 4: return launch_gemm_as<CG, TN, NP, OP_A, OP_B, MODE, TOUT, 4>(a, b, g, st);
      case 2: return launch_gemm_as<CG, TN, NP, OP_A, OP_B, MODE, TOUT, 2>(a, b, g, st);
    }
  }
  return launch_gemm_as<CG, TN, NP, OP_A, OP_B, MODE, TOUT, 1>(a, b, g, st);
}

// Microseconds of one product in tiles of 128 x 128 (shape 0), 256 x 128 (1) or 256 x 256 (2), the last two by pairs of
// CTAs: waves of tiles times the stages of one, and what a launch takes beside them.  Fitted to 17 sizes from 200 x 200
// to 4096 x 4096; at 40 sizes, batches of up to 24 among them, a call's 15 products and the passes before them are off
// by at most a fifth.  Both sides, one plane: at 512 x 512 shape 0 takes 90 us and 2 takes 137, at 4096 x 4096 1.32 ms
// and 1.03; two planes: at 1500 x 1500 (bfloat16 result) shape 0 takes 324 us and 1 takes 293.
int64_t tiles_of(const OrthoPlan& q, bool symmetric, int shape) {
  const int tm = shape == 0 ? 128 : 256, tn = shape == 2 ? 256 : 128;
  const int64_t sym = (q.m + tm - 1) / tm, tr = (q.rows + tm - 1) / tm, tc = (q.cols + tn - 1) / tn;
  return (symmetric ? tm / tn * (sym * (sym + 1) / 2) : tr * tc) * q.batch;
}
double product_cost(const OrthoPlan& q, bool symmetric, int contraction, int shape) {
  static const double kStage[2][3] = {{0.272, 0.239, 0.345}, {0.709, 0.669, 1.15}};
  static const double kFixed[2][3] = {{3.35, 4.1, 5.8}, {5.4, 5.0, 8.7}};
  const int64_t slots = sm_count() / (shape == 0 ? 1 : 2), tiles = tiles_of(q, symmetric, shape);
  const int64_t kb = (contraction + kTileK - 1) / kTileK;
  const int ks = shape == 0 ? split_of(tiles, (int)kb, q.planes) : 1;
  const double stages = ks > 1 ? (double)((kb + ks - 1) / ks) : (double)((tiles + slots - 1) / slots * kb);
  return stages * kStage[q.planes - 1][shape] + (ks > 1 ? kSplitCost[q.planes - 1] : 0.0) + kFixed[q.planes - 1][shape];
}

// Which shapes a call's products take.  A symmetric result is stored by blocks of as many rows as the tiles have, so
// either all products take shape 0, or each the better one of the other two.  Two planes with accumulators of one stage
// (kLongChunkFrom) always take shape 0: pairs would have to empty twice the accumulators every 64 of the contraction, and
// at 34 sizes between 130 x 130 and 1590 x 4000 no shape of theirs was faster (12 x 768 x 768: 474 us against 554, 4 x 1300 x
// 1700: 870 against 1263).
struct Shapes {
  bool pairs, wide_gram, wide_poly, wide_step;
};
Shapes choose_shapes(const OrthoPlan& q) {
  if (q.planes == 2 && q.chunk == 1) return Shapes{};
  const int n = q.rows < q.cols ? q.cols : q.rows;
  const bool symmetric[3] = {true, true, false};
  const int contraction[3] = {n, q.m, q.m};
  double one = 0, two = 0;
  bool wide[3];
  for (int i = 0; i < 3; ++i) {
    const double narrow = product_cost(q, symmetric[i], contraction[i], 1), broad = product_cost(q, symmetric[i], contraction[i], 2);
    one += product_cost(q, symmetric[i], contraction[i], 0);
    wide[i] = broad < narrow;
    two += wide[i] ? broad : narrow;
  }
  return Shapes{two < one, wide[0], wide[1], wide[2]};
}

// Calls f with the tile's columns: 256 (pairs of CTAs only) or 128.
template <int CG, typename F>
cudaError_t with_columns(bool wide, F&& f) {
  if constexpr (CG == 2)
    if (wide) return f(std::integral_constant<int, 256>{});
  return f(std::integral_constant<int, 128>{});
}

template <int CG, int NP>
cudaError_t launch_products(const OrthoPlan& q, const Shapes& shapes, const brace_ortho_params* p, char* ws,
                            const GemmArgs& last, int out_type, cudaStream_t st) {
  constexpr int TM = 128 * CG;
  const bool tall = q.rows > q.cols;
  const int64_t z = (int64_t)q.batch * q.planes;
  Operand xs[2] = {}, s = {}, ts[2] = {}, poly = {};
  auto place = [&](Operand& x, size_t off, int64_t rows, int64_t ld) {
    x.base = ws + off;
    x.rows = rows;
    x.ld = ld;
    x.z = z;
    x.planes = q.planes;
  };
  place(xs[0], q.off_x[0], q.rows, q.ld_x);
  place(xs[1], q.off_x[1], q.rows, q.ld_x);
  place(s, q.off_s, q.m, q.ld_s);
  for (int k = 0; k < 2; ++k) place(ts[k], q.off_t[k], q.m, q.ld_s);
  place(poly, q.off_p, q.m, q.ld_s);
  const int tm = (q.m + TM - 1) / TM;
  GemmArgs sym = {};
  sym.M = sym.N = q.m;
  auto sym_tiles = [&](GemmArgs& g, int tn) {
    g.tiles = TM / tn * (tm * (tm + 1) / 2);
    g.total = g.tiles * q.batch;
  };
  sym.ld_dst = q.ld_s;
  sym.chunk = q.chunk;
  sym.status = (int*)ws;
  GemmArgs step = last;
  step.M = q.rows;
  step.N = q.cols;
  step.K = q.m;
  const int step_columns = CG == 2 && shapes.wide_step ? 256 : 128;
  step.tiles_n = (q.cols + step_columns - 1) / step_columns;
  step.tiles = step.tiles_n * ((q.rows + TM - 1) / TM);
  step.total = step.tiles * q.batch;
  step.ld_dst = q.ld_x;
  step.chunk = sym.chunk;
  step.scale = kStepScale;
  step.status = (int*)ws;
  for (int k = 0; k < p->steps; ++k) {
    const int cur = k & 1;
    Operand &x = xs[cur], &t = ts[q.off_t[0] == q.off_t[1] ? 0 : cur];
    GemmArgs g = sym;
    g.K = tall ? q.rows : q.cols;
    g.scale = kGramScale;
    g.dst = (__half*)(ws + q.off_s);
    g.dst2 = (__half*)(ws + q.off_t[cur]);
    g.scale2 = p->c * kFromGram;
    g.diagonal2 = p->b * kSquareScale;
    cudaError_t err = with_columns<CG>(shapes.wide_gram, [&](auto n) {
      constexpr int TN = decltype(n)::value;
      sym_tiles(g, TN);
      return tall ? launch_gemm<CG, TN, NP, kAcross, kAcross, kModeGram>(x, x, g, st)
                  : launch_gemm<CG, TN, NP, kAlong, kAlong, kModeGram>(x, x, g, st);
    });
    if (err != cudaSuccess) return err;
    g = sym;
    g.K = q.m;
    if (NP == 2) {
      g.scale = kPolyScale;
    } else {
      g.scale = p->c * kFromGram * kGramScale;   // S S * 2^28
      g.scale2 = p->b * kFromGram;
      g.src = (const __half*)(ws + q.off_s);
    }
    g.diagonal = p->a * kSquareScale;
    g.dst = (__half*)(ws + q.off_p);
    err = with_columns<CG>(shapes.wide_poly, [&](auto n) {
      constexpr int TN = decltype(n)::value;
      sym_tiles(g, TN);
      return launch_gemm<CG, TN, NP, kSymmetric, kSymmetric, kModePoly>(s, NP == 2 ? t : s, g, st);
    });
    if (err != cudaSuccess) return err;
    step.dst = (__half*)(ws + q.off_x[cur ^ 1]);
    err = with_columns<CG>(shapes.wide_step, [&](auto n) {
      constexpr int TN = decltype(n)::value;
      if (k + 1 < p->steps)
        return tall ? launch_gemm<CG, TN, NP, kAlong, kSymmetric, kModeStep>(x, poly, step, st)
                    : launch_gemm<CG, TN, NP, kSymmetric, kAcross, kModeStep>(poly, x, step, st);
      return with_type(out_type, [&](auto t) {
        using TOUT = decltype(t);
        return tall ? launch_gemm<CG, TN, NP, kAlong, kSymmetric, kModeLast, TOUT>(x, poly, step, st)
                    : launch_gemm<CG, TN, NP, kSymmetric, kAcross, kModeLast, TOUT>(poly, x, step, st);
      });
    });
    if (err != cudaSuccess) return err;
  }
  return cudaSuccess;
}

cudaError_t launch_prep(const OrthoPlan& q, const PrepArgs& a, cudaStream_t st) {
  int64_t nb = ((int64_t)q.rows * (q.ld_x >> 3) + 511) / 512;
  const int64_t per = (kPrepBlocks + q.batch - 1) / q.batch;
  if (nb > per) nb = per;
  if (nb < 1) nb = 1;
  const dim3 g1((unsigned)q.norm_blocks, (unsigned)q.batch), g2((unsigned)nb, (unsigned)q.batch);
  cudaError_t err;
  switch (a.g.type) {
    case kTypeF32:
      err = launch(ortho_norm_kernel<kTypeF32>, g1, 256, 0, 1, st, a);
      return err != cudaSuccess ? err : launch(ortho_scale_kernel<kTypeF32>, g2, 256, 0, 1, st, a);
    case kTypeBF16:
      err = launch(ortho_norm_kernel<kTypeBF16>, g1, 256, 0, 1, st, a);
      return err != cudaSuccess ? err : launch(ortho_scale_kernel<kTypeBF16>, g2, 256, 0, 1, st, a);
    case kTypeF16:
      err = launch(ortho_norm_kernel<kTypeF16>, g1, 256, 0, 1, st, a);
      return err != cudaSuccess ? err : launch(ortho_scale_kernel<kTypeF16>, g2, 256, 0, 1, st, a);
    default:
      err = launch(ortho_norm_kernel<kTypeBits>, g1, 256, 0, 1, st, a);
      return err != cudaSuccess ? err : launch(ortho_scale_kernel<kTypeBits>, g2, 256, 0, 1, st, a);
  }
}

// One launch for matrices that a cluster of CTAs can hold.  `placed` false: nothing was launched, the device has no place
// for a cluster of that many CTAs (only up to 8 are certain: a part of a GPU may have fewer SMs wired together), and the
// matrix has to go through the tiled products.
template <int NP, int TYPE>
cudaError_t launch_resident_as(const ResidentArgs& r, int ctas, cudaStream_t st, bool* placed) {
  auto* kernel = ortho_resident_kernel<NP, TYPE>;
  static std::atomic<uint64_t> granted{0};
  int dev = 0;
  cudaError_t err = cudaGetDevice(&dev);
  if (err != cudaSuccess) return err;
  const uint64_t bit = 1ull << (dev & 63);
  if (!(granted.load(std::memory_order_relaxed) & bit)) {
    err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kResidentSmem);
    if (err == cudaSuccess) err = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (err != cudaSuccess) return err;
    granted.fetch_or(bit, std::memory_order_relaxed);
  }
  int64_t smem = resident_smem(NP, r.slice, ctas);
  // CTAs of two clusters must not share an SM: each would hold tensor memory that the other's cluster waits for
  if (ctas > 1 && smem < 118 * 1024) smem = 118 * 1024;
  const dim3 grid((unsigned)(r.last.total * ctas));
  if (ctas > 8) {
    // one CTA an SM whatever the matrix's size: the answer for a number of CTAs holds for all its launches
    static std::atomic<uint32_t> known[64];   // by device: bit ctas - 9 for a place, bit ctas + 7 for none
    std::atomic<uint32_t>& answers = known[dev & 63];
    uint32_t bits = answers.load(std::memory_order_relaxed);
    const uint32_t yes = 1u << (ctas - 9), no = 1u << (ctas + 7);
    if (!(bits & (yes | no))) {
      const LaunchConfig one(dim3((unsigned)ctas), kResidentThreads, (size_t)smem, ctas, st);
      int clusters = 0;
      err = cudaOccupancyMaxActiveClusters(&clusters, kernel, &one.cfg);
      if (err != cudaSuccess) return err;
      bits = clusters > 0 ? yes : no;
      answers.fetch_or(bits, std::memory_order_relaxed);
    }
    if (bits & no) {
      *placed = false;
      return cudaSuccess;
    }
  }
  return launch(kernel, grid, kResidentThreads, (size_t)smem, ctas, st, r);
}

template <int NP>
cudaError_t launch_resident(const ResidentArgs& r, int ctas, cudaStream_t st, bool* placed) {
  switch (r.prep.g.type) {
    case kTypeF32: return launch_resident_as<NP, kTypeF32>(r, ctas, st, placed);
    case kTypeBF16: return launch_resident_as<NP, kTypeBF16>(r, ctas, st, placed);
    case kTypeF16: return launch_resident_as<NP, kTypeF16>(r, ctas, st, placed);
    default: return launch_resident_as<NP, kTypeBits>(r, ctas, st, placed);
  }
}

// Long side per CTA and CTAs per matrix of the one-launch kernel; 0 CTAs where the matrix does not fit.
int resident_ctas(const OrthoPlan& q, int* slice) {
  const int n = q.rows < q.cols ? q.cols : q.rows;
  if (q.m > 128) return 0;
  const int widest = q.planes == 1 ? 256 : 128;   // what fits in shared memory
  if (n <= 256) {   // one CTA: nothing to exchange
    *slice = (int)round_up(n, 64);
    return 1;
  }
  const int ctas = (n + widest - 1) / widest;
  if (ctas > 16) return 0;
  *slice = (int)round_up((n + ctas - 1) / ctas, 64);
  return (n + *slice - 1) / *slice;
}

// Everything after the argument checks.
int run_ortho(const OrthoPlan& q, const brace_ortho_params* p, PrepArgs prep, const GemmArgs& last, int out_type, char* ws,
              cudaStream_t st) {
  prep.rows = q.rows;
  prep.cols = q.cols;
  prep.units_row = (q.cols + 7) / 8;
  prep.norm_blocks = q.norm_blocks;
  prep.partial = (double*)(ws + q.off_partial);
  prep.eps = p->eps;
  prep.x = (__half*)(ws + q.off_x[0]);
  prep.ld_x = q.ld_x;
  prep.planes = q.planes;
  prep.status = (int*)ws;
  int slice = 0;
  const int ctas = resident_ctas(q, &slice);
  if (ctas > 0) {
    ResidentArgs r = {};
    r.prep = prep;
    r.last = last;
    r.last.M = q.rows;
    r.last.N = q.cols;
    r.last.total = q.batch;
    r.m = q.m;
    r.slice = slice;
    r.tall = q.rows > q.cols;
    r.steps = p->steps;
    r.out_type = out_type;
    r.a = p->a;
    r.b = p->b;
    r.c = p->c;
    bool placed = true;
    const cudaError_t e = q.planes == 1 ? launch_resident<1>(r, ctas, st, &placed) : launch_resident<2>(r, ctas, st, &placed);
    if (e != cudaSuccess) return cuda_fail_no_ctx(e);
    if (placed) return BRACE_OK;
  }
  cudaError_t err = launch_prep(q, prep, st);
  if (err == cudaSuccess) {
    const Shapes shapes = choose_shapes(q);
    if (q.planes == 1)
      err = shapes.pairs ? launch_products<2, 1>(q, shapes, p, ws, last, out_type, st) : launch_products<1, 1>(q, shapes, p, ws, last, out_type, st);
    else
      err = shapes.pairs ? launch_products<2, 2>(q, shapes, p, ws, last, out_type, st) : launch_products<1, 2>(q, shapes, p, ws, last, out_type, st);
  }
  return err == cudaSuccess ? BRACE_OK : cuda_fail_no_ctx(err);
}

bool grad_ok(const void* p, int type, int64_t ld, int64_t bit_offset, int cols) {
  if (!p || (!float_type(type) && type != BRACE_TYPE_BITS) || ld < cols) return false;
  if (!aligned(p, (size_t)elem_bytes(type))) return false;
  return type != BRACE_TYPE_BITS || bit_offset >= 0;
}

MatRef mat_ref(const void* p, int type, int64_t ld, int64_t stride, int64_t bit0) {
  MatRef r = {};
  r.p = p;
  r.ld = ld;
  r.batch = stride;
  r.type = type;
  r.vec = type != BRACE_TYPE_BITS && wide_rows(p, type, ld, stride);
  r.bit0 = type == BRACE_TYPE_BITS ? bit0 : 0;
  return r;
}

// ---- the embedding table ----------------------------------------------------------------------------------------

struct EmbPlan {
  int64_t parts;
  int64_t tile;    // tokens of a tile of the wide sort
  int tiles, passes;
  size_t off_key[2], off_pos[2], off_hist, off_span, off_part, bytes;
};

EmbPlan emb_plan(int32_t clients, int64_t tokens, int64_t vocab, int32_t dim) {
  EmbPlan q;
  size_t at = 0;
  auto take = [&at](int64_t bytes) {
    const size_t here = at;
    at += (size_t)round_up(bytes, 256);
    return here;
  };
  const int64_t n = (int64_t)clients * tokens;
  const bool wide = tokens > kDirectTokens;
  const int64_t per = ((tokens + kSortTile - 1) / kSortTile + kMostTiles - 1) / kMostTiles;
  q.tile = per * kSortTile;
  q.tiles = wide ? (int)((tokens + q.tile - 1) / q.tile) : 0;
  q.passes = 0;
  while ((vocab >> (q.passes * kWideBits)) != 0) ++q.passes;   // the largest value of these bits stands for "no token"
  for (int i = 0; i < 2; ++i) {
    q.off_key[i] = take(wide ? 4 * n : 0);
    q.off_pos[i] = take(wide ? 4 * n : 0);
  }
  // for the most tiles that so many tokens or fewer can have: a workspace serves fewer tokens too
  const int64_t most = wide ? std::min<int64_t>((tokens + kSortTile - 1) / kSortTile, kMostTiles) : 0;
  q.off_hist = take(q.passes * clients * most * kWideDigits * 4);
  q.off_span = take(wide ? 8 * (int64_t)clients * vocab : 0);
  q.parts = wide ? (tokens + kPart - 1) / kPart : 0;
  q.off_part = take((int64_t)clients * q.parts * 2 * dim * 4);
  q.bytes = at > 256 ? at : 256;
  return q;
}

bool emb_sizes_ok(int32_t clients, int64_t tokens, int64_t vocab, int32_t dim) {
  const int64_t most = (int64_t)1 << 31;
  return clients >= 0 && clients <= 65535 && tokens >= 0 && tokens < most && vocab >= 1 && vocab < most && dim >= 1;
}

constexpr int kMostColumns = 1 << 22;   // stretches of columns are a grid's third dimension: at most 32768 of them

int emb_check(const brace_embedding* e, bool grad) {
  if (!e || !emb_sizes_ok(e->clients, e->tokens, e->vocab, e->dim)) return BRACE_ERR_INVALID_ARG;
  if (e->dim > kMostColumns) return BRACE_ERR_UNSUPPORTED;
  if (!float_type(e->table_type) || !float_type(e->act_type)) return BRACE_ERR_INVALID_ARG;
  if ((e->id_bytes != 4 && e->id_bytes != 8) || !std::isfinite(e->scale)) return BRACE_ERR_INVALID_ARG;
  // what is only read may be broadcast: rows of the gradient's activations that are all the same one
  if (e->ld_table < e->dim || (e->ld_act < e->dim && !(grad && e->ld_act == 0))) return BRACE_ERR_INVALID_ARG;
  return BRACE_OK;
}
bool emb_table_ok(const brace_embedding* e) { return e->d_table && aligned(e->d_table, (size_t)elem_bytes(e->table_type)); }
bool emb_act_ok(const brace_embedding* e) {
  return e->d_act && e->d_ids && aligned(e->d_act, (size_t)elem_bytes(e->act_type)) && aligned(e->d_ids, (size_t)e->id_bytes);
}

// Elements per thread: 8 where rows of both tensors are whole 16-byte words, 2 where pairs are aligned, else 1
// (neighbouring threads then take neighbouring elements, so the accesses still coalesce).
int emb_width(const brace_embedding* e) {
  auto pairs = [](const void* p, int type, int64_t ld, int64_t stride) {
    return aligned(p, 2 * (size_t)elem_bytes(type)) && ld % 2 == 0 && stride % 2 == 0;
  };
  if (e->dim % 8 == 0 && wide_rows(e->d_table, e->table_type, e->ld_table, e->stride_table) &&
      wide_rows(e->d_act, e->act_type, e->ld_act, e->stride_act))
    return 8;
  if (e->dim % 2 == 0 && pairs(e->d_table, e->table_type, e->ld_table, e->stride_table) &&
      pairs(e->d_act, e->act_type, e->ld_act, e->stride_act))
    return 2;
  return 1;
}

EmbArgs emb_args(const brace_embedding* e) {
  EmbArgs a = {};
  a.ids = e->d_ids;
  a.ld_table = e->ld_table;
  a.stride_table = e->stride_table;
  a.stride_ids = e->stride_ids;
  a.ld_act = e->ld_act;
  a.stride_act = e->stride_act;
  a.tokens = e->tokens;
  a.vocab = e->vocab;
  a.clients = e->clients;
  a.dim = e->dim;
  a.id_bytes = e->id_bytes;
  a.scale = e->scale;
  a.accumulate = e->accumulate != 0;
  return a;
}

template <typename TI, typename TO, int V>
cudaError_t launch_lookup(const EmbArgs& a, cudaStream_t st) {
  constexpr int kWide = 32 * (V >= 8 ? V : 4);   // columns of a warp's stretch
  const int64_t x = (a.tokens + 8 * kLookupRows - 1) / (8 * kLookupRows), z = (a.dim + kWide - 1) / kWide;
  return launch(embedding_lookup_kernel<TI, TO, V>, dim3((unsigned)x, (unsigned)a.clients, (unsigned)z), 256, 0, 1, st, a);
}

// Sorts the tokens; leaves a.key and a.pos at the result.
cudaError_t launch_sort(EmbArgs& a, const EmbPlan& q, char* ws, cudaStream_t st) {
  const dim3 grid((unsigned)q.tiles, (unsigned)a.clients);
  uint32_t* hist = (uint32_t*)(ws + q.off_hist);
  cudaError_t err = launch(embedding_count_kernel, grid, kSortThreads, 0, 1, st, a, hist, q.tile, q.passes);
  for (int pass = 0; err == cudaSuccess && pass < q.passes; ++pass) {
    uint32_t *key = (uint32_t*)(ws + q.off_key[pass & 1]), *pos = (uint32_t*)(ws + q.off_pos[pass & 1]);
    err = pass == 0 ? launch(embedding_scatter_kernel<true>, grid, kSortThreads, 0, 1, st, a, hist, q.tile, pass, q.passes, key, pos)
                    : launch(embedding_scatter_kernel<false>, grid, kSortThreads, 0, 1, st, a, hist, q.tile, pass, q.passes, key, pos);
    a.key = key;
    a.pos = pos;
  }
  return err;
}

constexpr int64_t kGradElements = 32768;   // of a CTA's rows

template <typename TI, typename TO, int V>
cudaError_t launch_grad(EmbArgs a, cudaStream_t st) {
  if (a.tokens <= kDirectTokens) {
    const int64_t blocks = (a.dim + Share<V>::kWide - 1) / Share<V>::kWide;
    // The columns are shared out, unless the table is far larger than L2: a frequent token's row is then more than one
    // CTA's work (2000 tokens, 1000 x 777: 40 -> 21 us), but lines that two CTAs write in part cost DRAM accesses where
    // L2 does not hold them (8 x 50000 x 777: 211 -> 370 us).
    int64_t z = a.vocab * a.clients * a.dim > ((int64_t)32 << 20) ? 1 : a.dim / 256;
    z = z < 1 ? 1 : z > blocks ? blocks : z;
    int64_t rows = kGradElements * z / a.dim;
    const int64_t even = a.vocab * a.clients * z / (4 * sm_count());
    if (rows > even) rows = even;
    a.rows_cta = rows < 1 ? 1 : rows > 64 ? 64 : (int)rows;
    return launch(embedding_direct_kernel<TI, TO, V>,
                  dim3((unsigned)((a.vocab + a.rows_cta - 1) / a.rows_cta), (unsigned)a.clients, (unsigned)z), 256, 0, 1, st, a);
  }
  // long runs of zeros, but 4 CTAs for each SM while the table has the rows
  int64_t rows = kGradElements / a.dim;
  const int64_t even = a.vocab * a.clients / (4 * sm_count());
  if (rows > even) rows = even;
  a.rows_cta = rows < 1 ? 1 : rows > 64 ? 64 : (int)rows;
  const unsigned row_ctas = (unsigned)((a.vocab + a.rows_cta - 1) / a.rows_cta);
  const int64_t blocks = (a.dim + Share<V>::kWide - 1) / Share<V>::kWide, groups = a.parts * a.clients;
  // few groups: their columns are shared out until every SM has four CTAs
  int64_t z = 4 * sm_count() / groups;
  z = z < 1 ? 1 : z > blocks ? blocks : z;
  const cudaError_t err = launch(embedding_sum_kernel<TI, TO, V>, dim3((unsigned)a.parts, (unsigned)a.clients, (unsigned)z), 256, 0, 1, st, a);
  if (err != cudaSuccess) return err;
  a.zero_ctas = a.accumulate ? 0 : row_ctas;
  a.join_split = (unsigned)(blocks < 16 ? blocks : 16);
  const int64_t ctas = a.zero_ctas + (a.parts + 7) / 8 * a.join_split;
  return launch(embedding_grad_kernel<TO, V>, dim3((unsigned)ctas, (unsigned)a.clients), 256, 0, 1, st, a);
}

}  // namespace

extern "C" {

int brace_embedding_lookup(const brace_embedding* e, brace_stream_t stream) {
  const int rc = emb_check(e, false);
  if (rc != BRACE_OK) return rc;
  if (e->clients == 0 || e->tokens == 0) return BRACE_OK;
  if (!emb_table_ok(e) || !emb_act_ok(e) || (e->clients > 1 && e->stride_act == 0)) return BRACE_ERR_INVALID_ARG;
  EmbArgs a = emb_args(e);
  a.table = e->d_table;
  a.out = e->d_act;
  const cudaStream_t st = (cudaStream_t)stream;
  const int width = emb_width(e);
  const cudaError_t err = with_type(e->table_type, [&](auto ti) {
    return with_type(e->act_type, [&](auto to) {
      using TI = decltype(ti);
      using TO = decltype(to);
      return width == 8 ? launch_lookup<TI, TO, 8>(a, st) : width == 2 ? launch_lookup<TI, TO, 2>(a, st) : launch_lookup<TI, TO, 1>(a, st);
    });
  });
  return err == cudaSuccess ? BRACE_OK : cuda_fail_no_ctx(err);
}

size_t brace_embedding_workspace_bytes(int32_t clients, int64_t tokens, int64_t vocab, int32_t dim) {
  return emb_sizes_ok(clients, tokens, vocab, dim) ? emb_plan(clients, tokens, vocab, dim).bytes : 0;
}

int brace_embedding_grad(const brace_embedding* e, void* d_workspace, size_t workspace_bytes, brace_stream_t stream) {
  const int rc = emb_check(e, true);
  if (rc != BRACE_OK) return rc;
  if (e->clients == 0) return BRACE_OK;
  if (!emb_table_ok(e) || (e->tokens > 0 && !emb_act_ok(e)) || (e->clients > 1 && e->stride_table == 0))
    return BRACE_ERR_INVALID_ARG;
  const EmbPlan q = emb_plan(e->clients, e->tokens, e->vocab, e->dim);
  if (!d_workspace || workspace_bytes < q.bytes || !aligned(d_workspace, 256)) return BRACE_ERR_WORKSPACE;
  if (e->tokens == 0 && e->accumulate) return BRACE_OK;
  char* ws = (char*)d_workspace;
  EmbArgs a = emb_args(e);
  a.grad = e->d_table;
  a.in = e->d_act;
  a.key = (uint32_t*)(ws + q.off_key[0]);
  a.pos = (uint32_t*)(ws + q.off_pos[0]);
  a.span = (uint2*)(ws + q.off_span);
  a.part = (float*)(ws + q.off_part);
  a.parts = q.parts;
  const cudaStream_t st = (cudaStream_t)stream;
  cudaError_t err = cudaSuccess;
  if (a.tokens > kDirectTokens) err = launch_sort(a, q, ws, st);
  if (err == cudaSuccess) {
    const int width = emb_width(e);
    err = with_type(e->act_type, [&](auto ti) {
      return with_type(e->table_type, [&](auto to) {
        using TI = decltype(ti);
        using TO = decltype(to);
        return width == 8 ? launch_grad<TI, TO, 8>(a, st) : width == 2 ? launch_grad<TI, TO, 2>(a, st) : launch_grad<TI, TO, 1>(a, st);
      });
    });
  }
  return err == cudaSuccess ? BRACE_OK : cuda_fail_no_ctx(err);
}

int brace_ortho_default_params(brace_ortho_params* params) {
  if (!params) return BRACE_ERR_INVALID_ARG;
  *params = brace_ortho_params{5, 3.4445f, -4.7750f, 2.0315f, 1e-7f, BRACE_ORTHO_AUTO};
  return BRACE_OK;
}

size_t brace_ortho_workspace_bytes(int32_t batch, int32_t rows, int32_t cols, const brace_ortho_params* params,
                                   int32_t out_type) {
  if (!coefficients_ok(params) || !float_type(out_type) || !sizes_ok(batch, rows, cols)) return 0;
  if (!sizes_served(batch, rows, cols)) return 0;
  if (batch == 0 || rows == 0 || cols == 0) return 256;
  return make_plan(batch, rows, cols, params, out_type).bytes;
}

int brace_orthogonalize(int32_t batch, int32_t rows, int32_t cols, const brace_ortho_params* params, const void* d_g,
                        int32_t g_type, int64_t ld_g, int64_t stride_g, int64_t bit_offset, void* d_out,
                        int32_t out_type, int64_t ld_out, int64_t stride_out, void* d_workspace,
                        size_t workspace_bytes, brace_stream_t stream) {
  if (!coefficients_ok(params) || !float_type(out_type) || !sizes_ok(batch, rows, cols)) return BRACE_ERR_INVALID_ARG;
  if (batch == 0 || rows == 0 || cols == 0) return BRACE_OK;
  if (!grad_ok(d_g, g_type, ld_g, bit_offset, cols)) return BRACE_ERR_INVALID_ARG;
  if (!d_out || ld_out < cols || !aligned(d_out, (size_t)elem_bytes(out_type))) return BRACE_ERR_INVALID_ARG;
  if (batch > 1 && stride_out == 0) return BRACE_ERR_INVALID_ARG;   // what is written is a place of its own for each
  if (!sizes_served(batch, rows, cols)) return BRACE_ERR_UNSUPPORTED;
  const OrthoPlan q = make_plan(batch, rows, cols, params, out_type);
  if (!d_workspace || workspace_bytes < q.bytes || !aligned(d_workspace, 256)) return BRACE_ERR_WORKSPACE;
  PrepArgs prep = {};
  prep.g = mat_ref(d_g, g_type, ld_g, stride_g, bit_offset);
  GemmArgs last = {};
  last.out = d_out;
  last.ld_out = ld_out;
  last.batch_out = stride_out;
  last.vec_out = wide_rows(d_out, out_type, ld_out, stride_out);
  last.vec_in = 1;   // there is none
  last.replicas = 1;
  return run_ortho(q, params, prep, last, out_type, (char*)d_workspace, (cudaStream_t)stream);
}

int brace_muon_step(int32_t batch, int32_t rows, int32_t cols, const brace_ortho_params* params,
                    const brace_muon* s, void* d_workspace, size_t workspace_bytes, brace_stream_t stream) {
  if (!s || !coefficients_ok(params) || !float_type(s->weights_type) || !sizes_ok(batch, rows, cols))
    return BRACE_ERR_INVALID_ARG;
  if (!std::isfinite(s->beta) || !std::isfinite(s->lr) || !std::isfinite(s->weight_decay) || !std::isfinite(s->scale))
    return BRACE_ERR_INVALID_ARG;
  if (s->replicas < 1) return BRACE_ERR_INVALID_ARG;
  if (batch == 0 || rows == 0 || cols == 0) return BRACE_OK;
  if (!grad_ok(s->d_grad, s->grad_type, s->ld_grad, s->bit_offset, cols)) return BRACE_ERR_INVALID_ARG;
  if (!s->d_momentum || !s->d_momentum_out || s->ld_momentum < cols || s->ld_momentum_out < cols ||
      !aligned(s->d_momentum, 4) || !aligned(s->d_momentum_out, 4))
    return BRACE_ERR_INVALID_ARG;
  const size_t wb = (size_t)elem_bytes(s->weights_type);
  if (!s->d_weights || !s->d_weights_out || s->ld_weights < cols || s->ld_weights_out < cols ||
      !aligned(s->d_weights, wb) || !aligned(s->d_weights_out, wb))
    return BRACE_ERR_INVALID_ARG;
  if (batch > 1 && (s->stride_momentum_out == 0 || s->stride_weights_out == 0)) return BRACE_ERR_INVALID_ARG;
  if (s->replicas > 1 && s->replica_weights_out == 0) return BRACE_ERR_INVALID_ARG;
  if (!sizes_served(batch, rows, cols)) return BRACE_ERR_UNSUPPORTED;
  const OrthoPlan q = make_plan(batch, rows, cols, params, s->weights_type);
  if (!d_workspace || workspace_bytes < q.bytes || !aligned(d_workspace, 256)) return BRACE_ERR_WORKSPACE;
  PrepArgs prep = {};
  prep.g = mat_ref(s->d_grad, s->grad_type, s->ld_grad, s->stride_grad, s->bit_offset);
  prep.m_in = s->d_momentum;
  prep.ld_m_in = s->ld_momentum;
  prep.batch_m_in = s->stride_momentum;
  prep.vec_m_in = wide_rows(s->d_momentum, BRACE_TYPE_F32, s->ld_momentum, s->stride_momentum);
  prep.m_out = s->d_momentum_out;
  prep.ld_m_out = s->ld_momentum_out;
  prep.batch_m_out = s->stride_momentum_out;
  prep.vec_m_out = wide_rows(s->d_momentum_out, BRACE_TYPE_F32, s->ld_momentum_out, s->stride_momentum_out);
  prep.beta = s->beta;
  prep.nesterov = s->nesterov != 0;
  GemmArgs last = {};
  last.out = s->d_weights_out;
  last.ld_out = s->ld_weights_out;
  last.batch_out = s->stride_weights_out;
  last.rep_out = s->replica_weights_out;
  last.vec_out = wide_rows(s->d_weights_out, s->weights_type, s->ld_weights_out, s->stride_weights_out, s->replica_weights_out);
  last.w_in = s->d_weights;
  last.ld_in = s->ld_weights;
  last.batch_in = s->stride_weights;
  last.rep_in = s->replica_weights;
  last.vec_in = wide_rows(s->d_weights, s->weights_type, s->ld_weights, s->stride_weights, s->replica_weights);
  last.replicas = s->replicas;
  last.keep = 1.f - s->lr * s->weight_decay;
  last.rate = s->lr * s->scale;
  return run_ortho(q, params, prep, last, s->weights_type, (char*)d_workspace, (cudaStream_t)stream);
}

int brace_ortho_status(const void* d_workspace, brace_stream_t stream) {
  if (!d_workspace) return BRACE_ERR_WORKSPACE;
  int code = 0;
  cudaError_t err = cudaMemcpyAsync(&code, d_workspace, sizeof(code), cudaMemcpyDeviceToHost, (cudaStream_t)stream);
  if (err == cudaSuccess) err = cudaStreamSynchronize((cudaStream_t)stream);
  if (err != cudaSuccess) return cuda_fail_no_ctx(err);
  return code ? BRACE_ERR_TIMEOUT : BRACE_OK;
}

}  // extern "C"
