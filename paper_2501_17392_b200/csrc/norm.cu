// Host side of the layer norm: argument checks, workspace, launches.
// C ABI declared in brace.h.
#include "brace.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "host.cuh"
#include "norm_kernels.cuh"

using namespace brace;

namespace {

// ---- layer norm -------------------------------------------------------------------------------------------------

constexpr int64_t kMost = (int64_t)1 << 31;
constexpr int kNormMostColumns = 1 << 22;

int pow2_ceil(int64_t x) {
  int p = 1;
  while (p < x) p <<= 1;
  return p;
}

// How a row is held: `group` threads with `nv` pieces of `v` columns each.  Groups as wide as a warp where the row gives
// each thread a piece: fewer rows at a time would leave fewer loads under way, more threads would hold nothing.
struct NormShape {
  int v, nv, group, block, slots;
};
NormShape norm_shape(int dim, int v, int most) {
  NormShape s;
  s.v = v;
  const int n = (dim + v - 1) / v;
  s.group = std::max(std::min(32, pow2_ceil(n)), pow2_ceil((n + most - 1) / most));
  s.nv = (n + s.group - 1) / s.group;
  s.block = s.group > 32 ? s.group : kNormThreads;
  s.slots = s.block / s.group;
  return s;
}
// Through a ring: pieces of 16 bytes of x, so that a warp's reads of shared memory do not meet in a bank; 8 columns without,
// or one where rows are not aligned.
constexpr int kRingFrom = 256;   // columns: shorter rows are not worth a copy of their own
NormShape norm_shape(int dim, int x_type, bool wide) {
  if (!wide) return norm_shape(dim, 1, 32);
  if (dim < kRingFrom) return norm_shape(dim, 8, 4);
  return x_type == BRACE_TYPE_F32 ? norm_shape(dim, 4, 8) : norm_shape(dim, 8, 4);
}
// Of the gradient: a thread has twice as much to keep for each column.  Of rows that take several warps it is given half as many,
// so that more threads are there (4 x 8192 rows of 2048 in bfloat16: 177 -> 114 us; rows of 768 would leave a warp for two, and
// take 264 us for 147).
NormShape norm_grad_shape(int dim, int x_type, bool wide) {
  if (!wide || dim <= 1024 || dim > 4096) return norm_shape(dim, x_type, wide);
  return x_type == BRACE_TYPE_F32 ? norm_shape(dim, 4, 4) : norm_shape(dim, 8, 2);
}

constexpr int kSms = 148;

// CTAs of an SM; narrow ones make room for more.
int resident_of(const NormShape& s, bool ring) {
  return (ring ? ring_resident(s.v * s.nv) : norm_resident(s.v * s.nv)) * (kNormThreads / s.block);
}

// CTAs of a client's gradient.  More rows never give fewer.
int64_t norm_parts(int32_t clients, int64_t rows, int32_t dim, int slots, int resident) {
  int64_t n = dim > kNormShort ? (rows + 31) / 32 : (rows + 4 * slots - 1) / (4 * slots);
  int64_t most = dim > kNormShort ? std::max<int64_t>((int64_t)kSms * 16 * kNormThreads / dim, 1) : kSms * resident;
  most /= std::max(clients, 1);
  n = std::min(n, std::max<int64_t>(most, 1));
  return std::max<int64_t>(n, 1);
}

bool norm_sizes_ok(int32_t clients, int64_t rows, int32_t dim) {
  return clients >= 0 && clients <= 65535 && rows >= 0 && rows < kMost && dim >= 1;
}

// What the forward pass and the gradient have in common.
int norm_check(const brace_layer_norm* e, bool grad) {
  if (!e || !norm_sizes_ok(e->clients, e->rows, e->dim)) return BRACE_ERR_INVALID_ARG;
  if (e->dim > kNormMostColumns) return BRACE_ERR_UNSUPPORTED;
  if (!float_type(e->x_type) || !float_type(e->y_type) || !float_type(e->weight_type)) return BRACE_ERR_INVALID_ARG;
  // what is only read may be broadcast
  if (e->ld_x < e->dim && e->ld_x != 0) return BRACE_ERR_INVALID_ARG;
  if (e->ld_y < e->dim && !(grad && e->ld_y == 0)) return BRACE_ERR_INVALID_ARG;
  if (grad ? !float_type(e->grad_type) || e->ld_dx < e->dim : !std::isfinite(e->eps) || !(e->eps >= 0.f))
    return BRACE_ERR_INVALID_ARG;
  return BRACE_OK;
}

NormArgs norm_args(const brace_layer_norm* e) {
  NormArgs a = {};
  a.x = e->d_x;
  a.weight = e->d_weight;
  a.bias = e->d_bias;
  a.y = e->d_y;
  a.mean = e->d_mean;
  a.rstd = e->d_rstd;
  a.ld_x = e->ld_x;
  a.stride_x = e->stride_x;
  a.stride_weight = e->stride_weight;
  a.stride_bias = e->stride_bias;
  a.ld_y = e->ld_y;
  a.stride_y = e->stride_y;
  a.stride_stats = e->stride_stats;
  a.rows = e->rows;
  a.dim = e->dim;
  a.weight_type = e->weight_type;
  a.eps = e->eps;
  return a;
}

// Calls f with the pieces a thread holds without a ring: one of 8 columns, scalars in three sizes.
template <typename F>
cudaError_t with_pieces(const NormShape& s, F&& f) {
  using std::integral_constant;
  if (s.v == 8) return f(integral_constant<int, 8>{}, integral_constant<int, 1>{});
  constexpr integral_constant<int, 1> v;
  if (s.nv <= 4) return f(v, integral_constant<int, 4>{});
  if (s.nv <= 12) return f(v, integral_constant<int, 12>{});
  return f(v, integral_constant<int, 32>{});
}
// And with one.
template <typename TX, typename F>
cudaError_t with_ring(const NormShape& s, F&& f) {
  using std::integral_constant;
  constexpr int V = 16 / (int)sizeof(TX), K = 8 / V;      // K pieces hold 8 columns
  constexpr integral_constant<int, V> v;
  const int n = (s.nv + K - 1) / K;
  if (n <= 1) return f(v, integral_constant<int, K>{});
  if (n <= 2) return f(v, integral_constant<int, 2 * K>{});
  if (n <= 3) return f(v, integral_constant<int, 3 * K>{});
  return f(v, integral_constant<int, 4 * K>{});
}
template <typename K>
cudaError_t launch_ring(K* kernel, std::atomic<uint64_t>& granted, const NormShape& s, dim3 grid, int row_bytes, NormArgs a, cudaStream_t st) {
  const cudaError_t err = grant_smem((const void*)kernel, granted, ring_bytes(32) + 1024);
  if (err != cudaSuccess) return err;
  a.row_bytes = row_bytes;
  a.stages = std::max(1, std::min(kRingMost, ring_bytes(s.v * s.nv) / (kNormThreads / s.block) / (s.slots * row_bytes)));
  return launch(kernel, grid, s.block, 1024 + s.slots * a.stages * row_bytes, 1, st, a);
}

}  // namespace

extern "C" {

int brace_layer_norm_forward(const brace_layer_norm* e, brace_stream_t stream) {
  const int rc = norm_check(e, false);
  if (rc != BRACE_OK) return rc;
  if (e->clients == 0 || e->rows == 0) return BRACE_OK;
  if (!typed(e->d_x, e->x_type) || !typed(e->d_y, e->y_type) || !typed_or_null(e->d_weight, e->weight_type) ||
      !typed_or_null(e->d_bias, e->weight_type) || !aligned(e->d_mean, 4) || !aligned(e->d_rstd, 4))
    return BRACE_ERR_INVALID_ARG;
  if (e->clients > 1 && (e->stride_y == 0 || ((e->d_mean || e->d_rstd) && e->stride_stats < e->rows)))
    return BRACE_ERR_INVALID_ARG;
  NormArgs a = norm_args(e);
  const cudaStream_t st = (cudaStream_t)stream;
  const bool wide = e->dim % 8 == 0 && wide_rows(e->d_x, e->x_type, e->ld_x, e->stride_x) &&
                    wide_rows(e->d_y, e->y_type, e->ld_y, e->stride_y);
  const NormShape s = norm_shape(e->dim, e->x_type, wide);
  const bool ring = wide && e->dim >= kRingFrom;
  const int resident = e->dim > kNormShort ? 4 : resident_of(s, ring);
  a.group = s.group;
  const int64_t slots = e->dim > kNormShort ? 1 : s.slots;
  const int64_t ctas = std::min((e->rows + slots - 1) / slots, std::max<int64_t>(1, kSms * resident / e->clients));
  const dim3 grid((unsigned)ctas, (unsigned)e->clients);
  const cudaError_t err = with_type(e->x_type, [&](auto tx) {
    return with_type(e->y_type, [&](auto ty) {
      using TX = decltype(tx);
      using TY = decltype(ty);
      if (e->dim > kNormShort)
        return wide ? launch(norm_forward_long_kernel<TX, TY, 8>, grid, kNormThreads, 0, 1, st, a)
                    : launch(norm_forward_long_kernel<TX, TY, 1>, grid, kNormThreads, 0, 1, st, a);
      if (ring)
        return with_ring<TX>(s, [&](auto v, auto nv) {
          static std::atomic<uint64_t> granted{0};
          return launch_ring(norm_forward_ring_kernel<TX, TY, decltype(v)::value, decltype(nv)::value>, granted, s, grid,
                             e->dim * (int)sizeof(TX), a, st);
        });
      return with_pieces(s, [&](auto v, auto nv) {
        return launch(norm_forward_kernel<TX, TY, decltype(v)::value, decltype(nv)::value>, grid, s.block, 0, 1, st, a);
      });
    });
  });
  return err == cudaSuccess ? BRACE_OK : cuda_fail_no_ctx(err);
}

size_t brace_layer_norm_workspace_bytes(int32_t clients, int64_t rows, int32_t dim) {
  if (!norm_sizes_ok(clients, rows, dim) || dim > kNormMostColumns) return 0;
  int64_t parts = 1;
  for (const bool wide : {false, true})      // of any types and alignment
    for (const int type : {BRACE_TYPE_F32, BRACE_TYPE_BF16}) {
      if (wide && dim % 8) continue;
      const NormShape s = norm_grad_shape(dim, type, wide);
      parts = std::max(parts, norm_parts(clients, rows, dim, s.slots, resident_of(s, wide && dim >= kRingFrom)));
    }
  return (size_t)round_up(std::max<int64_t>(parts * clients * 2 * dim * 4, 256), 256);
}

int brace_layer_norm_grad(const brace_layer_norm* e, void* d_workspace, size_t workspace_bytes, brace_stream_t stream) {
  const int rc = norm_check(e, true);
  if (rc != BRACE_OK) return rc;
  if (e->clients == 0) return BRACE_OK;
  const bool params = e->d_dweight || e->d_dbias;
  if (e->rows > 0 && (!typed(e->d_x, e->x_type) || !typed(e->d_y, e->y_type) || !typed(e->d_dx, e->x_type) ||
                      !typed(e->d_mean, BRACE_TYPE_F32) || !typed(e->d_rstd, BRACE_TYPE_F32) ||
                      !typed_or_null(e->d_weight, e->weight_type)))
    return BRACE_ERR_INVALID_ARG;
  if (!typed_or_null(e->d_dweight, e->grad_type) || !typed_or_null(e->d_dbias, e->grad_type)) return BRACE_ERR_INVALID_ARG;
  if (e->clients > 1 && (e->stride_dx == 0 || (e->d_dweight && e->stride_dweight == 0) || (e->d_dbias && e->stride_dbias == 0)))
    return BRACE_ERR_INVALID_ARG;
  const size_t need = brace_layer_norm_workspace_bytes(e->clients, e->rows, e->dim);
  if (!d_workspace || workspace_bytes < need || !aligned(d_workspace, 256)) return BRACE_ERR_WORKSPACE;
  if (e->rows == 0 && (e->accumulate || !params)) return BRACE_OK;
  NormArgs a = norm_args(e);
  a.dx = e->d_dx;
  a.dweight = e->d_dweight;
  a.dbias = e->d_dbias;
  a.ld_dx = e->ld_dx;
  a.stride_dx = e->stride_dx;
  a.stride_dweight = e->stride_dweight;
  a.stride_dbias = e->stride_dbias;
  a.grad_type = e->grad_type;
  a.accumulate = e->accumulate != 0;
  a.part = (float*)d_workspace;
  const cudaStream_t st = (cudaStream_t)stream;
  const bool wide = e->dim % 8 == 0 && wide_rows(e->d_x, e->x_type, e->ld_x, e->stride_x) &&
                    wide_rows(e->d_y, e->y_type, e->ld_y, e->stride_y) && wide_rows(e->d_dx, e->x_type, e->ld_dx, e->stride_dx);
  const NormShape s = norm_grad_shape(e->dim, e->x_type, wide);
  const bool ring = wide && e->dim >= kRingFrom;
  const bool is_long = e->dim > kNormShort;
  a.group = s.group;
  a.parts = (int)norm_parts(e->clients, e->rows, e->dim, s.slots, resident_of(s, ring));
  cudaError_t err = with_type(e->x_type, [&](auto tx) {
    return with_type(e->y_type, [&](auto ty) {
      using TX = decltype(tx);
      using TY = decltype(ty);
      if (!is_long && ring)
        return with_ring<TX>(s, [&](auto v, auto nv) {
          static std::atomic<uint64_t> granted{0};
          return launch_ring(norm_grad_ring_kernel<TX, TY, decltype(v)::value, decltype(nv)::value>, granted, s,
                             dim3((unsigned)a.parts, (unsigned)e->clients), e->dim * (int)(sizeof(TX) + sizeof(TY)), a, st);
        });
      if (!is_long)
        return with_pieces(s, [&](auto v, auto nv) {
          return launch(norm_grad_kernel<TX, TY, decltype(v)::value, decltype(nv)::value>,
                        dim3((unsigned)a.parts, (unsigned)e->clients), s.block, 0, 1, st, a);
        });
      const int64_t ctas = std::min(std::max<int64_t>(e->rows, 1), std::max<int64_t>(1, kSms * 4 / e->clients));
      const dim3 rows((unsigned)ctas, (unsigned)e->clients);
      const cudaError_t first = wide ? launch(norm_grad_long_kernel<TX, TY, 8>, rows, kNormThreads, 0, 1, st, a)
                                     : launch(norm_grad_long_kernel<TX, TY, 1>, rows, kNormThreads, 0, 1, st, a);
      if (first != cudaSuccess || !params) return first;
      const int per = kNormThreads * (wide ? 8 : 1);
      const dim3 columns((unsigned)((e->dim + per - 1) / per), (unsigned)a.parts, (unsigned)e->clients);
      return wide ? launch(norm_columns_kernel<TX, TY, 8>, columns, kNormThreads, 0, 1, st, a)
                  : launch(norm_columns_kernel<TX, TY, 1>, columns, kNormThreads, 0, 1, st, a);
    });
  });
  if (err == cudaSuccess && params && (is_long || a.parts > 1))
    err = launch(norm_join_kernel, dim3((unsigned)((2 * (int64_t)e->dim + 31) / 32), (unsigned)e->clients), 256, 0, 1, st, a);
  return err == cudaSuccess ? BRACE_OK : cuda_fail_no_ctx(err);
}

}  // extern "C"
