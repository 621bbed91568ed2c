// Host side of the layer norm and of the gradients' norm and clipping: argument checks, workspaces, launches.
// C ABI declared in brace.h.
#include "brace.h"

#include <algorithm>
#include <cmath>
#include <cstring>
#include <type_traits>

#include "clip_kernels.cuh"
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
NormShape norm_shape(int dim, bool wide) {
  NormShape s;
  s.v = wide ? 8 : 1;
  const int n = (dim + s.v - 1) / s.v, most = wide ? 4 : 32;
  s.group = std::max(std::min(32, pow2_ceil(n)), pow2_ceil((n + most - 1) / most));
  s.nv = (n + s.group - 1) / s.group;
  s.block = s.group > 32 ? s.group : kNormThreads;
  s.slots = s.block / s.group;
  return s;
}

constexpr int kNormForwardCtas = 148 * 4, kNormGradCtas = 148 * 3;

// CTAs of a client's gradient.  More rows never give fewer.
int64_t norm_parts(int32_t clients, int64_t rows, int32_t dim, int slots) {
  int64_t n = dim > kNormShort ? (rows + 31) / 32 : (rows + 4 * slots - 1) / (4 * slots);
  int64_t most = dim > kNormShort ? (int64_t)kNormGradCtas * kNormThreads / dim : kNormGradCtas;
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

bool typed(const void* p, int type) { return p && aligned(p, (size_t)elem_bytes(type)); }
bool typed_or_null(const void* p, int type) { return !p || aligned(p, (size_t)elem_bytes(type)); }

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

// Calls f with the pieces a thread holds; scalars in three sizes.
template <typename F>
cudaError_t with_pieces(const NormShape& s, F&& f) {
  using std::integral_constant;
  if (s.v == 8) {
    constexpr integral_constant<int, 8> v;
    if (s.nv <= 1) return f(v, integral_constant<int, 1>{});
    if (s.nv <= 2) return f(v, integral_constant<int, 2>{});
    if (s.nv <= 3) return f(v, integral_constant<int, 3>{});
    return f(v, integral_constant<int, 4>{});
  }
  constexpr integral_constant<int, 1> v;
  if (s.nv <= 4) return f(v, integral_constant<int, 4>{});
  if (s.nv <= 12) return f(v, integral_constant<int, 12>{});
  return f(v, integral_constant<int, 32>{});
}

// ---- clipping ---------------------------------------------------------------------------------------------------

constexpr int kClipCtas = 148 * 8;                        // of a launch's share in summing, or in clipping
constexpr int64_t kClipGroupBytes = (int64_t)32 << 20;    // of the clients that a launch sums and the next one clips
constexpr int kClipSmall = 8, kClipList = 40, kClipLongList = 340;   // tensors of a launch: its arguments hold them

// One run of elements on both sides (the gradients' alone where nothing is written).
bool clip_flat(const brace_tensor& t, bool clip) {
  return t.rows <= 1 || (t.ld_in == t.cols && (!clip || t.ld_out == t.cols));
}

// Units of a tensor, and of each of its rows (0: rows are walked together).
int64_t clip_units_of(const brace_tensor& t, bool clip, int64_t* row_units) {
  const bool flat = clip_flat(t, clip);
  const int64_t rows = flat ? 1 : t.rows, cols = flat ? t.rows * t.cols : t.cols;
  *row_units = flat || cols >= kClipNarrow ? (cols + kClipUnit - 1) / kClipUnit : 0;
  return *row_units ? rows * *row_units : (rows * cols + kClipUnit - 1) / kClipUnit;
}

struct ClipPlan {
  int group;        // clients that a launch sums
  int cap, lists;   // tensors of a launch, launches for a group
  int64_t ctas;     // most CTAs of a client and launch
};
ClipPlan clip_plan(int32_t clients, const brace_tensor* t, int32_t count, bool clip) {
  ClipPlan q;
  int64_t bytes = 0;
  for (int i = 0; i < count; ++i) bytes += t[i].rows * t[i].cols * elem_bytes(t[i].in_type);
  const int64_t fit = clip ? kClipGroupBytes / std::max<int64_t>(bytes, 1) : clients;
  q.group = (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(fit, clients), 32767));
  q.cap = count <= kClipSmall ? kClipSmall : count <= kClipList ? kClipList : kClipLongList;
  q.lists = std::max((count + q.cap - 1) / q.cap, 1);
  q.ctas = std::max(kClipCtas / q.group, 1);
  return q;
}

int clip_check(int32_t clients, const brace_tensor* t, int32_t count, bool clip) {
  if (clients < 0 || count < 0 || (count > 0 && !t)) return BRACE_ERR_INVALID_ARG;
  constexpr int64_t most = (int64_t)1 << 46;
  int64_t total = 0;
  for (int i = 0; i < count; ++i) {
    const brace_tensor& x = t[i];
    if (x.rows < 0 || x.cols < 0 || !float_type(x.in_type) || (clip && !float_type(x.out_type))) return BRACE_ERR_INVALID_ARG;
    if (x.rows == 0 || x.cols == 0) continue;
    if (x.cols > most / x.rows || (total += x.rows * x.cols) > most) return BRACE_ERR_UNSUPPORTED;
    if (clients == 0) continue;
    if (!typed(x.d_in, x.in_type) || (x.rows > 1 && x.ld_in < x.cols)) return BRACE_ERR_INVALID_ARG;
    if (!clip) continue;
    if (!typed(x.d_out, x.out_type) || (x.rows > 1 && x.ld_out < x.cols)) return BRACE_ERR_INVALID_ARG;
    if (clients > 1 && x.stride_out == 0) return BRACE_ERR_INVALID_ARG;
    // in place: every element where it was
    if (x.d_in == x.d_out && (x.in_type != x.out_type || (x.rows > 1 && x.ld_in != x.ld_out) ||
                              (clients > 1 && x.stride_in != x.stride_out)))
      return BRACE_ERR_INVALID_ARG;
  }
  return BRACE_OK;
}

template <int CAP>
cudaError_t launch_clip_as(const ClipArgs& a, int sum_count, const ClipTensor* tensors, int64_t ctas, cudaStream_t st) {
  ClipList<CAP> list;
  std::memcpy(list.t, tensors, sizeof(ClipTensor) * a.count);
  return launch(clip_kernel<CAP>, dim3((unsigned)ctas, (unsigned)(a.clip_count + sum_count)), kClipThreads, 0, 1, st, a, list);
}

int run_clip(int32_t clients, const brace_tensor* t, int32_t count, bool clip, ClipArgs a, double* ws, cudaStream_t st) {
  const ClipPlan q = clip_plan(clients, t, count, clip);
  ClipTensor tensors[kClipLongList];
  // what list l holds: fills `tensors`, says how many units and CTAs of a client that makes
  auto take = [&](int l, int64_t* units) {
    const int first = l * q.cap, n = std::min(count - first, q.cap);
    *units = 0;
    for (int i = 0; i < n; ++i) {
      const brace_tensor& x = t[first + i];
      ClipTensor& y = tensors[i];
      const bool flat = clip_flat(x, clip);
      y.in = x.d_in;
      y.out = x.d_out;
      y.rows = flat ? 1 : x.rows;
      y.cols = flat ? x.rows * x.cols : x.cols;
      y.ld_in = x.ld_in;
      y.ld_out = x.ld_out;
      y.stride_in = x.stride_in;
      y.stride_out = x.stride_out;
      y.in_type = x.in_type;
      y.out_type = x.out_type;
      y.unit0 = *units;
      *units += clip_units_of(x, clip, &y.row_units);
    }
    a.count = n;
    return std::max<int64_t>(1, std::min(*units, q.ctas));
  };
  a.part = ws;
  a.parts = 0;
  for (int l = 0; l < q.lists; ++l) a.parts += take(l, &a.units);
  const int stages = (clients + q.group - 1) / q.group;
  for (int s = 0; s <= stages; ++s) {   // stage s sums group s and clips the group before it
    if (!clip && s == stages) break;
    a.sum_first = s * q.group;
    const int sum_count = std::max(0, std::min(q.group, clients - a.sum_first));
    a.clip_first = a.sum_first - q.group;
    a.clip_count = clip && s > 0 ? std::min(q.group, clients - a.clip_first) : 0;
    a.part0 = 0;
    for (int l = 0; l < q.lists; ++l) {
      const int64_t ctas = take(l, &a.units);
      const cudaError_t err = q.cap == kClipSmall  ? launch_clip_as<kClipSmall>(a, sum_count, tensors, ctas, st)
                              : q.cap == kClipList ? launch_clip_as<kClipList>(a, sum_count, tensors, ctas, st)
                                                   : launch_clip_as<kClipLongList>(a, sum_count, tensors, ctas, st);
      if (err != cudaSuccess) return cuda_fail_no_ctx(err);
      a.part0 += ctas;
    }
  }
  if (!clip) {
    const cudaError_t err = launch(clip_norms_kernel, dim3((unsigned)clients), kClipThreads, 0, 1, st, a);
    if (err != cudaSuccess) return cuda_fail_no_ctx(err);
  }
  return BRACE_OK;
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
  const NormShape s = norm_shape(e->dim, wide);
  a.group = s.group;
  const int64_t slots = e->dim > kNormShort ? 1 : s.slots;
  const int64_t ctas = std::min((e->rows + slots - 1) / slots, std::max<int64_t>(1, kNormForwardCtas / e->clients));
  const dim3 grid((unsigned)ctas, (unsigned)e->clients);
  const cudaError_t err = with_type(e->x_type, [&](auto tx) {
    return with_type(e->y_type, [&](auto ty) {
      using TX = decltype(tx);
      using TY = decltype(ty);
      if (e->dim > kNormShort) return launch(norm_forward_long_kernel<TX, TY>, grid, kNormThreads, 0, 1, st, a);
      return with_pieces(s, [&](auto v, auto nv) {
        return launch(norm_forward_kernel<TX, TY, decltype(v)::value, decltype(nv)::value>, grid, s.block, 0, 1, st, a);
      });
    });
  });
  return err == cudaSuccess ? BRACE_OK : cuda_fail_no_ctx(err);
}

size_t brace_layer_norm_workspace_bytes(int32_t clients, int64_t rows, int32_t dim) {
  if (!norm_sizes_ok(clients, rows, dim) || dim > kNormMostColumns) return 0;
  const int slots = std::min(norm_shape(dim, false).slots, norm_shape((dim + 7) / 8 * 8, true).slots);
  return (size_t)round_up(std::max<int64_t>(norm_parts(clients, rows, dim, slots) * clients * 2 * dim * 4, 256), 256);
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
  const NormShape s = norm_shape(e->dim, wide);
  const bool is_long = e->dim > kNormShort;
  a.group = s.group;
  a.parts = (int)norm_parts(e->clients, e->rows, e->dim, s.slots);
  cudaError_t err = with_type(e->x_type, [&](auto tx) {
    return with_type(e->y_type, [&](auto ty) {
      using TX = decltype(tx);
      using TY = decltype(ty);
      if (!is_long)
        return with_pieces(s, [&](auto v, auto nv) {
          return launch(norm_grad_kernel<TX, TY, decltype(v)::value, decltype(nv)::value>,
                        dim3((unsigned)a.parts, (unsigned)e->clients), s.block, 0, 1, st, a);
        });
      const int64_t ctas = std::min(std::max<int64_t>(e->rows, 1), std::max<int64_t>(1, kNormForwardCtas / e->clients));
      const cudaError_t first = launch(norm_grad_long_kernel<TX, TY>, dim3((unsigned)ctas, (unsigned)e->clients), kNormThreads, 0, 1, st, a);
      if (first != cudaSuccess || !params) return first;
      return launch(norm_columns_kernel<TX, TY>,
                    dim3((unsigned)((e->dim + kNormThreads - 1) / kNormThreads), (unsigned)a.parts, (unsigned)e->clients),
                    kNormThreads, 0, 1, st, a);
    });
  });
  if (err == cudaSuccess && params && (is_long || a.parts > 1))
    err = launch(norm_join_kernel, dim3((unsigned)((2 * (int64_t)e->dim + 31) / 32), (unsigned)e->clients), 256, 0, 1, st, a);
  return err == cudaSuccess ? BRACE_OK : cuda_fail_no_ctx(err);
}

size_t brace_clip_workspace_bytes(int32_t clients, const brace_tensor* h_tensors, int32_t count) {
  if (clients < 0 || count < 0 || (count > 0 && !h_tensors)) return 0;
  for (int i = 0; i < count; ++i)
    if (h_tensors[i].rows < 0 || h_tensors[i].cols < 0 || !float_type(h_tensors[i].in_type) ||
        (h_tensors[i].rows > 0 && h_tensors[i].cols > ((int64_t)1 << 46) / h_tensors[i].rows))
      return 0;
  const ClipPlan q = clip_plan(clients, h_tensors, count, true);
  return (size_t)round_up(std::max<int64_t>((int64_t)clients * q.lists * q.ctas * 8, 256), 256);
}

int brace_gradient_norm(int32_t clients, const brace_tensor* h_tensors, int32_t count, float* d_norms, void* d_workspace,
                        size_t workspace_bytes, brace_stream_t stream) {
  const int rc = clip_check(clients, h_tensors, count, false);
  if (rc != BRACE_OK) return rc;
  if (clients == 0) return BRACE_OK;
  if (!typed(d_norms, BRACE_TYPE_F32)) return BRACE_ERR_INVALID_ARG;
  const size_t need = brace_clip_workspace_bytes(clients, h_tensors, count);
  if (!d_workspace || workspace_bytes < need || !aligned(d_workspace, 256)) return BRACE_ERR_WORKSPACE;
  ClipArgs a = {};
  a.norms = d_norms;
  return run_clip(clients, h_tensors, count, false, a, (double*)d_workspace, (cudaStream_t)stream);
}

int brace_gradient_clip(int32_t clients, const brace_tensor* h_tensors, int32_t count, float max_norm, float eps,
                        int32_t nonfinite, float* d_norms, void* d_workspace, size_t workspace_bytes, brace_stream_t stream) {
  if (!std::isfinite(max_norm) || !(max_norm >= 0.f) || !std::isfinite(eps) || !(eps >= 0.f)) return BRACE_ERR_INVALID_ARG;
  if (nonfinite != BRACE_CLIP_PROPAGATE && nonfinite != BRACE_CLIP_ZERO) return BRACE_ERR_INVALID_ARG;
  const int rc = clip_check(clients, h_tensors, count, true);
  if (rc != BRACE_OK) return rc;
  if (clients == 0) return BRACE_OK;
  if (!aligned(d_norms, 4)) return BRACE_ERR_INVALID_ARG;
  const size_t need = brace_clip_workspace_bytes(clients, h_tensors, count);
  if (!d_workspace || workspace_bytes < need || !aligned(d_workspace, 256)) return BRACE_ERR_WORKSPACE;
  ClipArgs a = {};
  a.norms = d_norms;
  a.max_norm = max_norm;
  a.eps = eps;
  a.zero_bad = nonfinite == BRACE_CLIP_ZERO;
  return run_clip(clients, h_tensors, count, true, a, (double*)d_workspace, (cudaStream_t)stream);
}

}  // extern "C"
