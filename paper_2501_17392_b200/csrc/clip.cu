// Host side of the gradients' norm and of clipping: argument checks, workspace, launches.  C ABI declared in brace.h.
#include "brace.h"

#include <algorithm>
#include <cmath>
#include <cstring>
#include <functional>
#include <memory>
#include <new>
#include <type_traits>

#include "clip_kernels.cuh"
#include "host.cuh"

using namespace brace;

namespace {

constexpr int kClipCtas = 148 * 4 * kClipResident;        // of a launch: four rounds, the last ones even the first ones out
// Units of a client that a cluster takes in one launch: two launches are as fast from some 200,000 elements on.  A CTA is given
// kClusterShare of them before another one is.
constexpr int64_t kClusterUnits = 64, kClusterShare = 2;
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

int clip_cap(int32_t count) { return count <= kClipSmall ? kClipSmall : count <= kClipList ? kClipList : kClipLongList; }

// Most CTAs of a client in a launch.
int64_t clip_ctas(int32_t clients) { return std::max(kClipCtas / std::max(clients, 1), 1); }

// Whether two tensors are written to one place: their CTAs would race on it.
bool clip_twice(const brace_tensor* t, int32_t count) {
  const void* few[kClipLongList];
  std::unique_ptr<const void*[]> many(count > kClipLongList ? new (std::nothrow) const void*[count] : nullptr);
  if (count > kClipLongList && !many) return false;      // no memory to look
  const void** p = many ? many.get() : few;
  int n = 0;
  for (int i = 0; i < count; ++i)
    if (t[i].rows && t[i].cols) p[n++] = t[i].d_out;
  std::sort(p, p + n, std::less<const void*>());
  return std::adjacent_find(p, p + n) != p + n;
}

int clip_check(int32_t clients, const brace_tensor* t, int32_t count, bool clip) {
  if (clients < 0 || clients > 65535 || count < 0 || (count > 0 && !t)) return BRACE_ERR_INVALID_ARG;
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
  return clip && clients > 0 && clip_twice(t, count) ? BRACE_ERR_INVALID_ARG : BRACE_OK;
}

// Calls f with a value of the pair's two element types and the list's size.
template <typename F>
cudaError_t with_list(int pair, int cap, F&& f) {
  using std::integral_constant;
  return with_type(pair / 3, [&](auto ti) {
    return with_type(pair % 3, [&](auto to) {
      return cap == kClipSmall  ? f(ti, to, integral_constant<int, kClipSmall>{})
             : cap == kClipList ? f(ti, to, integral_constant<int, kClipList>{})
                                : f(ti, to, integral_constant<int, kClipLongList>{});
    });
  });
}

enum { kSum, kApply, kCluster };

// One launch for the tensors of `a`, all of one pair of types.
cudaError_t launch_clip(int what, int pair, int cap, int clients, const ClipArgs& a, const ClipTensor* tensors, int64_t ctas,
                        cudaStream_t st) {
  return with_list(pair, cap, [&](auto ti, auto to, auto n) {
    using TI = decltype(ti);
    constexpr int CAP = decltype(n)::value;
    ClipList<CAP> list;
    std::memcpy(list.t, tensors, sizeof(ClipTensor) * a.count);
    const dim3 grid((unsigned)ctas, (unsigned)clients);
    if (what == kSum) return launch(clip_sum_kernel<TI, CAP>, grid, kClipThreads, 0, 1, st, a, list);
    if (what == kApply) return launch(clip_apply_kernel<TI, decltype(to), CAP>, grid, kClipThreads, 0, 1, st, a, list);
    return launch(clip_cluster_kernel<TI, decltype(to), CAP>, grid, kClipThreads, 0, (int)ctas, st, a, list);
  });
}

// What launches take of the tensors, one after the other: some of those of one pair of types, in their order.
struct ClipTake {
  int pair, next;   // the pair of types, and the tensor to look at next
};

int run_clip(int32_t clients, const brace_tensor* t, int32_t count, bool clip, ClipArgs a, char* ws, cudaStream_t st) {
  const int cap = clip_cap(count);
  const int64_t most = clip_ctas(clients);
  ClipTensor tensors[kClipLongList];
  // Fills `tensors`, a.count and a.units with what comes next; false at the end.
  auto take = [&](ClipTake& at) {
    a.count = 0;
    a.units = 0;
    for (; at.pair < 9; ++at.pair, at.next = 0) {
      for (; at.next < count && a.count < cap; ++at.next) {
        const brace_tensor& x = t[at.next];
        if (x.rows == 0 || x.cols == 0 || (clip ? x.in_type * 3 + x.out_type : x.in_type * 4) != at.pair) continue;
        ClipTensor& y = tensors[a.count++];
        const bool flat = clip_flat(x, clip);
        y.in = x.d_in;
        y.out = x.d_out;
        y.rows = flat ? 1 : x.rows;
        y.cols = flat ? x.rows * x.cols : x.cols;
        y.ld_in = x.ld_in;
        y.ld_out = x.ld_out;
        y.stride_in = x.stride_in;
        y.stride_out = x.stride_out;
        y.unit0 = a.units;
        a.units += clip_units_of(x, clip, &y.row_units);
      }
      if (a.count) return true;
    }
    return false;
  };
  a.part = (double*)ws;
  a.parts = 0;
  int launches = 0;
  for (ClipTake at = {}; take(at); ++launches) a.parts += std::min(a.units, most);
  cudaError_t err = cudaSuccess;
  if (clip && launches == 1) {
    ClipTake at = {};
    take(at);
    if (a.units <= kClusterUnits) {
      int64_t ctas = 1;
      while (ctas < kClusterMost && ctas * kClusterShare < a.units) ctas *= 2;
      err = launch_clip(kCluster, at.pair, cap, clients, a, tensors, ctas, st);
      return err == cudaSuccess ? BRACE_OK : cuda_fail_no_ctx(err);
    }
  }
  for (int what = kSum; what <= (clip ? kApply : kSum); ++what) {
    a.part0 = 0;
    for (ClipTake at = {}; err == cudaSuccess && take(at);) {
      const int64_t ctas = std::min(a.units, most);
      err = launch_clip(what, at.pair, cap, clients, a, tensors, ctas, st);
      a.part0 += ctas;
    }
  }
  if (err == cudaSuccess && a.norms && (!clip || !a.parts)) err = launch(clip_norms_kernel, dim3((unsigned)clients), kClipThreads, 0, 1, st, a);
  return err == cudaSuccess ? BRACE_OK : cuda_fail_no_ctx(err);
}

}  // namespace

extern "C" {

size_t brace_clip_workspace_bytes(int32_t clients, const brace_tensor* h_tensors, int32_t count) {
  if (clients < 0 || clients > 65535 || count < 0 || (count > 0 && !h_tensors)) return 0;
  for (int i = 0; i < count; ++i)
    if (h_tensors[i].rows < 0 || h_tensors[i].cols < 0 || !float_type(h_tensors[i].in_type) ||
        (h_tensors[i].rows > 0 && h_tensors[i].cols > ((int64_t)1 << 46) / h_tensors[i].rows))
      return 0;
  // a sum of each CTA of each list of tensors; a pair of types begins a list
  const int64_t parts = (count / clip_cap(count) + 9) * clip_ctas(clients);
  return (size_t)round_up(std::max<int64_t>(clients * parts * 8, 256), 256);
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
  return run_clip(clients, h_tensors, count, false, a, (char*)d_workspace, (cudaStream_t)stream);
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
  return run_clip(clients, h_tensors, count, true, a, (char*)d_workspace, (cudaStream_t)stream);
}

}  // extern "C"
