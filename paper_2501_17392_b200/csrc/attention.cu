// Host side of the windowed attention: argument checks, workspace, launches.  C ABI declared in brace.h.
#include "brace.h"

#include <algorithm>
#include <cmath>

#include "attention_rows.cuh"
#include "host.cuh"

using namespace brace;

namespace {

bool attn_sizes_ok(int32_t batch, int32_t tokens, int32_t heads) { return batch >= 0 && tokens >= 0 && heads >= 0; }
bool attn_served(int32_t batch, int32_t heads, int32_t dim) { return batch <= 65535 && heads <= 65535 && dim <= kHeadMost; }

size_t attn_bytes(int32_t batch, int32_t tokens, int32_t heads) {
  return (size_t)round_up(std::max<int64_t>((int64_t)batch * tokens * heads * 4, 256), 256);
}

int attn_check(const brace_window_attention* e) {
  if (!e || !attn_sizes_ok(e->batch, e->tokens, e->heads) || e->kv_heads < 0 || e->dim < 1) return BRACE_ERR_INVALID_ARG;
  if (!float_type(e->type) || e->window < 1 || e->sinks < 0 || !std::isfinite(e->scale)) return BRACE_ERR_INVALID_ARG;
  if (e->heads > 0 && (e->kv_heads < 1 || e->heads % e->kv_heads)) return BRACE_ERR_INVALID_ARG;
  if (!attn_served(e->batch, e->heads, e->dim)) return BRACE_ERR_UNSUPPORTED;
  return BRACE_OK;
}

// A tensor that is read: any strides that are not negative; one that is written: a place of its own for every row.
bool heads_ok(const brace_heads& x, const brace_window_attention* e, int heads, bool written) {
  if (!x.d || !aligned(x.d, (size_t)elem_bytes(e->type))) return false;
  if (x.ld < 0 || x.head < 0 || x.stride < 0) return false;
  if (!written) return true;
  return (e->tokens < 2 || x.ld >= e->dim) && (heads < 2 || x.head >= e->dim) && (e->batch < 2 || x.stride >= e->dim);
}

HeadRef head_ref(const brace_heads& x) { return HeadRef{x.d, x.ld, x.head, x.stride}; }

bool attn_common_ok(const brace_window_attention* e, bool grad) {
  if (!heads_ok(e->q, e, e->heads, false) || !heads_ok(e->k, e, e->kv_heads, false) || !heads_ok(e->v, e, e->kv_heads, false))
    return false;
  if (!aligned(e->d_lengths, 4) || !aligned(e->d_lse, 4) || (grad && !e->d_lse)) return false;
  if (!e->d_lse) return true;
  return (e->heads < 2 || e->head_lse >= e->tokens) && (e->batch < 2 || e->stride_lse >= e->tokens);
}

AttnArgs attn_args(const brace_window_attention* e) {
  AttnArgs a = {};
  a.q = head_ref(e->q);
  a.k = head_ref(e->k);
  a.v = head_ref(e->v);
  a.out = head_ref(e->out);
  a.lse = e->d_lse;
  a.stride_lse = e->stride_lse;
  a.head_lse = e->head_lse;
  a.lengths = e->d_lengths;
  a.batch = e->batch;
  a.tokens = e->tokens;
  a.heads = e->heads;
  a.kv_heads = e->kv_heads;
  a.share = e->heads / e->kv_heads;
  a.dim = e->dim;
  // nothing is further than that; sums of positions and these stay below 2^31
  a.window = std::min(e->window, e->tokens);
  a.sinks = std::min(e->sinks, e->tokens);
  a.scale = e->scale;
  return a;
}

dim3 row_grid(const brace_window_attention* e, int heads) {
  return dim3((unsigned)((e->tokens + 3) / 4), (unsigned)heads, (unsigned)e->batch);
}

}  // namespace

extern "C" {

int brace_window_attention_forward(const brace_window_attention* e, brace_stream_t stream) {
  const int rc = attn_check(e);
  if (rc != BRACE_OK) return rc;
  if (e->batch == 0 || e->tokens == 0 || e->heads == 0) return BRACE_OK;
  if (!attn_common_ok(e, false) || !heads_ok(e->out, e, e->heads, true)) return BRACE_ERR_INVALID_ARG;
  const AttnArgs a = attn_args(e);
  const cudaStream_t st = (cudaStream_t)stream;
  const cudaError_t err = with_type(e->type, [&](auto t) {
    return launch(attn_forward_rows_kernel<decltype(t)>, row_grid(e, e->heads), kRowThreads, 0, 1, st, a);
  });
  return err == cudaSuccess ? BRACE_OK : cuda_fail_no_ctx(err);
}

size_t brace_window_attention_workspace_bytes(int32_t batch, int32_t tokens, int32_t heads, int32_t kv_heads, int32_t dim,
                                              int32_t sinks) {
  if (!attn_sizes_ok(batch, tokens, heads) || kv_heads < 0 || dim < 1 || sinks < 0) return 0;
  if (heads > 0 && (kv_heads < 1 || heads % kv_heads)) return 0;
  if (!attn_served(batch, heads, dim)) return 0;
  return attn_bytes(batch, tokens, heads);
}

int brace_window_attention_grad(const brace_window_attention* e, void* d_workspace, size_t workspace_bytes,
                                brace_stream_t stream) {
  const int rc = attn_check(e);
  if (rc != BRACE_OK) return rc;
  if (e->batch == 0 || e->tokens == 0 || e->heads == 0) return BRACE_OK;
  if (!attn_common_ok(e, true) || !heads_ok(e->out, e, e->heads, false) || !heads_ok(e->dout, e, e->heads, false) ||
      !heads_ok(e->dq, e, e->heads, true) || !heads_ok(e->dk, e, e->kv_heads, true) || !heads_ok(e->dv, e, e->kv_heads, true))
    return BRACE_ERR_INVALID_ARG;
  const size_t need = brace_window_attention_workspace_bytes(e->batch, e->tokens, e->heads, e->kv_heads, e->dim, e->sinks);
  if (!d_workspace || workspace_bytes < need || !aligned(d_workspace, 256)) return BRACE_ERR_WORKSPACE;
  AttnArgs a = attn_args(e);
  a.dout = head_ref(e->dout);
  a.dq = head_ref(e->dq);
  a.dk = head_ref(e->dk);
  a.dv = head_ref(e->dv);
  a.delta = (float*)d_workspace;
  const cudaStream_t st = (cudaStream_t)stream;
  const cudaError_t err = with_type(e->type, [&](auto t) {
    using T = decltype(t);
    cudaError_t r = launch(attn_delta_kernel<T>, row_grid(e, e->heads), kRowThreads, 0, 1, st, a);
    if (r == cudaSuccess) r = launch(attn_dq_rows_kernel<T>, row_grid(e, e->heads), kRowThreads, 0, 1, st, a);
    if (r == cudaSuccess) r = launch(attn_dkv_rows_kernel<T>, row_grid(e, e->kv_heads), kRowThreads, 0, 1, st, a);
    return r;
  });
  return err == cudaSuccess ? BRACE_OK : cuda_fail_no_ctx(err);
}

}  // extern "C"
