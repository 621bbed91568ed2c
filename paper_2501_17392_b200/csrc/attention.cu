// Host side of the windowed attention: argument checks, workspace, launches.  C ABI declared in brace.h.
#include "brace.h"

#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <utility>

#include "attention_host.cuh"
#include "attention_tiles.cuh"

using namespace brace;

namespace {

bool attn_sizes_ok(int32_t batch, int32_t tokens, int32_t heads) { return batch >= 0 && tokens >= 0 && heads >= 0; }
// positions, sums of two of them, and blocks of 32 queries of all heads that share a key are 32-bit numbers
bool attn_served(int32_t batch, int32_t tokens, int32_t heads, int32_t kv_heads, int32_t dim) {
  return batch <= 65535 && tokens <= 1 << 29 && heads <= 65535 && dim <= kHeadMost &&
         (heads == 0 || (tokens / 32 + 2) * (int64_t)(heads / kv_heads) < (int64_t)1 << 31);
}

constexpr int kSms = 148, kGradCtas = 4 * kSms;   // the most that tiles are shared out over, but for long sums

// Head dimensions that the tensor cores' kernels serve.
bool tiles_dim(int32_t dim) { return dim % 8 == 0 && dim <= 128; }

int64_t tiles_of(int32_t tokens, int rows) { return ((int64_t)tokens + rows - 1) / rows; }

// CTAs that few tiles are shared out over: one an SM, and of the kernels in float32, whose tiles have 64 rows, two after one another.
int64_t spread(int rows) { return kSms * (128 / rows); }

// Long sums (kLongBlocks) of up to some hundred tiles are shared out over up to four CTAs a tile, so that the last ones to work
// keep the SMs busy; kLongCtas of them all together take a third of a GB of workspace at most.
constexpr int kLongCtas = 4 * kGradCtas;
int64_t long_pieces(int64_t blocks) { return std::min<int64_t>((blocks + kLongBlocks - 1) / kLongBlocks, 4); }

// Blocks of queries that a tile of keys behind the first tokens is seen by, at most.
int64_t blocks_of(int32_t tokens, int32_t heads, int32_t kv_heads, int32_t window, int rows) {
  return tiles_of((int32_t)std::min<int64_t>(tokens, (int64_t)window + rows - 1), kBlock) * (heads / kv_heads);
}

// What the gradient of dk and dv needs of float32 sums: the most pieces of all tiles that are shared out together (share_out),
// and one sum for each tile whose CTA takes them out of the tensor cores now and then.  More tokens, or a longer window, never
// give fewer.
struct Parts {
  int64_t shared, own;
};
Parts most_parts(int32_t batch, int32_t tokens, int32_t heads, int32_t kv_heads, int32_t window, int32_t sinks, int rows) {
  if (heads == 0) return {0, 0};
  const int64_t each = (int64_t)batch * kv_heads, blocks = blocks_of(tokens, heads, kv_heads, tokens, rows);   // of a tile, at most
  const int64_t first = tiles_of(std::min(sinks, tokens), rows) * each;
  const int64_t tiles = tiles_of(tokens, rows) * each;
  Parts x;
  x.shared = std::max(std::min(std::max<int64_t>(kGradCtas, first), first * blocks), std::min<int64_t>(spread(rows), tiles * blocks));
  x.own = 0;
  if (rows == 128) {
    const int64_t seen = blocks_of(tokens, heads, kv_heads, window, rows);
    x.shared = std::max({x.shared, std::min<int64_t>(kGradCtas, tiles * blocks), long_pieces(seen) > 1 ? std::min<int64_t>(kLongCtas, tiles * long_pieces(seen)) : 0});
    if (seen > kLongBlocks) x.own = tiles;
  }
  return x;
}

// Blocks of 128 keys that a tile of queries walks, at most.
int64_t key_blocks(int32_t tokens, int32_t window, int32_t sinks) {
  if (window >= tokens) return tiles_of(tokens, 128);
  return std::min(tiles_of(tokens, 128) + 1, tiles_of(std::min(sinks, tokens), 128) + tiles_of((int32_t)std::min<int64_t>(tokens, (int64_t)window + 127), 128));
}

// What the gradient keeps in its workspace: two numbers of every query, the ranges, float32 sums.  These are a few hundred MB at
// most, but for windows of more than 65,536 / (heads / kv_heads) queries, where there are up to 4 kv_heads / heads times q's size
// more, and those of more than 65,536 keys, where there is at least twice q's size.
struct GradPlan {
  int64_t padded;
  size_t off_shift, off_range, off_part, bytes;
};
GradPlan grad_plan(int32_t batch, int32_t tokens, int32_t heads, int32_t kv_heads, int32_t dim, int32_t window, int32_t sinks) {
  GradPlan q;
  q.padded = round_up(tokens, kBlock);
  const int64_t numbers = round_up((int64_t)batch * heads * q.padded * 4, 256);
  q.off_shift = (size_t)numbers;
  q.off_range = (size_t)(2 * numbers);
  q.off_part = q.off_range + (size_t)round_up((int64_t)batch * kv_heads * 8, 256);
  // of the tensor cores' kernels or of those in float32, whichever the call will take
  const Parts narrow = most_parts(batch, tokens, heads, kv_heads, window, sinks, kFloatRows);
  int64_t rows = narrow.shared * kFloatRows;
  if (tiles_dim(dim)) {
    const Parts wide = most_parts(batch, tokens, heads, kv_heads, window, sinks, 128);
    rows = std::max(rows, (wide.shared + wide.own) * 128);
    // dq's come first, in the same place
    if (key_blocks(tokens, window, sinks) > kLongKeys / 128) rows = std::max(rows, tiles_of(tokens, 128) * batch * heads * 64);
  }
  q.bytes = q.off_part + (size_t)(rows * 2 * (dim <= 64 ? 64 : dim <= 128 ? 128 : 256) * 4);
  if (q.bytes < 256) q.bytes = 256;
  return q;
}

int attn_check(const brace_window_attention* e) {
  if (!e || !attn_sizes_ok(e->batch, e->tokens, e->heads) || e->kv_heads < 0 || e->dim < 1) return BRACE_ERR_INVALID_ARG;
  if (!float_type(e->type) || e->window < 1 || e->sinks < 0 || !std::isfinite(e->scale)) return BRACE_ERR_INVALID_ARG;
  if (e->heads > 0 && (e->kv_heads < 1 || e->heads % e->kv_heads)) return BRACE_ERR_INVALID_ARG;
  if (!attn_served(e->batch, e->tokens, e->heads, e->kv_heads, e->dim)) return BRACE_ERR_UNSUPPORTED;
  return BRACE_OK;
}

// Whether runs of `run` elements lie apart: of each dimension (elements, stride) with more than one element, from the smallest
// stride on, a step is no shorter than what all those before it reach over.
bool apart(int64_t run, std::initializer_list<std::pair<int64_t, int64_t>> dims) {
  std::pair<int64_t, int64_t> by_stride[3];
  int n = 0;
  for (const auto& d : dims)
    if (d.first > 1) by_stride[n++] = {d.second, d.first};
  std::sort(by_stride, by_stride + n);
  for (int i = 0; i < n; ++i) {
    const int64_t stride = by_stride[i].first, more = by_stride[i].second - 1;
    if (stride < run) return false;
    run = stride > (INT64_MAX - run) / more ? INT64_MAX : run + stride * more;
  }
  return true;
}

// A tensor that is read: any strides that are not negative; one that is written: a place of its own for every row.
bool heads_ok(const brace_heads& x, const brace_window_attention* e, int heads, bool written) {
  if (!x.d || !aligned(x.d, (size_t)elem_bytes(e->type))) return false;
  if (x.ld < 0 || x.head < 0 || x.stride < 0) return false;
  if (!written) return true;
  return apart(e->dim, {{e->tokens, x.ld}, {heads, x.head}, {e->batch, x.stride}});
}

HeadRef head_ref(const brace_heads& x) { return HeadRef{x.d, x.ld, x.head, x.stride}; }

bool attn_common_ok(const brace_window_attention* e, bool grad) {
  if (!heads_ok(e->q, e, e->heads, false) || !heads_ok(e->k, e, e->kv_heads, false) || !heads_ok(e->v, e, e->kv_heads, false))
    return false;
  if (!aligned(e->d_lengths, 4) || !aligned(e->d_lse, 4) || (grad && !e->d_lse)) return false;
  if (!e->d_lse) return true;
  return apart(e->tokens, {{e->heads, e->head_lse}, {e->batch, e->stride_lse}});
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

// Whether the tensor cores' kernels serve this tensor: its rows start on 16-byte boundaries, as loads by tensor maps and
// wide stores ask for, and no dimension is broadcast.
bool tiles_ok(const brace_heads& x, const brace_window_attention* e, int heads) {
  auto stride_ok = [](int64_t s, int64_t n) { return n < 2 || (s > 0 && s % 8 == 0 && s < (int64_t)1 << 38); };
  return aligned(x.d, 16) && stride_ok(x.ld, e->tokens) && stride_ok(x.head, heads) && stride_ok(x.stride, e->batch);
}

bool tiles_served(const brace_window_attention* e, bool grad) {
  if (e->type == BRACE_TYPE_F32 || !tiles_dim(e->dim)) return false;
  if (!tiles_ok(e->q, e, e->heads) || !tiles_ok(e->k, e, e->kv_heads) || !tiles_ok(e->v, e, e->kv_heads)) return false;
  if (!tiles_ok(e->out, e, e->heads)) return false;
  return !grad || (tiles_ok(e->dout, e, e->heads) && tiles_ok(e->dq, e, e->heads) && tiles_ok(e->dk, e, e->kv_heads) && tiles_ok(e->dv, e, e->kv_heads));
}

// Boxes of 64 dimensions x `rows` tokens, 128-byte swizzle, zeros outside.
bool encode_map(CUtensorMap* map, const brace_heads& x, const brace_window_attention* e, int heads, int rows) {
  EncodeFn enc = encode_fn();
  if (!enc) return false;
  auto bytes = [](int64_t s, int64_t n) { return (cuuint64_t)(n < 2 ? 16 : s * 2); };   // of one element's dimension: any
  const cuuint64_t dim[4] = {(cuuint64_t)e->dim, (cuuint64_t)e->tokens, (cuuint64_t)heads, (cuuint64_t)e->batch};
  const cuuint64_t stride[3] = {bytes(x.ld, e->tokens), bytes(x.head, heads), bytes(x.stride, e->batch)};
  const cuuint32_t box[4] = {64, (cuuint32_t)rows, 1, 1}, one[4] = {1, 1, 1, 1};
  return enc(map, e->type == BRACE_TYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, x.d, dim,
             stride, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int D, bool LONG>
cudaError_t launch_forward(const AttnMaps& maps, const AttnArgs& a, cudaStream_t st) {
  using Shape = AttnShape<D, LONG>;
  static_assert(Shape::kSmem * Shape::kCtas <= 232448, "shared memory");
  static std::atomic<uint64_t> granted{0};
  auto* kernel = attn_forward_kernel<T, D, LONG>;
  const cudaError_t err = grant_smem((const void*)kernel, granted, Shape::kSmem);
  if (err != cudaSuccess) return err;
  const dim3 grid((unsigned)((a.tokens + 127) / 128), (unsigned)a.heads, (unsigned)a.batch);
  return launch(kernel, grid, Shape::kThreads, Shape::kSmem, 1, st, maps, a);
}

// The gradient on the tensor cores.  `sums`: the most blocks that a CTA of the kernel that makes dk and dv sums.
template <typename T, int D>
cudaError_t run_grad(const brace_window_attention* e, AttnArgs a, int64_t sums, cudaStream_t st) {
  AttnMaps queries = {}, keys = {};   // for dq, and for dk and dv
  if (!encode_map(&queries.q, e->q, e, e->heads, 128) || !encode_map(&queries.dout, e->dout, e, e->heads, 128) ||
      !encode_map(&queries.k, e->k, e, e->kv_heads, 128) || !encode_map(&queries.v, e->v, e, e->kv_heads, 128) ||
      !encode_map(&keys.q, e->q, e, e->heads, kBlock) || !encode_map(&keys.dout, e->dout, e, e->heads, kBlock))
    return cudaErrorNotSupported;
  keys.k = queries.k;
  keys.v = queries.v;
  constexpr bool kTwo = std::is_same<T, __half>::value;
  const unsigned tiles = (unsigned)((a.tokens + 127) / 128), heads = (unsigned)a.heads, kv_heads = (unsigned)a.kv_heads, batch = (unsigned)a.batch;
  cudaError_t err = cudaSuccess;
  if (kTwo) {
    err = cudaMemsetAsync(a.range, 0, (size_t)a.batch * a.kv_heads * 8, st);
    if (err == cudaSuccess) err = launch(attn_prepare_kernel, dim3((unsigned)(a.padded / kPrepRows), heads, batch), 256, 0, 1, st, a);
  } else {
    a.range = nullptr;
  }
  // kernels that take sums out are 2 to 3 % slower where there is nothing to take out
  const bool long_dq = key_blocks(a.tokens, a.window, a.sinks) > kLongKeys / 128, long_dkv = sums > kLongBlocks;
  auto* dq = long_dq ? attn_dq_kernel<T, D, true> : attn_dq_kernel<T, D, false>;
  auto* dkv = long_dkv ? attn_dkv_kernel<T, D, true> : attn_dkv_kernel<T, D, false>;
  static std::atomic<uint64_t> granted_dkv[2], granted_dq[2];
  // dq first: dk and dv take the numbers of the queries that it made
  if (err == cudaSuccess) err = grant_smem((const void*)dq, granted_dq[long_dq], DqShape<D, kTwo>::kSmem);
  if (err == cudaSuccess)
    err = launch(dq, dim3(tiles, heads, batch), kAttnThreads, DqShape<D, kTwo>::kSmem, 1, st, queries, a);
  if (err == cudaSuccess) err = grant_smem((const void*)dkv, granted_dkv[long_dkv], DkvShape<D>::kSmem);
  if (err == cudaSuccess)
    err = launch(dkv, dim3(a.first_tiles * a.pieces + tiles - a.first_tiles, kv_heads, batch), kAttnThreads,
                 DkvShape<D>::kSmem, 1, st, keys, a);
  if (err == cudaSuccess && a.first_tiles)
    err = launch(attn_join_kernel<T, D, 128>, dim3((unsigned)(a.first_tiles * 32), kv_heads, batch), 128, 0, 1, st, a);
  return err;
}

template <typename F>
cudaError_t with_half_type(int type, F&& f) {
  return type == BRACE_TYPE_BF16 ? f(__nv_bfloat16{}) : f(__half{});
}

// How many CTAs a tile of keys is shared out over, and which tiles are.  Those of first tokens, which all queries see: as many as
// make a CTA's work that of a tile behind them, but no more than give every SM some.  All of them, where there are tiles for less
// than half of the SMs and work for more than one CTA in each (`least` blocks: what is saved has to be more than a launch that
// joins): 3 x 501 tokens, 2 heads read by 6, float32, 118 -> 96 us; 1000 tokens, 8 heads on one of 64, bfloat16, 128 -> 43 us.
// Returns the most blocks that a CTA then sums.
int64_t share_out(const brace_window_attention* e, int rows, int least, AttnArgs& a) {
  const int64_t tiles = tiles_of(e->tokens, rows), first = tiles_of(std::min(e->sinks, e->tokens), rows), each = (int64_t)e->batch * e->kv_heads;
  const int64_t window = std::min<int64_t>(e->tokens, (int64_t)a.window + rows - 1), blocks = blocks_of(e->tokens, e->heads, e->kv_heads, a.window, rows);
  const Parts most = most_parts(e->batch, e->tokens, e->heads, e->kv_heads, a.window, e->sinks, rows);
  a.first_tiles = (int)first;
  a.pieces = 0;
  if (first) {
    const int64_t even = (e->tokens + window - 1) / window;
    a.pieces = (int)std::max<int64_t>(1, std::min(even, most.shared / (first * each)));
  }
  if (tiles * each * 2 <= kSms && blocks >= least) {
    a.first_tiles = (int)tiles;
    a.pieces = (int)std::min(spread(rows) / (tiles * each), blocks);
  }
  // On the tensor cores: long sums, and four CTAs an SM one after another where that leaves each 64 blocks (window as long as the
  // text, bfloat16: 4096 tokens, 16 heads on 2 of 128, 371 -> 280 us; 8192, 32 on 4, window 4096, 1480 -> 1348).
  const int64_t split = rows == 128 ? std::max(std::min(long_pieces(blocks), kLongCtas / (tiles * each)), std::min(kGradCtas / (tiles * each), blocks / 64)) : 1;
  if (split > 1 && (a.first_tiles == 0 || a.pieces <= split)) {     // no tile with first tokens in fewer pieces than above
    a.first_tiles = (int)tiles;
    a.pieces = (int)split;
  }
  a.parts = (int)(a.first_tiles * a.pieces + (most.own ? tiles - a.first_tiles : 0));
  const int64_t longest = first ? tiles_of(e->tokens, kBlock) * a.share : blocks;       // of the tiles that are shared out
  return std::max(a.first_tiles ? (longest + a.pieces - 1) / a.pieces : 0, a.first_tiles < tiles ? blocks : 0);
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
  if (tiles_served(e, false)) {
    AttnMaps maps = {};
    if (!encode_map(&maps.q, e->q, e, e->heads, 128) || !encode_map(&maps.k, e->k, e, e->kv_heads, 128) ||
        !encode_map(&maps.v, e->v, e, e->kv_heads, 128))
      return cuda_fail_no_ctx(cudaErrorNotSupported);
    const cudaError_t err = with_half_type(e->type, [&](auto t) {
      using T = decltype(t);
      const int least = e->dim > 64 && !std::is_same<T, __half>::value ? 4 * kLongKeys : kLongKeys;
      const bool longer = key_blocks(a.tokens, a.window, a.sinks) > least / 128;
      if (e->dim <= 64) return longer ? launch_forward<T, 64, true>(maps, a, st) : launch_forward<T, 64, false>(maps, a, st);
      return longer ? launch_forward<T, 128, true>(maps, a, st) : launch_forward<T, 128, false>(maps, a, st);
    });
    return err == cudaSuccess ? BRACE_OK : cuda_fail_no_ctx(err);
  }
  const cudaError_t err = attn_forward_float(e->type, a, st);
  return err == cudaSuccess ? BRACE_OK : cuda_fail_no_ctx(err);
}

size_t brace_window_attention_window_workspace_bytes(int32_t batch, int32_t tokens, int32_t heads, int32_t kv_heads, int32_t dim,
                                                     int32_t window, int32_t sinks) {
  if (!attn_sizes_ok(batch, tokens, heads) || kv_heads < 0 || dim < 1 || window < 1 || sinks < 0) return 0;
  if (heads > 0 && (kv_heads < 1 || heads % kv_heads)) return 0;
  if (!attn_served(batch, tokens, heads, kv_heads, dim)) return 0;
  return grad_plan(batch, tokens, heads, kv_heads, dim, window, sinks).bytes;
}

size_t brace_window_attention_workspace_bytes(int32_t batch, int32_t tokens, int32_t heads, int32_t kv_heads, int32_t dim,
                                              int32_t sinks) {
  return brace_window_attention_window_workspace_bytes(batch, tokens, heads, kv_heads, dim, INT32_MAX, sinks);
}

int brace_window_attention_grad(const brace_window_attention* e, void* d_workspace, size_t workspace_bytes,
                                brace_stream_t stream) {
  const int rc = attn_check(e);
  if (rc != BRACE_OK) return rc;
  if (e->batch == 0 || e->tokens == 0 || e->heads == 0) return BRACE_OK;
  if (!attn_common_ok(e, true) || !heads_ok(e->out, e, e->heads, false) || !heads_ok(e->dout, e, e->heads, false) ||
      !heads_ok(e->dq, e, e->heads, true) || !heads_ok(e->dk, e, e->kv_heads, true) || !heads_ok(e->dv, e, e->kv_heads, true))
    return BRACE_ERR_INVALID_ARG;
  const size_t need = brace_window_attention_window_workspace_bytes(e->batch, e->tokens, e->heads, e->kv_heads, e->dim, e->window, e->sinks);
  if (!d_workspace || workspace_bytes < need || !aligned(d_workspace, 256)) return BRACE_ERR_WORKSPACE;
  AttnArgs a = attn_args(e);
  a.dout = head_ref(e->dout);
  a.dq = head_ref(e->dq);
  a.dk = head_ref(e->dk);
  a.dv = head_ref(e->dv);
  const GradPlan q = grad_plan(e->batch, e->tokens, e->heads, e->kv_heads, e->dim, e->window, e->sinks);
  char* ws = (char*)d_workspace;
  a.delta = (float*)ws;
  a.shift = (float*)(ws + q.off_shift);
  a.range = (uint32_t*)(ws + q.off_range);
  a.part = (float*)(ws + q.off_part);
  a.padded = q.padded;
  const cudaStream_t st = (cudaStream_t)stream;
  if (tiles_served(e, true)) {
    const int64_t sums = share_out(e, 128, 16, a);
    const cudaError_t err = with_half_type(e->type, [&](auto t) {
      using T = decltype(t);
      return e->dim <= 64 ? run_grad<T, 64>(e, a, sums, st) : run_grad<T, 128>(e, a, sums, st);
    });
    return err == cudaSuccess ? BRACE_OK : cuda_fail_no_ctx(err);
  }
  share_out(e, kFloatRows, 3, a);
  const cudaError_t err = attn_grad_float(e->type, a, st);
  return err == cudaSuccess ? BRACE_OK : cuda_fail_no_ctx(err);
}

}  // extern "C"
