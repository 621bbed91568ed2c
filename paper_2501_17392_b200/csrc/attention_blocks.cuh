// Windowed attention: the blocks of columns that a CTA walks, what a CTA of the backward pass computes, and how the pieces
// of tiles of keys that are shared out are joined.
#pragma once

#include "attention_rows.cuh"

namespace brace {

// The blocks of keys that a CTA walks: those of the first tokens that lie before the window of its first query, then the
// window's, from the first key of the first query's window on.
struct KeyBlocks {
  int lo, first, nfirst, count;
  __device__ __forceinline__ KeyBlocks(const AttnArgs& p, int q_first, int q_end, int width) {
    lo = max(0, q_first - p.window + 1);
    first = min(p.sinks, lo);
    nfirst = (first + width - 1) / width;
    count = nfirst + (q_end - lo + width - 1) / width;
  }
  __device__ __forceinline__ int key(int k, int width) const { return k < nfirst ? k * width : lo + (k - nfirst) * width; }
};

// What a CTA of the backward pass computes: `rows` rows of dq, or of dk and dv (dkv), over its blocks of `width` columns.
// The first p.first_tiles tiles of keys (those with first tokens, which all queries see, or all where there are few) are each
// shared out over p.pieces CTAs, which leave float32 sums.  grid: dkv (pieces of those tiles, then tiles; kv heads; sequences),
// else (tiles of queries, heads, sequences)
struct GradWork {
  int row0, head, count;                   // first row; head of the rows; blocks
  int tile, piece;                         // that is shared out, or -1
  int begin, per_head, width;              // first block, blocks of queries of a head (dkv)
  KeyBlocks keys;                          // (dq)
  bool dkv;
  __device__ __forceinline__ GradWork(const AttnArgs& p, int n, bool of_keys, int rows, int block)
      : row0(first_row(p, of_keys, rows)), head(blockIdx.y), count(0), tile(-1), piece(-1), begin(0), per_head(1), width(block),
        keys(p, row0, min(n, row0 + rows), block), dkv(of_keys) {
    if (dkv && (int)blockIdx.x < p.first_tiles * p.pieces) {
      tile = blockIdx.x / p.pieces;
      piece = blockIdx.x % p.pieces;
    }
    if (row0 >= n) return;
    if (!dkv) {
      count = keys.count;
      return;
    }
    // the tile's queries: from its first key to the end of its last one's window, or all from there on
    const int stop = row0 < p.sinks || p.window + rows - 1 > n - row0 ? n : row0 + rows - 1 + p.window;
    per_head = (stop - row0 + block - 1) / block;
    const int64_t all = (int64_t)per_head * p.share;
    if (piece >= 0) begin = (int)(all * piece / p.pieces);
    count = (piece >= 0 ? (int)(all * (piece + 1) / p.pieces) : (int)all) - begin;
  }
  static __device__ __forceinline__ int first_row(const AttnArgs& p, bool dkv, int rows) {
    const int x = blockIdx.x, first = p.first_tiles * p.pieces;
    if (!dkv) return rows * (int)(gridDim.x - 1 - blockIdx.x);     // the last queries first: they have the longest windows
    return rows * (x < first ? x / p.pieces : p.first_tiles + x - first);
  }
  // block k: its head, its first column
  __device__ __forceinline__ int head_of(int k, const AttnArgs& p) const {
    return dkv ? head * p.share + (begin + k) / per_head : head / p.share;
  }
  __device__ __forceinline__ int first(int k) const { return dkv ? row0 + (begin + k) % per_head * width : keys.key(k, width); }
  // where this CTA's float32 sums of dv (which = 0) or dk lie: those of a piece, or of a tile of its own
  __device__ __forceinline__ int64_t part_of(const AttnArgs& p, int b, int which, int rows, int d) const {
    const int at = piece >= 0 ? tile * p.pieces + piece : p.first_tiles * (p.pieces - 1) + row0 / rows;
    return ((((int64_t)b * p.kv_heads + head) * p.parts + at) * 2 + which) * rows * d;
  }
};

// dv and dk of the tiles that are shared out from their pieces: a warp a row.  grid: (rows of the tiles / 4, kv heads, sequences)
template <typename T, int D, int ROWS>
__global__ void __launch_bounds__(128) attn_join_kernel(const AttnArgs p) {
  grid_trigger();
  grid_wait();
  const int j = blockIdx.x * 4 + (threadIdx.x >> 5), g = blockIdx.y, b = blockIdx.z, lane = threadIdx.x & 31, n = attn_length(p, b);
  if (j >= p.tokens) return;
  bool bad = false;
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    T* to = head_row<T>(r ? p.dk : p.dv, b, j, g);
    const float* from = p.part + ((((int64_t)b * p.kv_heads + g) * p.parts + j / ROWS * p.pieces) * 2 + r) * ROWS * D + j % ROWS * D;
#pragma unroll
    for (int col = 0; col < D; col += 32) {
      const int d = col + lane;
      float sum = 0.f;
      if (j < n)
        for (int k = 0; k < p.pieces; ++k) sum += from[(int64_t)k * 2 * ROWS * D + d];
      if (d < p.dim) {
        bad |= !isfinite(sum);
        to[d] = from_f32<T>(sum);
      }
    }
  }
  __syncwarp();
  if (__any_sync(0xffffffffu, bad)) dkv_row<T>(p, b, g, j, n);
}

}  // namespace brace
