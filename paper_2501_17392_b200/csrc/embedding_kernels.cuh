// Kernels of the embedding table (sm_100a): rows for tokens, and the table's gradient by sorted tokens.
//
//   lookup    out[c][t] = scale * table[c][id[c][t]], 0 for an id outside [0, vocab)
//   gradient  grad[c][v] = scale * sum over the t with id[c][t] = v, in increasing t, of dy[c][t]
//
// Both are bound by memory.  The gradient needs, for every row of the table, the tokens that hit it: each client's
// ids are sorted (stably, so the sums have one order and the result is the same every time; no atomics), then the
// table is written once, row by row, zeros included.
#pragma once

#include "elements.cuh"
#include "sm100.cuh"

namespace brace {

constexpr uint32_t kNoToken = 0xffffffffu;   // sorts behind every id
constexpr int kDirectTokens = 2048;          // up to so many tokens no sort is needed: one launch does it all
constexpr int kSortItems = 4;                // elements per thread of the sort
constexpr int kSortThreads = 512;
constexpr int kSortTile = kSortThreads * kSortItems;
// The sort: digits of 9 bits, tiles of a multiple of kSortTile tokens, at most kMostTiles a client.
constexpr int kWideBits = 9;
constexpr int kWideDigits = 1 << kWideBits;
constexpr int kMostTiles = 256;
constexpr int kPart = 32;                    // sorted tokens of a group: a CTA's share of the sums
constexpr int kManyGroups = 16;              // from here on a whole CTA adds a row's partial sums
constexpr int kManyTokens = 16;              // ... or its tokens, where there are few in all

struct EmbArgs {
  const void* table;      // lookup: the table
  void* grad;             // gradient: the table's gradient
  const void* ids;
  const void* in;         // gradient: dy
  void* out;              // lookup: rows
  int64_t ld_table, stride_table, stride_ids, ld_act, stride_act;
  int64_t tokens, vocab;
  int clients, dim;
  int id_bytes;
  float scale;
  int accumulate;
  // gradient
  uint32_t *key, *pos;    // [clients][tokens], sorted by (key, pos)
  uint2* span;            // [clients][vocab]: where an id's sorted tokens begin and end; only those of ids that occur
                          // are written, what else is there is told by the keys (see has_tokens)
  float* part;            // [clients][parts][2][dim]: of each group of kPart sorted tokens, the sums of the first id
                          // if its tokens began in an earlier group, and of the last one if they only go on in the next
  int64_t parts;
  int rows_cta;           // rows of a CTA that writes zeros
  uint32_t zero_ctas, join_split;   // those CTAs, and the CTAs that share the columns of eight groups' joins
};

__device__ __forceinline__ int64_t load_id(const EmbArgs& p, int64_t c, int64_t t) {
  return p.id_bytes == 8 ? ((const int64_t*)p.ids)[c * p.stride_ids + t]
                         : (int64_t)((const int32_t*)p.ids)[c * p.stride_ids + t];
}

// ---- lookup -----------------------------------------------------------------------------------------------------
// A warp takes kLookupRows rows and of each a stretch of 32 V Q columns, all loads first.  Rows that do not start on
// whole words are read and written element by element, 32 neighbours at a time.  Bound by HBM: 16 x 8192 rows of 768 in
// 65.5 us, 0.87 of the copy rate by the rows read once and written once (threads that divided a flat index took 79 us).
constexpr int kLookupRows = 4;

template <typename TI, typename TO, int V>
__global__ void __launch_bounds__(256) embedding_lookup_kernel(const EmbArgs p) {
  constexpr int Q = V >= 8 ? 1 : V == 2 ? 2 : 4, R = kLookupRows;
  grid_wait();
  grid_trigger();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t c = blockIdx.y, t0 = ((int64_t)blockIdx.x * 8 + warp) * R;
  const int rows = (int)min((int64_t)R, p.tokens - t0);
  if (rows <= 0) return;
  const int col = (int)blockIdx.z * (32 * V * Q) + lane * V, left = p.dim - col;
  // lane r knows row r's id; what is no token is -1
  int64_t id = -1;
  if (lane < rows) {
    id = load_id(p, c, t0 + lane);
    if (id >= p.vocab) id = -1;
  }
  const TI* table = (const TI*)p.table + c * p.stride_table + col;
  TO* out = (TO*)p.out + c * p.stride_act + t0 * p.ld_act + col;
  Pack<TI, V> x[R][Q];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int64_t v = __shfl_sync(0xffffffffu, id, r);
    const TI* row = table + v * p.ld_table;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      if (v >= 0 && 32 * V * q < left) {
        x[r][q].load(row + 32 * V * q);
      } else {
#pragma unroll
        for (int j = 0; j < V; ++j) x[r][q].t[j] = from_f32<TI>(0.f);
      }
    }
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (r >= rows) break;
#pragma unroll
    for (int q = 0; q < Q; ++q)
      if (32 * V * q < left) {
        Pack<TO, V> y;
#pragma unroll
        for (int j = 0; j < V; ++j) y.t[j] = from_f32<TO>(to_f32(x[r][q].t[j]) * p.scale);
        y.store_stream(out + r * p.ld_act + 32 * V * q);
      }
  }
}

// ---- gradient: sort ---------------------------------------------------------------------------------------------
// The lanes of a warp with this lane's digit, bit by bit (a match instruction takes several times as long).
template <int BITS>
__device__ __forceinline__ uint32_t same_digit(uint32_t digit) {
  uint32_t same = 0xffffffffu;
#pragma unroll
  for (int b = 0; b < BITS; ++b) {
    const bool set = (digit >> b) & 1u;
    const uint32_t with = __ballot_sync(0xffffffffu, set);
    same &= set ? with : ~with;
  }
  return same;
}

// More tokens: least significant digit first over tiles.  16 x 8192 ids of 17 bits take 21 us in three launches, bound by
// the latency of each; sorting them in one CTA a client took 20 us and grew with the tokens, merging sorted runs by
// searches 20 us a level.  hist[pass][client][tile][digit] counts
// the digits of a pass in each tile of its input.  This kernel counts the first pass and clears the others' counts.
__global__ void __launch_bounds__(kSortThreads) embedding_count_kernel(const EmbArgs p, uint32_t* hist, int64_t tile, int passes) {
  __shared__ uint32_t s_count[kWideDigits];
  grid_wait();
  grid_trigger();
  const int64_t c = blockIdx.y, first = (int64_t)blockIdx.x * tile, last = min(p.tokens, first + tile);
  s_count[threadIdx.x] = 0;
  __syncthreads();
  for (int64_t t = first + threadIdx.x; t < last; t += kSortThreads) {
    const int64_t id = load_id(p, c, t);
    const uint32_t key = id >= 0 && id < p.vocab ? (uint32_t)id : kNoToken;
    atomicAdd(&s_count[key & (kWideDigits - 1)], 1u);
  }
  __syncthreads();
  const int64_t plane = (int64_t)gridDim.y * gridDim.x * kWideDigits;
  uint32_t* mine = hist + (c * gridDim.x + blockIdx.x) * kWideDigits + threadIdx.x;
  *mine = s_count[threadIdx.x];
  for (int q = 1; q < passes; ++q) mine[q * plane] = 0;
}

// One pass: a tile's elements go behind those of smaller digits and of earlier tiles, in their order.  Counts the next
// pass's digits as it goes (adding whole numbers, so the order of the additions does not matter).
template <bool FIRST>
__global__ void __launch_bounds__(kSortThreads) embedding_scatter_kernel(const EmbArgs p, uint32_t* hist, int64_t tile, int pass,
                                                                         int passes, uint32_t* out_key, uint32_t* out_pos) {
  constexpr int kWarps = kSortThreads / 32;
  static_assert(kSortThreads == kWideDigits, "a thread per digit");
  __shared__ uint32_t s_count[kWarps][kWideDigits];
  __shared__ uint32_t s_base[kWideDigits];
  __shared__ uint32_t s_warp[kWarps];
  grid_wait();
  grid_trigger();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int64_t c = blockIdx.y, first = (int64_t)blockIdx.x * tile, last = min(p.tokens, first + tile);
  const int64_t plane = (int64_t)gridDim.y * gridDim.x * kWideDigits;
  const uint32_t* counts = hist + pass * plane + c * gridDim.x * kWideDigits + tid;
  uint32_t before = 0, total = 0;
#pragma unroll 8
  for (unsigned t = 0; t < gridDim.x; ++t) {
    const uint32_t n = counts[(int64_t)t * kWideDigits];
    total += n;
    before += t < blockIdx.x ? n : 0;
  }
  uint32_t incl = total;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t v = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += v;
  }
  if (lane == 31) s_warp[warp] = incl;
  __syncthreads();
  uint32_t front = lane < warp ? s_warp[lane] : 0;
#pragma unroll
  for (int o = 16; o; o >>= 1) front += __shfl_xor_sync(0xffffffffu, front, o);
  s_base[tid] = front + incl - total + before;
  const int shift = pass * kWideBits;
  uint32_t* next = hist + (pass + 1) * plane + c * gridDim.x * kWideDigits;
  for (int64_t t0 = first; t0 < last; t0 += kSortTile) {
#pragma unroll
    for (int w = 0; w < kWarps; ++w) s_count[w][tid] = 0;
    __syncthreads();
    uint32_t key[kSortItems], pos[kSortItems], rank[kSortItems];
#pragma unroll
    for (int i = 0; i < kSortItems; ++i) {
      const int64_t t = t0 + (warp * kSortItems + i) * 32 + lane;
      key[i] = kNoToken;
      pos[i] = (uint32_t)t;
      if (t < last) {
        if (FIRST) {
          const int64_t id = load_id(p, c, t);
          if (id >= 0 && id < p.vocab) key[i] = (uint32_t)id;
        } else {
          key[i] = p.key[c * p.tokens + t];
          pos[i] = p.pos[c * p.tokens + t];
        }
      }
    }
#pragma unroll
    for (int i = 0; i < kSortItems; ++i) {
      const bool live = t0 + (warp * kSortItems + i) * 32 + lane < last;
      const uint32_t digit = (key[i] >> shift) & (kWideDigits - 1);
      const uint32_t same = same_digit<kWideBits>(digit) & __ballot_sync(0xffffffffu, live);
      const uint32_t already = s_count[warp][digit];
      rank[i] = already + __popc(same & ((1u << lane) - 1u));
      __syncwarp();
      if (live && lane == __ffs(same) - 1) s_count[warp][digit] = already + __popc(same);
      __syncwarp();
    }
    __syncthreads();
    uint32_t run = s_base[tid];
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const uint32_t n = s_count[w][tid];
      s_count[w][tid] = run;
      run += n;
    }
    s_base[tid] = run;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kSortItems; ++i) {
      if (t0 + (warp * kSortItems + i) * 32 + lane < last) {
        const uint32_t to = s_count[warp][(key[i] >> shift) & (kWideDigits - 1)] + rank[i];
        out_key[c * p.tokens + to] = key[i];
        out_pos[c * p.tokens + to] = pos[i];
        if (pass + 1 < passes)
          atomicAdd(&next[(int64_t)(to / (uint32_t)tile) * kWideDigits + ((key[i] >> (shift + kWideBits)) & (kWideDigits - 1))], 1u);
      }
    }
    __syncthreads();
  }
}

// ---- gradient: sums ---------------------------------------------------------------------------------------------
// A warp's share of a row: lane l takes the V elements from l V on of each of Q stretches of 32 V, so that narrow
// accesses too have several loads under way.
template <int V>
struct Share {
  static constexpr int Q = V >= 8 ? 1 : V == 2 ? 2 : 4;
  static constexpr int kWide = 32 * V * Q;
  float sum[Q][V];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int j = 0; j < V; ++j) sum[q][j] = 0.f;
  }
  // R rows at a time, all their loads first.
  template <typename T, int R, typename At>
  __device__ __forceinline__ void add_some(int i, int left, At at) {
    Pack<T, V> x[R][Q];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const T* row = at(i + r);
#pragma unroll
      for (int q = 0; q < Q; ++q)
        if (32 * V * q < left) x[r][q].load(row + 32 * V * q);
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int q = 0; q < Q; ++q)
        if (32 * V * q < left)
#pragma unroll
          for (int j = 0; j < V; ++j) sum[q][j] += to_f32(x[r][q].t[j]);
  }
  // Adds `n` rows at(0) .. at(n - 1); `left`: elements of the row from the lane's first one on.
  template <typename T, typename At>
  __device__ __forceinline__ void add(int n, int left, At at) {
    constexpr int R = V * sizeof(T) * Q <= 16 ? 4 : 2;
    int i = 0;
#pragma unroll 1
    for (; i + R <= n; i += R) add_some<T, R>(i, left, at);
#pragma unroll 1
    for (; i < n; ++i) add_some<T, 1>(i, left, at);
  }
  // Warps first, first + 1, .. of the CTA hold shares of one sum; the first of them gets it.
  __device__ __forceinline__ void join(float (*scratch)[kWide], int first, int warps) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int j = 0; j < V; ++j) scratch[warp][(q * V + j) * 32 + lane] = sum[q][j];
    __syncthreads();
    if (warp == first)
      for (int t = 1; t < warps; ++t)
#pragma unroll
        for (int q = 0; q < Q; ++q)
#pragma unroll
          for (int j = 0; j < V; ++j) sum[q][j] += scratch[first + t][(q * V + j) * 32 + lane];
    __syncthreads();
  }
  __device__ __forceinline__ void to_part(float* p, int left) const {
#pragma unroll
    for (int q = 0; q < Q; ++q)
      if (32 * V * q < left)
#pragma unroll
        for (int j = 0; j < V; ++j) p[32 * V * q + j] = sum[q][j];
  }
  template <typename TO>
  __device__ __forceinline__ void to_row(TO* p, int left, float scale, bool accumulate) const {
#pragma unroll
    for (int q = 0; q < Q; ++q)
      if (32 * V * q < left) {
        Pack<TO, V> y;
        if (accumulate) y.load(p + 32 * V * q);
#pragma unroll
        for (int j = 0; j < V; ++j) y.t[j] = from_f32<TO>((accumulate ? to_f32(y.t[j]) : 0.f) + sum[q][j] * scale);
        y.store_stream(p + 32 * V * q);
      }
  }
};

// Bound by the latency of scattered rows: 16 x 8192 tokens of 768 in 85 us, 2.4 TB/s of activations (with one row in
// flight a warp it took 98).
// A CTA takes a group of kPart sorted tokens: notes where each id's tokens begin and end, writes the rows of the ids
// whose tokens all lie in the group, and leaves a partial sum of an id that goes on before ([0]) or only after ([1]).
template <typename TI, typename TO, int V>
__global__ void __launch_bounds__(256, 4) embedding_sum_kernel(const EmbArgs p) {
  static_assert(kPart == 32, "a lane per token of a group");
  using S = Share<V>;
  __shared__ float s_sum[8][S::kWide];
  __shared__ uint32_t s_key[32], s_pos[32];
  // ids with one token, all of it here: where it is; the other segments: where they begin and end, and whether the id
  // has tokens in an earlier group (1) or a later one (2)
  __shared__ int s_single[32], s_first[32], s_last[32], s_goes[32], s_counts[2];
  grid_wait();
  grid_trigger();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t c = blockIdx.y, g = blockIdx.x;
  if (warp == 0) {
    const int64_t i = g * kPart + lane;
    const uint32_t* key = p.key + c * p.tokens;
    const uint32_t k = i < p.tokens ? key[i] : kNoToken;
    uint32_t before = __shfl_up_sync(0xffffffffu, k, 1), after = __shfl_down_sync(0xffffffffu, k, 1);
    if (lane == 0) before = i > 0 ? key[i - 1] : kNoToken;
    if (lane == 31) after = i + 1 < p.tokens ? key[i + 1] : kNoToken;
    const bool token = k != kNoToken, head = token && (lane == 0 || before != k), tail = token && (lane == 31 || after != k);
    if (token) {   // (every CTA of a group writes the same)
      if (before != k) p.span[c * p.vocab + k].x = (uint32_t)i;
      if (after != k) p.span[c * p.vocab + k].y = (uint32_t)i + 1;
      s_key[lane] = k;
      s_pos[lane] = p.pos[c * p.tokens + i];
    }
    const int goes = (lane == 0 && token && before == k ? 1 : 0) | (lane == 31 && token && after == k ? 2 : 0);
    const bool single = head && tail && goes == 0;
    const uint32_t singles = __ballot_sync(0xffffffffu, single);
    const uint32_t heads = __ballot_sync(0xffffffffu, head && !single), tails = __ballot_sync(0xffffffffu, tail && !single);
    const uint32_t below = (1u << lane) - 1u;
    if (single) s_single[__popc(singles & below)] = lane;
    if (head && !single) s_first[__popc(heads & below)] = lane;
    if (tail && !single) s_last[__popc(tails & below)] = lane + 1;
    const int early = __shfl_sync(0xffffffffu, goes, 0) & 1, late = __shfl_sync(0xffffffffu, goes, 31) & 2;
    const int n = __popc(heads);
    if (lane < n) s_goes[lane] = (lane == 0 ? early : 0) | (lane == n - 1 ? late : 0);
    if (lane == 0) {
      s_counts[0] = __popc(singles);
      s_counts[1] = n;
    }
  }
  __syncthreads();
  // the row's columns are shared by gridDim.z CTAs
  const int all = (p.dim + S::kWide - 1) / S::kWide, block0 = all * (int)blockIdx.z / (int)gridDim.z;
  const int blocks = all * ((int)blockIdx.z + 1) / (int)gridDim.z - block0;
  const TI* dy = (const TI*)p.in + c * p.stride_act;
  TO* grad = (TO*)p.grad + c * p.stride_table;

  // rows with one token: four at a time, their loads first
  const int singles = s_counts[0], quads = (singles + 3) / 4 * blocks;
  int q = 0, block = warp;
  for (int u = warp; u < quads; u += 8, block += 8) {
    for (; block >= blocks; block -= blocks) ++q;
    const int col = (block0 + block) * S::kWide + lane * V, left = p.dim - col;
    Pack<TI, V> x[4][S::Q];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const TI* row = dy + (int64_t)s_pos[s_single[min(4 * q + r, singles - 1)]] * p.ld_act + col;
#pragma unroll
      for (int k = 0; k < S::Q; ++k)
        if (32 * V * k < left) x[r][k].load(row + 32 * V * k);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      if (4 * q + r >= singles) break;
      TO* row = grad + (int64_t)s_key[s_single[4 * q + r]] * p.ld_table + col;
#pragma unroll
      for (int k = 0; k < S::Q; ++k)
        if (32 * V * k < left) {
          Pack<TO, V> y;
          if (p.accumulate) y.load(row + 32 * V * k);
#pragma unroll
          for (int j = 0; j < V; ++j)
            y.t[j] = from_f32<TO>((p.accumulate ? to_f32(y.t[j]) : 0.f) + to_f32(x[r][k].t[j]) * p.scale);
          y.store_stream(row + 32 * V * k);
        }
    }
  }

  // the others: a warp, or several, for a stretch of a segment
  const int segments = s_counts[1], tasks = segments * blocks;
  const int warps = tasks > 4 ? 1 : tasks > 2 ? 2 : tasks > 1 ? 4 : 8;   // per task; several: all tasks at once
  const int s = warp & (warps - 1), stride = 8 / warps;
  q = 0;
  block = warp / warps;
  for (int u0 = 0; u0 < tasks; u0 += stride, block += stride) {
    const int u = u0 + warp / warps;
    for (; block >= blocks; block -= blocks) ++q;
    S share;
    share.clear();
    const int col = (block0 + block) * S::kWide + lane * V, left = p.dim - col;
    if (u < tasks) {
      const int first = s_first[q], n = s_last[q] - first, from = first + n * s / warps, to = first + n * (s + 1) / warps;
      share.template add<TI>(to - from, left, [&](int t) { return dy + (int64_t)s_pos[from + t] * p.ld_act + col; });
    }
    if (warps > 1) share.join(s_sum, warp - s, warps);
    if (u < tasks && s == 0) {
      if (s_goes[q])
        share.to_part(p.part + ((c * p.parts + g) * 2 + (s_goes[q] & 1 ? 0 : 1)) * p.dim + col, left);
      else
        share.to_row(grad + (int64_t)s_key[s_first[q]] * p.ld_table + col, left, p.scale, p.accumulate);
    }
  }
}

// Whether id v has tokens.  The table's entry counts only where the key it points at says so: that of an id without
// tokens holds whatever was in the workspace.
__device__ __forceinline__ bool has_tokens(const EmbArgs& p, int64_t c, int64_t v) {
  const uint32_t at = p.span[c * p.vocab + v].x;
  return (int64_t)at < p.tokens && p.key[c * p.tokens + at] == (uint32_t)v;
}

// Zeros over n elements from p on by a warp: 16 bytes a lane between the first and the last 16-byte boundary.
template <typename T>
__device__ __forceinline__ void zero_run(T* p, uint32_t n) {
  constexpr uint32_t kPer = 16 / sizeof(T);
  const uint32_t lane = threadIdx.x & 31;
  const uint32_t head = min(n, ((16u - ((uint32_t)reinterpret_cast<uintptr_t>(p) & 15u)) & 15u) / (uint32_t)sizeof(T));
  const uint32_t words = (n - head) / kPer, tail = head + words * kPer;
  const T zero = from_f32<T>(0.f);
  if (lane < head) p[lane] = zero;
  uint4* w = reinterpret_cast<uint4*>(p + head) + lane;
  for (uint32_t i = lane; i < words; i += 32, w += 32) __stcs(w, make_uint4(0, 0, 0, 0));
  if (tail + lane < n) p[tail + lane] = zero;
}

// Few tokens (up to kDirectTokens): every CTA looks through all of a client's ids for those of its rows_cta rows, puts
// what it finds in order by row, and writes its rows, zeros and sums.  One launch: at 33 tokens, 256 x 64, 3.6 us against
// 8.2 for a sort, sums and zeros as launches of their own; at 2048 tokens, 50000 x 768, 31 us against 35.
template <typename TI, typename TO, int V>
__global__ void __launch_bounds__(256, 4) embedding_direct_kernel(const EmbArgs p) {
  using S = Share<V>;
  __shared__ float s_sum[8][S::kWide];
  __shared__ uint16_t s_found[kDirectTokens], s_sorted[kDirectTokens];
  __shared__ uint8_t s_of[kDirectTokens];
  __shared__ int s_count[64], s_first[64], s_warp[8];
  __shared__ uint8_t s_rows[64];
  __shared__ int s_some;
  const int64_t c = blockIdx.y, v0 = (int64_t)blockIdx.x * p.rows_cta;
  const int rows = (int)min((int64_t)p.rows_cta, p.vocab - v0);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x < 64) s_count[threadIdx.x] = 0;
  grid_wait();
  grid_trigger();
  __syncthreads();
  // neighbouring tokens to a thread, so that the threads' finds follow one another in the tokens' order
  const int tokens = (int)p.tokens, per = (tokens + 255) / 256, t0 = threadIdx.x * per;
  int row[kDirectTokens / 256], n = 0;
#pragma unroll
  for (int i = 0; i < kDirectTokens / 256; ++i) {
    row[i] = -1;
    if (i < per && t0 + i < tokens) {
      const int64_t r = load_id(p, c, t0 + i) - v0;
      if (r >= 0 && r < rows) {
        row[i] = (int)r;
        ++n;
        atomicAdd(&s_count[r], 1);
      }
    }
  }
  int incl = n;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += v;
  }
  if (lane == 31) s_warp[warp] = incl;
  __syncthreads();
  int at = incl - n, found = 0;
#pragma unroll
  for (int w = 0; w < 8; ++w) {
    at += w < warp ? s_warp[w] : 0;
    found += s_warp[w];
  }
#pragma unroll
  for (int i = 0; i < kDirectTokens / 256; ++i)
    if (row[i] >= 0) {
      s_found[at] = (uint16_t)(t0 + i);
      s_of[at++] = (uint8_t)row[i];
    }
  TO* grad = (TO*)p.grad + c * p.stride_table + v0 * p.ld_table;
  // the columns are shared by gridDim.z CTAs, so that a frequent token's row is not one CTA's work
  const int all_blocks = (p.dim + S::kWide - 1) / S::kWide;
  const int block0 = all_blocks * (int)blockIdx.z / (int)gridDim.z, block1 = all_blocks * ((int)blockIdx.z + 1) / (int)gridDim.z;
  const uint32_t width = (uint32_t)(min(block1 * S::kWide, p.dim) - block0 * S::kWide);
  TO* zeros = grad + block0 * S::kWide;
  if (found == 0) {   // most CTAs of a large table
    if (!p.accumulate)
      for (int r = warp; r < rows; r += 8) zero_run(zeros + (int64_t)r * p.ld_table, width);
    return;
  }
  __syncthreads();
  if (warp == 0) {   // by row, in the tokens' order: two rows' counts a lane, then 32 finds at a time
    const int a = s_count[2 * lane], b = s_count[2 * lane + 1];
    int sum = a + b;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += v;
    }
    s_first[2 * lane] = sum - a - b;
    s_first[2 * lane + 1] = sum - b;
    const uint32_t ma = __ballot_sync(0xffffffffu, a > 0), mb = __ballot_sync(0xffffffffu, b > 0);
    const uint32_t below = (1u << lane) - 1u;
    int k = __popc(ma & below) + __popc(mb & below);   // rows that have tokens
    if (a > 0) s_rows[k++] = (uint8_t)(2 * lane);
    if (b > 0) s_rows[k] = (uint8_t)(2 * lane + 1);
    if (lane == 0) s_some = __popc(ma) + __popc(mb);
    __syncwarp();
    for (int i = 0; i < found; i += 32) {
      const bool live = i + lane < found;
      const uint32_t r = live ? s_of[i + lane] : 0;
      const uint32_t same = same_digit<6>(r) & __ballot_sync(0xffffffffu, live);
      const int to = s_first[r] + __popc(same & below);
      __syncwarp();
      if (live) {
        s_sorted[to] = s_found[i + lane];
        if (lane == __ffs(same) - 1) s_first[r] = to + __popc(same);   // (the first lane's place is the rows' next one)
      }
      __syncwarp();
    }
  } else if (!p.accumulate) {
    for (int r = warp - 1; r < rows; r += 7)
      if (s_count[r] == 0) zero_run(zeros + (int64_t)r * p.ld_table, width);
  }
  __syncthreads();
  // s_first now is where a row's tokens end
  const int some = s_some;
  const TI* dy = (const TI*)p.in + c * p.stride_act;
  int turn = 0;
  for (int k = 0; k < some; ++k) {
    const int r = s_rows[k], m = s_count[r], first = s_first[r] - m;
    TO* out = grad + (int64_t)r * p.ld_table;
    for (int b = block0; b < block1; ++b) {
      const int col = b * S::kWide + lane * V, left = p.dim - col;
      const bool all = m > kManyTokens;   // the whole CTA for a frequent token, else a warp
      if (!all && (turn++ & 7) != warp) continue;
      const int from = all ? m * warp / 8 : 0, to = all ? m * (warp + 1) / 8 : m;
      S share;
      share.clear();
      share.template add<TI>(to - from, left, [&](int t) { return dy + (int64_t)s_sorted[first + from + t] * p.ld_act + col; });
      if (all) share.join(s_sum, 0, 8);
      if (!all || warp == 0) share.to_row(out + col, left, p.scale, p.accumulate);
    }
  }
}

// Bound by HBM's writes: 16 x 50000 x 768 floats in 338 us, 6.7 TB/s.
// The rest of the table's gradient.  The first zero_ctas CTAs of a client write zeros to the rows of ids without tokens,
// rows_cta (up to 64) each.  The others look at 8 groups each for an id whose tokens begin there and go on, and add
// the partial sums of its groups for their share of the columns.
template <typename TO, int V>
__global__ void __launch_bounds__(256, 6) embedding_grad_kernel(const EmbArgs p) {
  using S = Share<V>;
  __shared__ float s_sum[8][S::kWide];
  __shared__ uint32_t s_some[2];
  __shared__ int64_t s_end[8];
  __shared__ uint32_t s_key[8];
  const int64_t c = blockIdx.y;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  TO* grad = (TO*)p.grad + c * p.stride_table;
  grid_wait();
  grid_trigger();
  if (blockIdx.x < p.zero_ctas) {
    const int64_t v0 = (int64_t)blockIdx.x * p.rows_cta;
    const int rows = (int)min((int64_t)p.rows_cta, p.vocab - v0);
    if (warp < 2) {
      const bool some = (int)threadIdx.x < rows && has_tokens(p, c, v0 + threadIdx.x);
      const uint32_t mask = __ballot_sync(0xffffffffu, some);
      if (lane == 0) s_some[warp] = mask;
    }
    __syncthreads();
    const uint64_t some = (uint64_t)s_some[1] << 32 | s_some[0];
    for (int r = warp; r < rows; r += 8)
      if (!(some >> r & 1)) zero_run(grad + (v0 + r) * p.ld_table, (uint32_t)p.dim);
    return;
  }
  const int blocks = (p.dim + S::kWide - 1) / S::kWide;
  const uint32_t u = blockIdx.x - p.zero_ctas, z = u % p.join_split;
  const int64_t g0 = (int64_t)(u / p.join_split) * 8;
  const int first = blocks * (int)z / (int)p.join_split, last = blocks * (int)(z + 1) / (int)p.join_split;
  if (lane == 0) {   // the warp's group: does its last token's id begin in it and go on?
    const int64_t g = g0 + warp, i = g * kPart + kPart - 1;
    const uint32_t* key = p.key + c * p.tokens;
    s_end[warp] = 0;
    if (i + 1 < p.tokens) {
      const uint32_t k = key[i];
      if (k != kNoToken && key[i + 1] == k) {
        const uint2 span = p.span[c * p.vocab + k];
        if (span.x / kPart == g) {
          s_end[warp] = (span.y - 1) / kPart + 1;
          s_key[warp] = k;
        }
      }
    }
  }
  __syncthreads();
  const float* part = p.part + c * p.parts * 2 * p.dim;
  auto take = [&](S& share, int64_t g, int col, int left, int64_t from, int64_t to) {   // the id's groups from .. to - 1
    share.clear();
    share.template add<float>((int)(to - from), left, [&](int t) {
      return part + ((from + t) * 2 + (from + t == g ? 1 : 0)) * p.dim + col;
    });
  };
  int turn = 0;
  for (int w = 0; w < 8; ++w) {
    const int64_t g = g0 + w, n = s_end[w] - g;
    if (s_end[w] == 0) continue;
    TO* row = grad + (int64_t)s_key[w] * p.ld_table;
    for (int b = first; b < last; ++b) {
      const int col = b * S::kWide + lane * V, left = p.dim - col;
      S share;
      if (n <= kManyGroups) {   // a warp for each stretch
        if ((turn++ & 7) != warp) continue;
        take(share, g, col, left, g, g + n);
        share.to_row(row + col, left, p.scale, p.accumulate);
      } else {                  // all of them
        take(share, g, col, left, g + n * warp / 8, g + n * (warp + 1) / 8);
        share.join(s_sum, 0, 8);
        if (warp == 0) share.to_row(row + col, left, p.scale, p.accumulate);
      }
    }
  }
}

}  // namespace brace
