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
constexpr int kSortItems = 4;                // elements per thread of the sort
constexpr int kSortThreads = 512;
constexpr int kSortTile = kSortThreads * kSortItems;   // elements one CTA sorts
constexpr int kDigitBits = 6;
constexpr int kDigits = 1 << kDigitBits;
constexpr int kCountRow = kDigits + 1;
constexpr int kMergeRuns = 16;               // sorted runs merged at a time
constexpr int kPart = 32;                    // sorted tokens of a group: a CTA's share of the sums
constexpr int kManyGroups = 16;              // from here on a whole CTA adds a row's partial sums

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
                          // are written, what else is there is told by the keys (see span_of)
  float* part;            // [clients][parts][2][dim]: of each group of kPart sorted tokens, the sums of the first id
                          // if its tokens began in an earlier group, and of the last one if they only go on in the next
  int64_t parts;
  int rows_cta;
};

__device__ __forceinline__ int64_t load_id(const EmbArgs& p, int64_t c, int64_t t) {
  return p.id_bytes == 8 ? ((const int64_t*)p.ids)[c * p.stride_ids + t]
                         : (int64_t)((const int32_t*)p.ids)[c * p.stride_ids + t];
}

// ---- lookup -----------------------------------------------------------------------------------------------------
// A warp takes kLookupRows rows and of each a stretch of 32 V Q columns, all loads first.  Rows that do not start on
// whole words are read and written element by element, 32 neighbours at a time.
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
// One CTA sorts up to a tile of consecutive tokens of a client by id: least significant digit first, 6 bits at a
// time.  A warp holds 32 * ITEMS consecutive elements; equal digits within 32 are ranked by ballots, across the warp's
// rounds by a counter per (digit, warp), across warps by a scan of the counters.
template <int ITEMS>
__global__ void __launch_bounds__(1024) embedding_sort_kernel(const EmbArgs p, int tile, int bits) {
  extern __shared__ uint32_t sort_smem[];
  uint32_t* s_key = sort_smem;                                   // [tile]
  uint32_t* s_pos = s_key + tile;                                // [tile]
  uint32_t* s_count = s_pos + tile;                              // [warps][kDigits + 1]: a warp's digits in different banks
  __shared__ uint32_t s_warp[32];
  grid_wait();
  grid_trigger();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
  const int64_t c = blockIdx.y, first = (int64_t)blockIdx.x * tile;
  const int n = (int)min((int64_t)tile, p.tokens - first);
  uint32_t key[ITEMS], pos[ITEMS];
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const int k = (warp * ITEMS + i) * 32 + lane;
    key[i] = kNoToken;
    pos[i] = (uint32_t)(first + k);
    if (k < n) {
      const int64_t id = load_id(p, c, first + k);
      if (id >= 0 && id < p.vocab) key[i] = (uint32_t)id;
    }
  }
  for (int shift = 0; shift < bits; shift += kDigitBits) {
    for (int i = tid; i < kCountRow * warps; i += blockDim.x) s_count[i] = 0;
    __syncthreads();
    uint32_t rank[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const uint32_t digit = (key[i] >> shift) & (kDigits - 1);
      // the lanes with this lane's digit, bit by bit (a match instruction takes several times as long)
      uint32_t same = 0xffffffffu;
#pragma unroll
      for (int b = 0; b < kDigitBits; ++b) {
        const bool set = (digit >> b) & 1u;
        const uint32_t with = __ballot_sync(0xffffffffu, set);
        same &= set ? with : ~with;
      }
      const uint32_t before = s_count[warp * kCountRow + digit];
      rank[i] = before + __popc(same & ((1u << lane) - 1u));
      __syncwarp();
      if (lane == __ffs(same) - 1) s_count[warp * kCountRow + digit] = before + __popc(same);
      __syncwarp();
    }
    __syncthreads();
    // exclusive scan of the counters in (digit, warp) order: each thread takes two neighbours
    constexpr int kPer = kDigits / 32;
    uint32_t own[kPer], sum = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int k = tid * kPer + i;
      own[i] = s_count[k % warps * kCountRow + k / warps];
      sum += own[i];
    }
    uint32_t incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t v = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += v;
    }
    if (lane == 31) s_warp[warp] = incl;
    __syncthreads();
    uint32_t offset = lane < warp ? s_warp[lane] : 0;
#pragma unroll
    for (int o = 16; o; o >>= 1) offset += __shfl_xor_sync(0xffffffffu, offset, o);
    uint32_t run = offset + incl - sum;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int k = tid * kPer + i;
      s_count[k % warps * kCountRow + k / warps] = run;
      run += own[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const uint32_t digit = (key[i] >> shift) & (kDigits - 1);
      const uint32_t to = s_count[warp * kCountRow + digit] + rank[i];
      s_key[to] = key[i];
      s_pos[to] = pos[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int k = (warp * ITEMS + i) * 32 + lane;
      key[i] = s_key[k];
      pos[i] = s_pos[k];
    }
    __syncthreads();
  }
  // what is no token was given the largest key and comes last, after the padding of the tile in its turn
  uint32_t* out_key = p.key + c * p.tokens + first;
  uint32_t* out_pos = p.pos + c * p.tokens + first;
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const int k = (warp * ITEMS + i) * 32 + lane;
    if (k < n) {
      out_key[k] = key[i];
      out_pos[k] = pos[i];
    }
  }
}

// Merges groups of RUNS sorted runs of `run` elements: an element's place is its own index plus the number of elements
// in front of it in each other run, found by searches that all runs make in step.
template <int RUNS>
__global__ void __launch_bounds__(256) embedding_merge_kernel(const EmbArgs p, int run, uint32_t* out_key, uint32_t* out_pos) {
  grid_wait();
  grid_trigger();
  const int64_t c = blockIdx.y;
  const uint32_t i = blockIdx.x * 256u + threadIdx.x, n = (uint32_t)p.tokens;
  if (i >= n) return;
  const uint32_t* key = p.key + c * p.tokens;
  const uint32_t k = key[i], group = (uint32_t)(i / ((uint64_t)run * RUNS) * ((uint64_t)run * RUNS));
  const uint32_t mine = (i - group) / (uint32_t)run;
  uint32_t lo[RUNS], len[RUNS];
#pragma unroll
  for (uint32_t r = 0; r < RUNS; ++r) {
    const uint64_t start = (uint64_t)group + (uint64_t)r * run;
    lo[r] = (uint32_t)start;                       // the number in front is between lo - start and lo - start + len
    len[r] = r == mine || start >= n ? 0 : min((uint32_t)run, n - (uint32_t)start);
  }
  for (uint32_t left = (uint32_t)run; left > 0; left >>= 1) {
    uint32_t v[RUNS];
#pragma unroll
    for (uint32_t r = 0; r < RUNS; ++r) v[r] = len[r] > 0 ? key[lo[r] + (len[r] >> 1)] : 0;
#pragma unroll
    for (uint32_t r = 0; r < RUNS; ++r) {
      const uint32_t half = len[r] >> 1;
      const bool front = len[r] > 0 && (v[r] < k || (v[r] == k && r < mine));
      lo[r] += front ? half + 1 : 0;
      len[r] = front ? len[r] - half - 1 : half;
    }
  }
  uint32_t to = group + (i - group - mine * (uint32_t)run);
#pragma unroll
  for (uint32_t r = 0; r < RUNS; ++r) to += r == mine ? 0 : lo[r] - (uint32_t)((uint64_t)group + (uint64_t)r * run);
  out_key[c * p.tokens + to] = k;
  out_pos[c * p.tokens + to] = p.pos[c * p.tokens + i];
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
  // Adds `n` rows at(0) .. at(n - 1), two at a time; `left`: elements of the row from the lane's first one on.
  template <typename T, typename At>
  __device__ __forceinline__ void add(int n, int left, At at) {
#pragma unroll 1
    for (int i = 0; i < n; i += 2) {
      Pack<T, V> x[2][Q];
      const bool two = i + 1 < n;
      const T *p0 = at(i), *p1 = two ? at(i + 1) : p0;
#pragma unroll
      for (int q = 0; q < Q; ++q)
        if (32 * V * q < left) {
          x[0][q].load(p0 + 32 * V * q);
          if (two) x[1][q].load(p1 + 32 * V * q);
        }
#pragma unroll
      for (int q = 0; q < Q; ++q)
        if (32 * V * q < left)
#pragma unroll
          for (int j = 0; j < V; ++j) {
            sum[q][j] += to_f32(x[0][q].t[j]);
            if (two) sum[q][j] += to_f32(x[1][q].t[j]);
          }
    }
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
        if (accumulate) y.load_plain(p + 32 * V * q);
#pragma unroll
        for (int j = 0; j < V; ++j) y.t[j] = from_f32<TO>((accumulate ? to_f32(y.t[j]) : 0.f) + sum[q][j] * scale);
        y.store_stream(p + 32 * V * q);
      }
  }
};

// A CTA takes a group of kPart sorted tokens: notes where each id's tokens begin and end, writes the rows of the ids
// whose tokens all lie in the group, and leaves a partial sum of an id that goes on before ([0]) or only after ([1]).
template <typename TI, typename TO, int V>
__global__ void __launch_bounds__(256, 6) embedding_sum_kernel(const EmbArgs p) {
  static_assert(kPart == 32, "a lane per token of a group");
  using S = Share<V>;
  __shared__ float s_sum[8][S::kWide];
  __shared__ uint32_t s_key[32], s_pos[32];
  __shared__ int s_first[33], s_segments, s_goes;
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
    const bool token = k != kNoToken;
    if (token) {   // (every CTA of a group writes the same)
      if (before != k) p.span[c * p.vocab + k].x = (uint32_t)i;
      if (after != k) p.span[c * p.vocab + k].y = (uint32_t)i + 1;
      s_key[lane] = k;
      s_pos[lane] = p.pos[c * p.tokens + i];
    }
    const uint32_t heads = __ballot_sync(0xffffffffu, token && (lane == 0 || before != k));
    const int tokens = __popc(__ballot_sync(0xffffffffu, token));
    if (token && (heads >> lane & 1u)) s_first[__popc(heads & ((1u << lane) - 1u))] = lane;
    const bool early = __shfl_sync(0xffffffffu, token && before == k, 0), late = __shfl_sync(0xffffffffu, token && after == k, 31);
    if (lane == 0) {
      s_segments = __popc(heads);
      s_first[__popc(heads)] = tokens;
      s_goes = (early ? 1 : 0) | (late ? 2 : 0);
    }
  }
  __syncthreads();
  const int segments = s_segments, goes = s_goes;
  // the row's columns are shared by gridDim.z CTAs
  const int all = (p.dim + S::kWide - 1) / S::kWide, block0 = all * (int)blockIdx.z / (int)gridDim.z;
  const int blocks = all * ((int)blockIdx.z + 1) / (int)gridDim.z - block0, tasks = segments * blocks;
  const int warps = tasks > 4 ? 1 : tasks > 2 ? 2 : tasks > 1 ? 4 : 8;   // per task; several: all tasks at once
  const TI* dy = (const TI*)p.in + c * p.stride_act;
  const int s = warp & (warps - 1), stride = 8 / warps;
  int q = 0, block = warp / warps;   // this warp's task: a segment and a stretch of its columns
  for (int u0 = 0; u0 < tasks; u0 += stride, block += stride) {
    const int u = u0 + warp / warps;
    for (; block >= blocks; block -= blocks) ++q;
    S share;
    share.clear();
    const int col = (block0 + block) * S::kWide + lane * V, left = p.dim - col;
    if (u < tasks) {
      const int first = s_first[q], n = s_first[q + 1] - first, from = first + n * s / warps, to = first + n * (s + 1) / warps;
      share.template add<TI>(to - from, left, [&](int t) { return dy + (int64_t)s_pos[from + t] * p.ld_act + col; });
    }
    if (warps > 1) share.join(s_sum, warp - s, warps);
    if (u < tasks && s == 0) {
      const bool early = q == 0 && (goes & 1), late = q + 1 == segments && (goes & 2);
      if (early || late)
        share.to_part(p.part + ((c * p.parts + g) * 2 + (early ? 0 : 1)) * p.dim + col, left);
      else
        share.to_row((TO*)p.grad + c * p.stride_table + (int64_t)s_key[s_first[q]] * p.ld_table + col, left, p.scale, p.accumulate);
    }
  }
}

// The sorted tokens of id v.  The table's entry counts only where the key it points at says so: that of an id without
// tokens holds whatever was in the workspace.
__device__ __forceinline__ uint2 span_of(const EmbArgs& p, int64_t c, int64_t v) {
  if (p.tokens == 0) return make_uint2(0, 0);
  const uint2 s = p.span[c * p.vocab + v];
  const uint32_t* key = p.key + c * p.tokens;
  if ((int64_t)s.x >= p.tokens || key[s.x] != (uint32_t)v) return make_uint2(0, 0);
  return s;
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

// The other rows of the table's gradient, rows_cta (up to 64) a CTA: zeros where an id has no tokens, and the sums of
// the partial sums of the ids whose tokens lie in several groups.
template <typename TO, int V>
__global__ void __launch_bounds__(256, 6) embedding_grad_kernel(const EmbArgs p) {
  using S = Share<V>;
  __shared__ float s_sum[8][S::kWide];
  __shared__ uint32_t s_start[64], s_end[64];
  __shared__ int s_row[64], s_rows[2];
  __shared__ uint32_t s_some[2];
  const int64_t c = blockIdx.y, v0 = (int64_t)blockIdx.x * p.rows_cta;
  const int rows = (int)min((int64_t)p.rows_cta, p.vocab - v0);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  grid_wait();
  grid_trigger();
  uint2 span = make_uint2(0, 0);
  if ((int)threadIdx.x < rows) span = span_of(p, c, v0 + threadIdx.x);
  if (warp < 2) {
    const bool wide = span.x < span.y && span.x / kPart != (span.y - 1) / kPart;
    const uint32_t has = __ballot_sync(0xffffffffu, wide), some = __ballot_sync(0xffffffffu, span.x < span.y);
    if (lane == 0) s_some[warp] = some;
    s_start[threadIdx.x] = span.x;
    s_end[threadIdx.x] = span.y;
    if (lane == 0) s_rows[warp] = __popc(has);
    // the rows of several groups in order, those of the second warp from 32 on
    if (wide) s_row[warp * 32 + __popc(has & ((1u << lane) - 1u))] = threadIdx.x;
  }
  __syncthreads();
  TO* grad = (TO*)p.grad + c * p.stride_table + v0 * p.ld_table;
  if (!p.accumulate) {
    // the rows without tokens
    uint64_t none = ~((uint64_t)s_some[1] << 32 | s_some[0]);
    for (int r = warp; r < rows; r += 8)
      if (none >> r & 1) zero_run(grad + (int64_t)r * p.ld_table, (uint32_t)p.dim);
  }
  const int blocks = (p.dim + S::kWide - 1) / S::kWide, first = s_rows[0], full = first + s_rows[1];
  const float* part = p.part + c * p.parts * 2 * p.dim;
  auto take = [&](S& share, int r, int col, int left, int64_t from, int64_t to) {   // groups from .. to - 1 of the row's
    share.clear();
    const int64_t g0 = s_start[r] / kPart;
    share.template add<float>((int)(to - from), left, [&](int t) {
      const int64_t g = from + t;
      return part + (g * 2 + (g == g0 ? 1 : 0)) * p.dim + col;
    });
  };
  for (int u = warp; u < full * blocks; u += 8) {   // a warp for each part of a row of few groups
    const int k = u / blocks, r = s_row[k < first ? k : 32 + k - first];
    const int64_t g0 = s_start[r] / kPart, g1 = (s_end[r] - 1) / kPart + 1;
    if (g1 - g0 > kManyGroups) continue;
    const int col = (u - k * blocks) * S::kWide + lane * V, left = p.dim - col;
    S share;
    take(share, r, col, left, g0, g1);
    share.to_row(grad + (int64_t)r * p.ld_table + col, left, p.scale, p.accumulate);
  }
  for (int k = 0; k < full; ++k) {                  // the CTA together for one of many
    const int r = s_row[k < first ? k : 32 + k - first];
    const int64_t g0 = s_start[r] / kPart, g1 = (s_end[r] - 1) / kPart + 1, n = g1 - g0;
    if (n <= kManyGroups) continue;
    for (int b = 0; b < blocks; ++b) {
      const int col = b * S::kWide + lane * V, left = p.dim - col;
      S share;
      take(share, r, col, left, g0 + n * warp / 8, g0 + n * (warp + 1) / 8);
      share.join(s_sum, 0, 8);
      if (warp == 0) share.to_row(grad + (int64_t)r * p.ld_table + col, left, p.scale, p.accumulate);
    }
  }
}

}  // namespace brace
