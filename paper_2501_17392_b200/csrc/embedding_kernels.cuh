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
constexpr int kSortItems = 8;                // elements per thread of the sort
constexpr int kSortTile = 1024 * kSortItems; // elements one CTA sorts
constexpr int kDigitBits = 6;
constexpr int kDigits = 1 << kDigitBits;
constexpr int kMergeRuns = 16;               // sorted runs merged at a time
constexpr int kPart = 32;                    // sorted tokens per partial sum

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
  float* part;            // [clients][parts][dim]: sums of aligned groups of kPart sorted tokens with one id
  int64_t parts;
  int rows_cta;
};

__device__ __forceinline__ int64_t load_id(const EmbArgs& p, int64_t c, int64_t t) {
  return p.id_bytes == 8 ? ((const int64_t*)p.ids)[c * p.stride_ids + t]
                         : (int64_t)((const int32_t*)p.ids)[c * p.stride_ids + t];
}

// ---- lookup -----------------------------------------------------------------------------------------------------
// A thread moves U groups of V elements, so that the loads of U rows are under way together.
template <typename TI, typename TO, int V, int U>
__global__ void __launch_bounds__(256) embedding_lookup_kernel(const EmbArgs p) {
  grid_wait();
  grid_trigger();
  const uint32_t groups = (uint32_t)(p.dim / V);
  const int64_t c = blockIdx.y;
  const uint64_t total = (uint64_t)p.tokens * groups;
  uint64_t u = (uint64_t)blockIdx.x * (256 * U) + threadIdx.x;
  Pack<TI, V> x[U];
  bool live[U], hit[U];
  TO* to[U];
#pragma unroll
  for (int i = 0; i < U; ++i, u += 256) {
    live[i] = u < total;
    hit[i] = false;
    if (live[i]) {
      const int64_t t = (int64_t)(total >> 32 ? u / groups : (uint32_t)u / groups);
      const int col = (int)(u - (uint64_t)t * groups) * V;
      const int64_t id = load_id(p, c, t);
      to[i] = (TO*)p.out + c * p.stride_act + t * p.ld_act + col;
      hit[i] = id >= 0 && id < p.vocab;
      if (hit[i]) x[i].load((const TI*)p.table + c * p.stride_table + id * p.ld_table + col);
    }
  }
#pragma unroll
  for (int i = 0; i < U; ++i)
    if (live[i]) {
      Pack<TO, V> y;
#pragma unroll
      for (int j = 0; j < V; ++j) y.t[j] = from_f32<TO>(hit[i] ? to_f32(x[i].t[j]) * p.scale : 0.f);
      y.store_stream(to[i]);
    }
}

// ---- gradient: sort ---------------------------------------------------------------------------------------------
// One CTA sorts up to 1024 * ITEMS consecutive tokens of a client by id: least significant digit first, 6 bits at a
// time.  A warp holds 32 * ITEMS consecutive elements; equal digits within 32 are ranked by a match, across the warp's
// rounds by a counter per (digit, warp), across warps by a scan of the counters.
template <int ITEMS>
__global__ void __launch_bounds__(1024) embedding_sort_kernel(const EmbArgs p, int tile, int bits) {
  extern __shared__ uint32_t sort_smem[];
  uint32_t* s_key = sort_smem;                                   // [tile]
  uint32_t* s_pos = s_key + tile;                                // [tile]
  uint32_t* s_count = s_pos + tile;                              // [kDigits][warps]
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
    for (int i = tid; i < kDigits * warps; i += blockDim.x) s_count[i] = 0;
    __syncthreads();
    uint32_t rank[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const uint32_t digit = (key[i] >> shift) & (kDigits - 1);
      const uint32_t same = __match_any_sync(0xffffffffu, digit);
      const uint32_t before = s_count[digit * warps + warp];
      rank[i] = before + __popc(same & ((1u << lane) - 1u));
      __syncwarp();
      if (lane == __ffs(same) - 1) s_count[digit * warps + warp] = before + __popc(same);
      __syncwarp();
    }
    __syncthreads();
    // exclusive scan of the counters in (digit, warp) order: each thread takes `per` neighbours
    const int counters = kDigits * warps, per = (counters + blockDim.x - 1) / blockDim.x;
    uint32_t sum = 0;
    for (int i = 0; i < per; ++i) {
      const int k = tid * per + i;
      if (k < counters) sum += s_count[k];
    }
    uint32_t incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t v = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += v;
    }
    if (lane == 31) s_warp[warp] = incl;
    __syncthreads();
    uint32_t offset = 0;
    for (int w = 0; w < warp; ++w) offset += s_warp[w];
    uint32_t run = offset + incl - sum;
    for (int i = 0; i < per; ++i) {
      const int k = tid * per + i;
      if (k < counters) {
        const uint32_t v = s_count[k];
        s_count[k] = run;
        run += v;
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const uint32_t digit = (key[i] >> shift) & (kDigits - 1);
      const uint32_t to = s_count[digit * warps + warp] + rank[i];
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

// Merges groups of kMergeRuns sorted runs of `run` elements: an element's place is its own index plus the number of
// elements in front of it in each other run, found by searches that all runs make in step.
__global__ void __launch_bounds__(256) embedding_merge_kernel(const EmbArgs p, int64_t run, uint32_t* out_key, uint32_t* out_pos) {
  grid_wait();
  grid_trigger();
  const int64_t c = blockIdx.y, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= p.tokens) return;
  const uint32_t* key = p.key + c * p.tokens;
  const uint32_t k = key[i];
  const int64_t group = i / (run * kMergeRuns) * (run * kMergeRuns);
  const int mine = (int)((i - group) / run);
  int64_t lo[kMergeRuns], len[kMergeRuns];
#pragma unroll
  for (int r = 0; r < kMergeRuns; ++r) {
    const int64_t start = group + r * run;
    lo[r] = 0;
    len[r] = r == mine ? 0 : max((int64_t)0, min(run, p.tokens - start));
  }
  for (int64_t left = run; left > 0; left >>= 1) {
#pragma unroll
    for (int r = 0; r < kMergeRuns; ++r) {
      // the number in front lies in [lo, lo + len]
      if (len[r] > 0) {
        const int64_t half = len[r] >> 1;
        const uint32_t v = key[group + r * run + lo[r] + half];
        const bool front = v < k || (v == k && r < mine);
        lo[r] += front ? half + 1 : 0;
        len[r] = front ? len[r] - half - 1 : half;
      }
    }
  }
  int64_t to = group + (i - group - mine * run);
#pragma unroll
  for (int r = 0; r < kMergeRuns; ++r) to += lo[r];
  out_key[c * p.tokens + to] = k;
  out_pos[c * p.tokens + to] = p.pos[c * p.tokens + i];
}

// ---- gradient: sums ---------------------------------------------------------------------------------------------
// Sums of the aligned groups of kPart sorted tokens that have one id, so that the row of a frequent token is not one
// CTA's work.
template <typename TI, int V>
__global__ void __launch_bounds__(128) embedding_part_kernel(const EmbArgs p) {
  grid_wait();
  grid_trigger();
  const int64_t c = blockIdx.z, g = blockIdx.x, first = g * kPart;
  if (first + kPart > p.tokens) return;
  const uint32_t* key = p.key + c * p.tokens + first;
  const uint32_t k = key[0];
  if (k == kNoToken || k != key[kPart - 1]) return;
  const int col = (int)(blockIdx.y * 128 + threadIdx.x) * V;
  if (col >= p.dim) return;
  const uint32_t* pos = p.pos + c * p.tokens + first;
  const TI* dy = (const TI*)p.in + c * p.stride_act + col;
  float sum[V];
#pragma unroll
  for (int j = 0; j < V; ++j) sum[j] = 0.f;
#pragma unroll 1
  for (int i = 0; i < kPart; i += 8) {
    Pack<TI, V> x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j].load(dy + (int64_t)pos[i + j] * p.ld_act);
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int e = 0; e < V; ++e) sum[e] += to_f32(x[j].t[e]);
  }
  float* part = p.part + (c * p.parts + g) * p.dim + col;
#pragma unroll
  for (int j = 0; j < V; ++j) part[j] = sum[j];
}

// Number of the n sorted keys that are below `k`, found by a whole warp: 32 probes at a time.
__device__ __forceinline__ int64_t warp_lower_bound(const uint32_t* key, int64_t n, uint32_t k) {
  const int lane = threadIdx.x & 31;
  int64_t lo = 0, len = n;   // the answer lies in [lo, lo + len]
  while (len > 0) {
    const int64_t step = (len + 31) / 32;
    const int64_t at = lo + (int64_t)(lane + 1) * step - 1;   // last element of this lane's share
    const bool below = at < lo + len && key[at] < k;
    const int full = __popc(__ballot_sync(0xffffffffu, below));
    const int64_t end = lo + len;
    lo += full * step;
    len = min(step - 1, end - lo);
    if (len < 0) len = 0;
  }
  return lo;
}

// The table's gradient: a CTA writes rows_cta rows.  V elements per thread at a time.
template <typename TI, typename TO, int V>
__global__ void __launch_bounds__(256) embedding_grad_kernel(const EmbArgs p) {
  __shared__ int64_t s_bound[2];
  __shared__ int s_start[64], s_end[64];   // of each row, counted from s_bound[0]
  const int64_t c = blockIdx.y, v0 = (int64_t)blockIdx.x * p.rows_cta;
  const int rows = (int)min((int64_t)p.rows_cta, p.vocab - v0);
  const int warp = threadIdx.x >> 5;
  if (threadIdx.x < 64) s_start[threadIdx.x] = s_end[threadIdx.x] = 0;
  grid_wait();
  grid_trigger();
  const uint32_t* key = p.key + c * p.tokens;
  const uint32_t* pos = p.pos + c * p.tokens;
  if (warp < 2) {
    const int64_t b = warp_lower_bound(key, p.tokens, (uint32_t)(v0 + (warp ? rows : 0)));
    if ((threadIdx.x & 31) == 0) s_bound[warp] = b;
  }
  __syncthreads();
  const int64_t base = s_bound[0];
  const int n = (int)(s_bound[1] - base);
  if (n <= 8 * 256) {
    for (int i = threadIdx.x; i < n; i += 256) {
      const uint32_t k = key[base + i];
      if (i == 0 || key[base + i - 1] != k) s_start[k - (uint32_t)v0] = i;
      if (i == n - 1 || key[base + i + 1] != k) s_end[k - (uint32_t)v0] = i + 1;
    }
  } else {   // a frequent token: its entries are not walked, the rows' ends are searched
    for (int r = warp; r < rows; r += 8) {
      const int end = (int)warp_lower_bound(key + base, n, (uint32_t)(v0 + r + 1));
      if ((threadIdx.x & 31) == 0) {
        s_end[r] = end;
        if (r + 1 < rows) s_start[r + 1] = end;
      }
    }
  }
  __syncthreads();
  const int groups = p.dim / V;
  TO* grad = (TO*)p.grad + c * p.stride_table + v0 * p.ld_table;
  for (int u = threadIdx.x; u < rows * groups; u += 256) {
    const int r = u / groups, col = (u - r * groups) * V;
    TO* to = grad + (int64_t)r * p.ld_table + col;
    int64_t i = base + s_start[r];
    const int64_t end = base + s_end[r];
    Pack<TO, V> y;
    if (i == end) {
      if (p.accumulate) continue;
#pragma unroll
      for (int j = 0; j < V; ++j) y.t[j] = from_f32<TO>(0.f);
    } else {
      const TI* dy = (const TI*)p.in + c * p.stride_act + col;
      float sum[V];
#pragma unroll
      for (int j = 0; j < V; ++j) sum[j] = 0.f;
      while (i < end) {
        if (i % kPart == 0 && i + kPart <= end) {
          const float* part = p.part + (c * p.parts + i / kPart) * p.dim + col;
#pragma unroll
          for (int j = 0; j < V; ++j) sum[j] += part[j];
          i += kPart;
        } else {
          Pack<TI, V> x;
          x.load(dy + (int64_t)pos[i] * p.ld_act);
#pragma unroll
          for (int j = 0; j < V; ++j) sum[j] += to_f32(x.t[j]);
          ++i;
        }
      }
      if (p.accumulate) {
        y.load_plain(to);
#pragma unroll
        for (int j = 0; j < V; ++j) y.t[j] = from_f32<TO>(to_f32(y.t[j]) + sum[j] * p.scale);
      } else {
#pragma unroll
        for (int j = 0; j < V; ++j) y.t[j] = from_f32<TO>(sum[j] * p.scale);
      }
    }
    y.store_stream(to);
  }
}

}  // namespace brace
