// Windowed attention on the tensor cores: bfloat16 and float16, head dimensions up to 128 in tiles of 64 or 128.
// Formulas and the treatment of single rows are in attention_rows.cuh.
//
// Forward.  A CTA has two groups of 128 queries -- two heads that share their keys, or two neighbouring stretches of one
// head -- and walks the blocks of 128 keys that either of them sees: the first tokens', then the window's.  Per block and
// group: scores S = Q K^T into tensor memory; a thread takes a query's 128 scores into registers, masks them, brings its
// running maximum up to date and writes exp2 of the differences, rounded to the inputs' type, back over S; P V is added to
// the group's result in tensor memory.  While one group's threads are at their exponentials, the tensor cores work for the
// other.  The result is scaled again only when a maximum has grown by more than 2^8 (the sum and P have room for that).
//
// A product with P = 0 where a key is hidden gives NaN if that key's value is not finite.  A row whose result is not
// finite is therefore computed again, key by key, from what it sees.
#pragma once

#include <type_traits>

#include "attention_rows.cuh"

namespace brace {

constexpr int kAttnThreads = 320;          // two groups of four warps, a warp that loads, a warp that issues products
constexpr int kKeys = 128;                 // of a block
constexpr float kGrown = 8.f;              // log2 of what a maximum may grow by before the result is scaled again

template <int D>
struct AttnShape {
  static constexpr int kTile = 128 * D * 2;                // bytes of 128 rows: D / 64 blocks of 64 columns
  static constexpr int kStages = D == 64 ? 6 : 4;
  static constexpr int kSmem = 1024 + (2 + kStages) * kTile + 256;
};

struct AttnMaps {
  CUtensorMap q, k, v, dout;               // (dimension, token, head, sequence)
};

// Both operands bfloat16 (format 1) or both float16 (format 0).
template <typename T>
__device__ __forceinline__ constexpr uint32_t attn_idesc(int n, bool b_mn) {
  return f16_idesc(128, n, false, b_mn) | (std::is_same<T, __nv_bfloat16>::value ? (1u << 7) | (1u << 10) : 0u);
}

template <typename T>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  uint32_t r;
  if (std::is_same<T, __nv_bfloat16>::value)
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  else
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

__device__ __forceinline__ float exp2_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// ROWS rows of a head from token `t` on: D / 64 boxes of 64 columns.
template <int D, int ROWS>
__device__ __forceinline__ void load_rows(uint32_t dst, const CUtensorMap* map, int t, int head, int b, uint32_t bar) {
#pragma unroll
  for (int x = 0; x < D / 64; ++x) tma_load<1>(dst + x * ROWS * 128, map, 64 * x, t, head, b, bar);
}

// dst[0..dim) = v * factor, 32 columns from `col` on, of one row.
template <typename T>
__device__ __forceinline__ void put_columns(T* row, const float (&v)[32], float factor, int col, int dim) {
#pragma unroll
  for (int i = 0; i < 32; i += 8) {
    if (col + i >= dim) break;              // dim is a multiple of 8
    uint4 w;
    w.x = pack2<T>(v[i] * factor, v[i + 1] * factor);
    w.y = pack2<T>(v[i + 2] * factor, v[i + 3] * factor);
    w.z = pack2<T>(v[i + 4] * factor, v[i + 5] * factor);
    w.w = pack2<T>(v[i + 6] * factor, v[i + 7] * factor);
    *reinterpret_cast<uint4*>(row + col + i) = w;
  }
}
template <typename T>
__device__ __forceinline__ void put_zeros(T* row, int dim) {
  for (int i = 0; i < dim; i += 8) *reinterpret_cast<uint4*>(row + i) = make_uint4(0, 0, 0, 0);
}

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

// grid: (pairs of groups, heads or pairs of heads, sequences)
template <typename T, int D, bool SHARED>
__global__ void __launch_bounds__(kAttnThreads, 1) attn_forward_kernel(const __grid_constant__ AttnMaps maps, const AttnArgs p) {
  using Shape = AttnShape<D>;
  constexpr int STAGES = Shape::kStages;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_addr(smem_raw) + 1023u) & ~1023u;
  const uint32_t ring = base + 2 * Shape::kTile, bars = ring + STAGES * Shape::kTile;
  const uint32_t full = bars, empty = full + 8 * STAGES, q_full = empty + 8 * STAGES;
  const uint32_t s_full = q_full + 8, p_full = s_full + 16, o_full = p_full + 16, tail = o_full + 16;
  volatile int* dead = (volatile int*)(smem_raw + (tail - smem_addr(smem_raw)));
  uint32_t* tmem_slot = (uint32_t*)(smem_raw + (tail + 8 - smem_addr(smem_raw)));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    *dead = 0;
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(full + 8 * s, 1);
      mbar_init(empty + 8 * s, 1);
    }
    mbar_init(q_full, 1);
    for (int r = 0; r < 2; ++r) {
      mbar_init(s_full + 8 * r, 1);
      mbar_init(p_full + 8 * r, 4);
      mbar_init(o_full + 8 * r, 1);
    }
    mbar_init_visible();
    tma_prefetch(&maps.q);
    tma_prefetch(&maps.k);
    tma_prefetch(&maps.v);
  }
  if (warp == 9) tmem_alloc<1>(smem_addr(tmem_slot), 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  grid_trigger();
  grid_wait();
  fence_async_global();

  // the last queries first: they have the longest windows
  const int b = blockIdx.z, pair = gridDim.x - 1 - blockIdx.x, n = attn_length(p, b);
  const int q0 = SHARED ? pair * 128 : pair * 256, h0 = SHARED ? 2 * (int)blockIdx.y : (int)blockIdx.y, g = h0 / p.share;
  auto group_query = [&](int r) { return SHARED ? q0 : q0 + 128 * r; };
  auto group_head = [&](int r) { return SHARED ? h0 + r : h0; };
  const int groups = q0 >= n ? 0 : SHARED || q0 + 128 < n ? 2 : 1;
  const KeyBlocks blocks(p, q0, min(n, q0 + (SHARED ? 128 : 256)), kKeys);
  const int count = groups ? blocks.count : 0;
  // whether a query of group r sees a key of block k
  auto active = [&](int r, int k) {
    if (r >= groups || k >= count) return false;
    if (SHARED || k < blocks.nfirst) return true;
    const int j = blocks.key(k, kKeys), q = group_query(r);
    return j <= q + 127 && (q - p.window + 1 < j + kKeys || j < p.sinks);
  };

  if (warp == 8) {                         // loads
    const bool lead = elect_one();
    if (lead && groups) {
      mbar_expect_tx(q_full, groups * Shape::kTile);
      for (int r = 0; r < groups; ++r)
        load_rows<D, 128>(base + r * Shape::kTile, &maps.q, group_query(r), group_head(r), b, q_full);
    }
    __syncwarp();
    int s = 0, issued = 0;
    uint32_t ph = 0;
    bool ok = true;
    for (int i = 0; ok && i < 2 * count; ++i) {
      if (!mbar_wait(empty + 8 * s, ph ^ 1u, dead)) {
        ok = false;
        break;
      }
      if (lead) {
        mbar_expect_tx(full + 8 * s, Shape::kTile);
        load_rows<D, 128>(ring + s * Shape::kTile, i & 1 ? &maps.v : &maps.k, blocks.key(i >> 1, kKeys), g, b, full + 8 * s);
      }
      __syncwarp();
      ++issued;
      if (++s == STAGES) {
        s = 0;
        ph ^= 1u;
      }
    }
    if (!ok)     // gave up: let the copies in flight land before the memory goes
      for (int i = issued > STAGES ? issued - STAGES : 0; i < issued; ++i)
        mbar_wait(full + 8 * (i % STAGES), (uint32_t)(i / STAGES) & 1u, dead);
  } else if (warp == 9) {                  // products
    const bool lead = elect_one();
    constexpr uint32_t kScores = attn_idesc<T>(kKeys, false), kValues = attn_idesc<T>(D, true);
    const uint64_t q_desc = operand_desc(base, 16384), ring_desc = operand_desc(ring, 16384);
    bool ok = count == 0 || mbar_wait(q_full, 0, dead);
    uint32_t p_phase = 0;
    bool begun[2] = {false, false};
    for (int k = -1; ok && k < count; ++k) {
      // stage of block k's keys: 2 k; of its values: 2 k + 1
      const int sk = (2 * k + 2) % STAGES, sv = (2 * k + 1 + STAGES) % STAGES;
      if (k >= 0 && !mbar_wait(full + 8 * sv, (uint32_t)((2 * k + 1) / STAGES) & 1u, dead)) break;
      if (k + 1 < count && !mbar_wait(full + 8 * sk, (uint32_t)((2 * k + 2) / STAGES) & 1u, dead)) break;
      tc_fence_after();
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const uint32_t scores = tmem + 128 * r, result = tmem + 256 + D * r;
        const bool now = k >= 0 && active(r, k), next = active(r, k + 1);
        if (now) {
          if (!mbar_wait(p_full + 8 * r, (p_phase >> r) & 1u, dead)) {
            ok = false;
            break;
          }
          p_phase ^= 1u << r;
          tc_fence_after();
          if (lead) {
            const uint64_t db = ring_desc + (uint64_t)(sv * Shape::kTile >> 4);
#pragma unroll
            for (int i = 0; i < kKeys / 16; ++i) mma_f16_ts(result, scores + 8 * i, db + i * (2048 >> 4), kValues, begun[r] || i);
          }
          begun[r] = true;
        }
        if (next) {
          if (lead) {
            const uint64_t da = q_desc + (uint64_t)(r * Shape::kTile >> 4), db = ring_desc + (uint64_t)(sk * Shape::kTile >> 4);
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
              const uint64_t at = (uint64_t)((i / 4) * 16384 + (i % 4) * 32) >> 4;
              mma_f16<1>(scores, da + at, db + at, kScores, i > 0);
            }
            mma_commit<1>(s_full + 8 * r);
          }
        }
        __syncwarp();
      }
      if (!ok) break;
      if (lead) {
        if (k >= 0) mma_commit<1>(empty + 8 * sv);
        if (k + 1 < count) mma_commit<1>(empty + 8 * sk);
      }
      __syncwarp();
    }
    if (lead)
      for (int r = 0; r < groups; ++r) mma_commit<1>(o_full + 8 * r);
    __syncwarp();
  } else {                                 // a query a thread
    const int r = warp >> 2, row = (warp & 3) * 32 + lane, i = group_query(r) + row, h = group_head(r);
    const uint32_t mine = tmem + ((uint32_t)((warp & 3) * 32) << 16), scores = mine + 128 * r, result = mine + 256 + D * r;
    // scores of 0 where the scale is 0, and -inf stays -inf
    const float c = fmaxf(fabsf(p.scale) * kLog2e, 1e-30f);
    const bool negative = p.scale < 0.f;
    float top = -INFINITY, total = 0.f;
    uint32_t phase = 0;
    bool ok = true;
    for (int k = 0; k < count; ++k) {
      if (!active(r, k)) continue;
      if (!mbar_wait(s_full + 8 * r, phase, dead)) {
        ok = false;
        break;
      }
      phase ^= 1u;
      tc_fence_after();
      float s[kKeys];
      tmem_fetch64(scores, s);
      tmem_fetch64(scores + 64, s + 64);
      tmem_loaded();
      tmem_use(s);
      if (negative)
#pragma unroll
        for (int e = 0; e < kKeys; ++e) s[e] = -s[e];
      const int j = blocks.key(k, kKeys), q = group_query(r);
      if (k < blocks.nfirst) {             // first tokens before the window: all queries see them
        const int here = blocks.first - j;
        if (here < kKeys)
#pragma unroll
          for (int e = 0; e < kKeys; ++e) s[e] = e < here ? s[e] : -INFINITY;
      } else if (j + kKeys - 1 > q || j <= q + 127 - p.window) {
        const int last = i - j, early = i - p.window - j, first = p.sinks - j;   // e <= last, and e > early or e < first
#pragma unroll
        for (int e = 0; e < kKeys; ++e) s[e] = e <= last && (e > early || e < first) ? s[e] : -INFINITY;
      }
      float m[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
      for (int e = 4; e < kKeys; ++e) m[e & 3] = fmaxf(m[e & 3], s[e]);
      const float most = fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
      if (top == -INFINITY) top = most;    // nothing summed yet
      const bool grown = (most - top) * c > kGrown;
      if (__any_sync(0xffffffffu, grown)) {
        const float keep = grown ? exp2_fast((top - most) * c) : 1.f;
        if (grown) top = most;
        total *= keep;
        // the products so far are complete: the scores of this block were issued after them
#pragma unroll
        for (int x = 0; x < D; x += 32) {
          float o[32];
          tmem_fetch32(result + x, o);
          tmem_loaded();
          tmem_use(o);
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] *= keep;
          tmem_store32(result + x, reinterpret_cast<const uint32_t*>(o));
        }
      }
      const float shift = top == -INFINITY ? 0.f : -top * c;
      float part[4] = {0.f, 0.f, 0.f, 0.f};
      uint32_t w[kKeys / 2];
#pragma unroll
      for (int e = 0; e < kKeys; e += 2) {
        const float x = exp2_fast(fmaf(s[e], c, shift)), y = exp2_fast(fmaf(s[e + 1], c, shift));
        part[(e >> 1) & 3] += x + y;
        w[e >> 1] = pack2<T>(x, y);
      }
      tmem_store32(scores, w);
      tmem_store32(scores + 32, w + 32);
      total += (part[0] + part[1]) + (part[2] + part[3]);
      tmem_stored();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(p_full + 8 * r);
    }
    if (ok && r < groups) ok = mbar_wait(o_full + 8 * r, 0, dead);
    tc_fence_after();
    const bool exists = i < p.tokens, real = i < n;
    float factor = ok ? 1.f / total : NAN;   // a wait that ran out shows in the result
    bool bad = !isfinite(factor);
    T* out = head_row<T>(p.out, b, exists ? i : 0, h);
    if (r < groups) {
#pragma unroll
      for (int x = 0; x < D; x += 32) {
        float o[32];
        tmem_fetch32(result + x, o);
        tmem_loaded();
        tmem_use(o);
#pragma unroll
        for (int e = 0; e < 32; ++e) bad |= !isfinite(o[e]) && x + e < p.dim;
        if (real) put_columns(out, o, factor, x, p.dim);
      }
    }
    if (exists && !real) put_zeros(out, p.dim);
    if (exists && p.lse) attn_lse(p, b, h, i) = real ? (top * c + log2f(total)) * kLn2 : -INFINITY;
    __syncwarp();   // what follows may write the same rows
    // a key that some row of the group does not see, or a key that it sees, is not finite
    unsigned again = __ballot_sync(0xffffffffu, bad && real && ok);
    for (; again; again &= again - 1) forward_row<T>(p, b, h, group_query(r) + (warp & 3) * 32 + __ffs(again) - 1, n);
  }
  __syncthreads();
  if (*dead)     // a wait ran out: products may still be under way
    for (int i = 0; i < 200; ++i) __nanosleep(1000);
  tc_fence_before();
  __syncthreads();
  if (warp == 9) {
    tc_fence_after();
    tmem_free<1>(tmem, 512);
  }
}

}  // namespace brace
