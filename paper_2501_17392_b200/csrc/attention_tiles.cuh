// Windowed attention on the tensor cores: bfloat16 and float16, head dimensions up to 128 in tiles of 64 or 128.
// Formulas and the treatment of single rows are in attention_rows.cuh.
//
// Forward.  A CTA has 128 queries and walks the blocks of 128 keys that they see: the first tokens', then the window's.  Per
// block: scores S = Q K^T into tensor memory; a thread takes a query's scores into registers, masks them, brings its running
// maximum up to date and writes exp2 of the differences, rounded to the inputs' type, back to tensor memory as P; P V is added
// to the result there.  The result is scaled again only when a maximum has grown by more than 2^8, or 2^6.9 in float16 (the sum
// and P have room for that).  Two CTAs share an SM: one's exponentials go on while the tensor cores work for the other, and one
// begins or ends while the other is under way.
//
// Backward, in two kernels, so that every result is summed in one order.  Scores and dp = do v of a block go into tensor memory,
// a thread makes p and ds of its columns and writes them back there, rounded to the inputs' type, and the products with k (with
// do and q) add to the results.
//   * dq: 128 queries by blocks of 128 keys; eight warps, half of a row a thread.  ds has a place of its own, so that the next
//     block's scores are made meanwhile.  In bfloat16 it also makes delta and -log2(e) lse of its queries, which dk and dv take:
//     a launch of its own for them costs 581 us for 566 at 4 x 4096 tokens, 16 heads on 4 of 128, window 1024, and 230 for 207
//     at 8 x 2048 tokens, 12 heads of 64, window 128.
//   * dk and dv: 128 keys by blocks of 64 queries of all heads that share them; two groups of four warps take the blocks by
//     turns.  With both results there is no such room: p and ds take the scores' and dp's place, and a group's next scores wait
//     for their products.  Tiles of first tokens are seen by all queries: their blocks are shared out over several CTAs, whose
//     float32 sums a last launch adds up.
// In float16 P, p and ds are held times powers of two, since they are often below what float16 holds at full precision: P times
// 2^9 (AttnRange), p times 2^15, ds times what the largest |do| and |v| allow without overflow.
//
// Bound by the chain of a block rather than by a unit: forward, 8192 tokens, 12 heads of 64, window 1024, 64 us, with the
// exponentials' unit busy for 45 % of the cycles, issue 30 %, matrix instructions 22 %; the operations alone would take 15 us.
// Backward, 4 x 4096 tokens, 16 heads on 4 of 128, window 1024, 559 us (183): matrix instructions 41 % (dq) and 54 % (dk, dv).
// Scores and dp are made in both kernels, seven products for the five of the formulas, and those of 64 queries run at half rate.
//
// A product with P = 0 where a key is hidden gives NaN if that key's value is not finite.  A row whose result is not
// finite is therefore computed again, key by key, from what it sees.
#pragma once

#include <type_traits>

#include "attention_blocks.cuh"

namespace brace {

constexpr int kAttnThreads = 320;          // of the backward pass: eight warps, one that loads, one that issues products
// log2 of what a maximum may grow by before the result is scaled again, and of what P is held times.  float16 keeps no full
// precision below 2^-14, which the weights of many keys beside a few large ones fall below: 2^9 times the 2^6.9 of a grown
// maximum is the most that it holds (weights of 2^-25 beside one of 1: off by 0.7 % with 2^7 and 2^8, 0.2 % with these; 2^11 and
// 2^4 rescale more often: 4 x 4096 tokens, 16 heads on 4 of 128, 189 us for 180).
template <typename T>
struct AttnRange {
  static constexpr bool kHalf = std::is_same<T, __half>::value;
  static constexpr float kGrown = kHalf ? 6.9f : 8.f, kUp = kHalf ? 9.f : 0.f;
};

// Of the forward pass, two CTAs an SM.  With D = 64 a CTA's half of the tensor memory holds a block's scores, its P and the
// result; with D = 128 P takes the scores' place, and the next scores have to wait for its product.  LONG keeps float32 sums in
// shared memory beside (attn_forward_kernel); of D = 128 that leaves room for one CTA.
template <int D, bool LONG>
struct AttnShape {
  static constexpr int kKeys = 128;
  static constexpr bool kApart = D == 64;                  // P has a place of its own
  static constexpr int kTile = 128 * D * 2;                // bytes of 128 rows: D / 64 blocks of 64 columns
  static constexpr int kStages = LONG ? (D == 64 ? 3 : 4) : D == 64 ? 5 : 2;
  static constexpr int kKept = LONG ? 128 * D * 4 : 0;     // bytes of the sums
  static constexpr int kSmem = 1024 + (1 + kStages) * kTile + kKept + 256;
  static constexpr int kCtas = LONG && D == 128 ? 1 : 2;   // of an SM
  static constexpr int kP = kApart ? 128 : 0, kResult = kApart ? 192 : 128, kColumns = 256;   // of tensor memory
  static constexpr int kThreads = 192;                     // four warps of queries, one that loads, one that issues products
};

// Sums on the tensor cores are cut off at every step of 16 keys (or queries), by 2e-7 of the sum on average: sums of one sign come
// out 1e-7 too small for each step.  262,144 keys, values of one sign: 1.7e-3 too small, where half a step of float16 is 4.9e-4
// and of bfloat16 3.9e-3.  From 65,536 keys on (four times as many in bfloat16 with D = 128, where it costs most) what has been
// summed is therefore taken out after every 16,384 of them and added up in float32, to nearest: 1.0e-4.  131,072 tokens, 2 heads
// on one, all keys, float16: heads of 64 5.8 -> 5.9 ms, heads of 128 (one CTA an SM) 8.4 -> 11.4.
constexpr int kLongKeys = 65536;
constexpr int kFoldKeys = 128;             // blocks of keys

struct AttnMaps {
  CUtensorMap q, k, v, dout;               // (dimension, token, head, sequence); boxes of 64 x 128, or of 64 x kBlock
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

// The lowest n bits set.
__device__ __forceinline__ uint32_t low_bits(int n) { return n >= 32 ? ~0u : (1u << max(n, 0)) - 1u; }

// ROWS rows of a head from token `t` on: D / 64 boxes of 64 columns.
template <int D, int ROWS>
__device__ __forceinline__ void load_rows(uint32_t dst, const CUtensorMap* map, int t, int head, int b, uint32_t bar) {
#pragma unroll
  for (int x = 0; x < D / 64; ++x) tma_load<1>(dst + x * ROWS * 128, map, 64 * x, t, head, b, bar);
}

// After `issued` loads into a ring of STAGES, once a wait ran out: what is under way lands before the CTA's memory goes.
template <int STAGES>
__device__ __forceinline__ void rows_landed(uint32_t full, int issued, volatile int* dead) {
#pragma unroll 1
  for (int i = max(issued - STAGES, 0); i < issued; ++i) mbar_wait(full + 8 * (i % STAGES), (uint32_t)(i / STAGES) & 1u, dead);
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

// v += 32 columns of this row's sums at `part`.
__device__ __forceinline__ void add_to(float (&v)[32], const float* part) {
#pragma unroll
  for (int e = 0; e < 32; e += 4) {
    const float4 x = *reinterpret_cast<const float4*>(part + e);
    v[e] += x.x;
    v[e + 1] += x.y;
    v[e + 2] += x.z;
    v[e + 3] += x.w;
  }
}
// 32 columns of a result in tensor memory to this row's sums at `part`, added to what is there (`more`) or the first ones.
__device__ __forceinline__ void add_sums(uint32_t result, float* part, bool more) {
  float v[32];
  tmem_fetch32(result, v);
  tmem_loaded();
  tmem_use(v);
  if (more) add_to(v, part);
#pragma unroll
  for (int e = 0; e < 32; e += 4) *reinterpret_cast<float4*>(part + e) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
}

// LONG: sums over more than kLongKeys.  grid: (tiles of 128 queries, heads, sequences)
template <typename T, int D, bool LONG>
__global__ void __launch_bounds__(AttnShape<D, LONG>::kThreads, AttnShape<D, LONG>::kCtas)
    attn_forward_kernel(const __grid_constant__ AttnMaps maps, const AttnArgs p) {
  using Shape = AttnShape<D, LONG>;
  constexpr int STAGES = Shape::kStages, KEYS = Shape::kKeys;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_addr(smem_raw) + 1023u) & ~1023u;
  const uint32_t ring = base + Shape::kTile, bars = ring + STAGES * Shape::kTile + Shape::kKept;
  const uint32_t full = bars, empty = full + 8 * STAGES, q_full = empty + 8 * STAGES;
  // scores are there, scores have been read, P is there, its product is complete
  const uint32_t s_full = q_full + 8, s_free = s_full + 8, p_full = s_free + 8, p_done = p_full + 8, tail = p_done + 8;
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
    mbar_init(s_full, 1);
    mbar_init(s_free, 4);
    mbar_init(p_full, 4);
    mbar_init(p_done, 1);
    mbar_init_visible();
    tma_prefetch(&maps.q);
    tma_prefetch(&maps.k);
    tma_prefetch(&maps.v);
  }
  if (warp == 5) tmem_alloc<1>(smem_addr(tmem_slot), Shape::kColumns);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  grid_trigger();
  grid_wait();
  fence_async_global();

  // the last queries first: they have the longest windows
  const int b = blockIdx.z, h = blockIdx.y, g = h / p.share, n = attn_length(p, b), q0 = 128 * (int)(gridDim.x - 1 - blockIdx.x);
  const KeyBlocks blocks(p, q0, min(n, q0 + 128), KEYS);
  const int count = q0 < n ? blocks.count : 0;
  // a few first tokens: the rest of their block is left out
  auto narrow = [&](int k) { return k < blocks.nfirst && blocks.first - k * KEYS <= 32; };

  if (warp == 4) {                         // loads: keys and values in the order in which the products take them
    const bool lead = elect_one();
    if (lead && count) {
      mbar_expect_tx(q_full, Shape::kTile);
      load_rows<D, 128>(base, &maps.q, q0, h, b, q_full);
    }
    __syncwarp();
    int s = 0, issued = 0;
    uint32_t ph = 0;
    for (int i = 0; i < 2 * count; ++i) {
      if (!mbar_wait(empty + 8 * s, ph ^ 1u, dead)) break;
      if (lead) {
        // P apart: the keys of block 0; then, with the values of each block, the keys of the next one before them
        const bool last = i == 2 * count - 1, values = Shape::kApart ? last || (i > 0 && (i & 1) == 0) : i & 1;
        const int k = !Shape::kApart ? i / 2 : last ? count - 1 : values ? i / 2 - 1 : (i + 1) / 2;
        mbar_expect_tx(full + 8 * s, Shape::kTile);
        load_rows<D, KEYS>(ring + s * Shape::kTile, values ? &maps.v : &maps.k, blocks.key(k, KEYS), g, b, full + 8 * s);
      }
      __syncwarp();
      ++issued;
      if (++s == STAGES) {
        s = 0;
        ph ^= 1u;
      }
    }
    dead[1] = issued;
  } else if (warp == 5) {                  // products
    const bool lead = elect_one();
    constexpr uint32_t kScores = attn_idesc<T>(KEYS, false), kValues = attn_idesc<T>(D, true);
    const uint64_t q_desc = operand_desc(base, 16384), ring_desc = operand_desc(ring, 16384);
    int at = 0;                            // loads taken
    auto scores = [&](int k) {
      const int s = at % STAGES;
      if (!mbar_wait(full + 8 * s, (uint32_t)(at / STAGES) & 1u, dead)) return false;
      if (Shape::kApart && k > 0 && !mbar_wait(s_free, (uint32_t)(k - 1) & 1u, dead)) return false;
      ++at;
      tc_fence_after();
      if (lead) {
        const uint64_t db = ring_desc + (uint64_t)(s * Shape::kTile >> 4);
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
          const uint64_t step = (uint64_t)((i / 4) * 16384 + (i % 4) * 32) >> 4;
          mma_f16<1>(tmem, q_desc + step, db + step, kScores, i > 0);
        }
        mma_commit<1>(s_full);
        mma_commit<1>(empty + 8 * s);
      }
      __syncwarp();
      return true;
    };
    bool ok = count > 0 && mbar_wait(q_full, 0, dead) && scores(0);
    for (int k = 0; ok && k < count; ++k) {
      // P apart: the next scores are issued as soon as these have been read
      if (Shape::kApart && k + 1 < count && !(ok = scores(k + 1))) break;
      const int s = at % STAGES;
      if (!mbar_wait(full + 8 * s, (uint32_t)(at / STAGES) & 1u, dead) || !mbar_wait(p_full, (uint32_t)k & 1u, dead)) break;
      ++at;
      tc_fence_after();
      if (lead) {
        const uint64_t db = ring_desc + (uint64_t)(s * Shape::kTile >> 4);
#pragma unroll
        for (int i = 0; i < KEYS / 16; ++i)
          if (i < 2 || !narrow(k))
            mma_f16_ts(tmem + Shape::kResult, tmem + Shape::kP + 8 * i, db + i * (2048 >> 4), kValues,
                       i > 0 || (LONG ? k % kFoldKeys > 0 : k > 0));
        mma_commit<1>(p_done);
        mma_commit<1>(empty + 8 * s);
      }
      __syncwarp();
      if (!Shape::kApart && k + 1 < count) ok = scores(k + 1);
    }
  } else {                                 // a query a thread
    const int row = warp * 32 + lane, i = q0 + row;
    const uint32_t mine = tmem + ((uint32_t)(warp * 32) << 16), weights = mine + Shape::kP, result = mine + Shape::kResult;
    // scores of 0 where the scale is 0, and -inf stays -inf
    const float c = fmaxf(fabsf(p.scale) * kLog2e, kTinyScale);
    const bool negative = p.scale < 0.f;
    constexpr float kGrown = AttnRange<T>::kGrown, kUp = AttnRange<T>::kUp;
    float* kept = (float*)(smem_raw + (ring + STAGES * Shape::kTile - smem_addr(smem_raw))) + row;      // column x at 128 x
    float top = -INFINITY, total = 0.f;
    // One block of which COLS columns are looked at; MASKED: those that are seen, in `seen`.
    auto block = [&](auto cols, auto masked, int k, const uint32_t* seen) {
      constexpr int COLS = decltype(cols)::value;
      constexpr bool MASKED = decltype(masked)::value;
      float s[COLS];
      if constexpr (COLS == 32) {
        tmem_fetch32(mine, s);
      } else {
        tmem_fetch64(mine, s);
        tmem_fetch64(mine + 64, s + 64);
      }
      tmem_loaded();
      tmem_use(s);
      if (Shape::kApart) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(s_free);
      }
      if (negative)
#pragma unroll
        for (int e = 0; e < COLS; ++e) s[e] = -s[e];
      if (MASKED)
#pragma unroll
        for (int e = 0; e < COLS; ++e) s[e] = seen[e / 32] >> (e % 32) & 1u ? s[e] : -INFINITY;
      float m[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
      for (int e = 0; e < COLS; e += 2) m[e / 2 & 3] = fmaxf(m[e / 2 & 3], fmaxf(s[e], s[e + 1]));
      const float most = fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
      if (top == -INFINITY) top = most;    // nothing summed yet
      const bool grown = (most - top) * c > kGrown, rescale = __any_sync(0xffffffffu, grown);
      float keep = 1.f;
      if (grown) {
        keep = exp2_fast((top - most) * c);
        top = most;
      }
      const float shift = top == -INFINITY ? 0.f : fmaf(-top, c, kUp);
      const uint64_t cc = pack_f32x2(c, c), shifts = pack_f32x2(shift, shift);
      uint64_t part[4] = {0, 0, 0, 0};
      uint32_t w[COLS / 2];
#pragma unroll
      for (int e = 0; e < COLS; e += 2) {
        float2 x = unpack_f32x2(fma_f32x2(pack_f32x2(s[e], s[e + 1]), cc, shifts));
        x = make_float2(exp2_fast(x.x), exp2_fast(x.y));
        part[e / 2 & 3] = add_f32x2(part[e / 2 & 3], pack_f32x2(x.x, x.y));
        w[e / 2] = pack2<T>(x.x, x.y);
      }
      const float2 sum = unpack_f32x2(add_f32x2(add_f32x2(part[0], part[1]), add_f32x2(part[2], part[3])));
      total = fmaf(total, keep, sum.x + sum.y);
      // the product with the block before has read its P and is part of the result (with P in the scores' place it was
      // issued before these scores)
      if (Shape::kApart && k && !mbar_wait(p_done, (uint32_t)(k - 1) & 1u, dead)) return false;
      tc_fence_after();
      if constexpr (LONG) {
        if (k && (rescale || k % kFoldKeys == 0)) {      // the sums before, and the result where the product begins anew
#pragma unroll 1
          for (int x = 0; x < D; x += 16) {
            float o[16];
            tmem_load16(result + x, o);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              float& sum = kept[(x + e) * 128];
              if (k % kFoldKeys == 0)
                sum = (k > kFoldKeys ? sum + o[e] : o[e]) * keep;
              else {
                if (k > kFoldKeys) sum *= keep;
                o[e] *= keep;
              }
            }
            if (k % kFoldKeys) tmem_store16(result + x, reinterpret_cast<const uint32_t*>(o));
          }
        }
      } else if (rescale && k) {
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
      if constexpr (COLS == 32) {
        tmem_store16(weights, w);
      } else {
        tmem_store32(weights, w);
        tmem_store32(weights + 32, w + 32);
      }
      tmem_stored();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(p_full);
      return true;
    };
    using std::integral_constant;
    using std::false_type;
    using std::true_type;
    bool ok = true;
    for (int k = 0; ok && k < count; ++k) {
      if (!mbar_wait(s_full, (uint32_t)k & 1u, dead)) {
        ok = false;
        break;
      }
      tc_fence_after();
      const int j = blocks.key(k, KEYS);
      const bool first = k < blocks.nfirst;
      if (first || j + KEYS - 1 > q0 || j <= q0 + 127 - p.window) {
        // first tokens before the window: all queries see them; else key j + e is not behind query i, and is in its window or
        // one of the first tokens
        uint32_t seen[KEYS / 32];
#pragma unroll
        for (int x = 0; x < KEYS; x += 32)
          seen[x / 32] = first ? low_bits(blocks.first - j - x)
                               : low_bits(i - j + 1 - x) & (~low_bits(i - p.window + 1 - j - x) | low_bits(p.sinks - j - x));
        ok = narrow(k) ? block(integral_constant<int, 32>{}, true_type{}, k, seen) : block(integral_constant<int, KEYS>{}, true_type{}, k, seen);
      } else {
        ok = block(integral_constant<int, KEYS>{}, false_type{}, k, nullptr);
      }
    }
    if (ok && count) ok = mbar_wait(p_done, (uint32_t)(count - 1) & 1u, dead);
    tc_fence_after();
    const bool exists = i < p.tokens, real = i < n;
    float factor = ok ? 1.f / total : NAN;   // a wait that ran out shows in the result
    bool bad = !isfinite(factor);
    T* out = head_row<T>(p.out, b, exists ? i : 0, h);
    if (count) {
#pragma unroll
      for (int x = 0; x < D; x += 32) {
        float o[32];
        tmem_fetch32(result + x, o);
        tmem_loaded();
        tmem_use(o);
        if (LONG && count > kFoldKeys)
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] += kept[(x + e) * 128];
#pragma unroll
        for (int e = 0; e < 32; ++e) bad |= !isfinite(o[e]) && x + e < p.dim;
        if (real) put_columns(out, o, factor, x, p.dim);
      }
    }
    if (exists && !real) put_zeros(out, p.dim);
    if (exists && p.lse) attn_lse(p, b, h, i) = !real ? -INFINITY : ok ? (top * c + (log2f(total) - kUp)) * kLn2 : NAN;
    __syncwarp();   // what follows may write the same rows
    // a key that some row of the tile does not see, or a key that it sees, is not finite
    unsigned again = __ballot_sync(0xffffffffu, bad && real && ok);
    for (; again; again &= again - 1) forward_row<T>(p, b, h, q0 + warp * 32 + __ffs(again) - 1, n);
  }
  __syncthreads();
  if (*dead) {   // a wait ran out: loads and products may still be under way
    if (warp == 4 && count) {
      mbar_wait(q_full, 0, dead);
      rows_landed<STAGES>(full, dead[1], dead);
    }
    for (int i = 0; i < 200; ++i) __nanosleep(1000);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 5) {
    tc_fence_after();
    tmem_free<1>(tmem, Shape::kColumns);
  }
}

// ---- backward

constexpr int kBlock = 64;                 // queries of a block (dk, dv)
// Long sums as in the forward pass: a CTA that sums more than kLongBlocks blocks (65,536 queries: 4e-4 are lost, close to half a
// step of float16) adds what it has to float32 sums in the workspace after every kFoldBlocks and begins anew.  17,000 tokens, 64 heads on one of
// 64, window 4096, do > 0, one float16 CTA a tile: error of dv 1.5e-3 -> 2.4e-4 and of dk 4.4e-4 -> 2.1e-4
// (their rounding alone 2.2e-4 and 2.1e-4).
constexpr int kLongBlocks = 1024, kFoldBlocks = 256;
constexpr float kWeightUp = 32768.f;       // float16 p (at most 1) is held times this, so that small weights keep their precision too

template <int D>
struct DkvShape {
  static constexpr int kTile = 128 * D * 2, kHalf = kBlock * D * 2;
  static constexpr int kStage = 2 * kHalf + 1024;          // a block's queries and do, and its queries' numbers
  static constexpr int kStages = D == 64 ? 6 : 4;
  static constexpr int kSmem = 1024 + 2 * kTile + kStages * kStage + 256;
};

template <int D, bool TWO>
struct DqShape {
  static constexpr int kTile = 128 * D * 2;
  static constexpr int kRingK = 3, kRingV = D == 64 ? 3 : 2;       // blocks; a block's values are free again once dp is made
  static constexpr int kSmem = (2 + kRingK + kRingV) * kTile + 256 + 2 * 128 * 4;
  static_assert(kSmem <= 232448, "shared memory");
  static constexpr int kDs = 256 + D;      // columns of tensor memory: scores, dp, dq, ds (in float16 two values of it)
  static_assert(kDs + (TWO ? 128 : 64) <= 512, "tensor memory");
};

__device__ __forceinline__ float4 lds_f32x4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr));
  return v;
}

constexpr int kPrepRows = 64;              // queries of a CTA that prepares the backward pass

// float16: delta, -log2(e) lse, and the ranges of do and v, which have to be known before ds is held; 16 lanes a row.  (In
// bfloat16 the kernel that makes dq makes the two numbers.)  grid: (padded / kPrepRows, heads, sequences)
__global__ void __launch_bounds__(256) attn_prepare_kernel(const AttnArgs p) {
  using T = __half;
  grid_trigger();
  grid_wait();
  const int h = blockIdx.y, b = blockIdx.z, n = attn_length(p, b), part = threadIdx.x & 15;
  float most_do = 0.f, most_v = 0.f;
  for (int i = blockIdx.x * kPrepRows + (threadIdx.x >> 4); i < (int)(blockIdx.x + 1) * kPrepRows; i += 16) {
    float s = 0.f;
    const bool here = i < n && 8 * part < p.dim;
    if (here) {
      Pack<T, 8> o, d;
      o.load(head_row<const T>(p.out, b, i, h) + 8 * part);
      d.load(head_row<const T>(p.dout, b, i, h) + 8 * part);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = to_f32(d.t[e]);
        s = fmaf(to_f32(o.t[e]), x, s);
        if (isfinite(x)) most_do = fmaxf(most_do, fabsf(x));
      }
      if (h % p.share == 0) {
        Pack<T, 8> v;
        v.load(head_row<const T>(p.v, b, i, h / p.share) + 8 * part);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float x = to_f32(v.t[e]);
          if (isfinite(x)) most_v = fmaxf(most_v, fabsf(x));
        }
      }
    }
    for (int o = 8; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (part == 0) {
      p.delta[attn_delta(p, b, h, i)] = i < n ? s : 0.f;
      p.shift[attn_delta(p, b, h, i)] = i < n ? -kLog2e * attn_lse(p, b, h, i) : 0.f;
    }
  }
  for (int o = 16; o; o >>= 1) {
    most_do = fmaxf(most_do, __shfl_xor_sync(0xffffffffu, most_do, o));
    most_v = fmaxf(most_v, __shfl_xor_sync(0xffffffffu, most_v, o));
  }
  if ((threadIdx.x & 31) == 0) {           // of numbers that are not negative the bits are in the same order
    uint32_t* to = p.range + ((int64_t)b * p.kv_heads + h / p.share) * 2;
    if (most_do > 0.f) atomicMax(to, __float_as_uint(most_do));
    if (most_v > 0.f) atomicMax(to + 1, __float_as_uint(most_v));
  }
}

// The power of two that ds is held times: |dp - delta| <= 2 D max|do| max|v| then stays below 2^15.
__device__ __forceinline__ float attn_grad_scale(const AttnArgs& p, int b, int g) {
  if (!p.range) return 1.f;
  const uint32_t* r = p.range + ((int64_t)b * p.kv_heads + g) * 2;
  const float bound = p.dim * __uint_as_float(r[0]) * __uint_as_float(r[1]);
  return bound > 0.f ? ldexpf(1.f, 13 - ilogbf(bound)) : 1.f;
}

// dq.  LONG: sums over more than kLongKeys.  grid: that of GradWork
template <typename T, int D, bool LONG>
__global__ void __launch_bounds__(kAttnThreads, 1) attn_dq_kernel(const __grid_constant__ AttnMaps maps, const AttnArgs p) {
  // float16: ds as the sum of two values.  With one, its rounding and the result's together are 1.5 times the result's alone
  constexpr bool kTwo = std::is_same<T, __half>::value;
  using Shape = DqShape<D, kTwo>;
  constexpr int RK = Shape::kRingK, RV = Shape::kRingV, BLOCK = 128, COLS = BLOCK / 2;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  const uint32_t base = smem_addr(smem_raw), ring_k = base + 2 * Shape::kTile, ring_v = ring_k + RK * Shape::kTile;
  const uint32_t bars = ring_v + RV * Shape::kTile;
  const uint32_t full_k = bars, empty_k = full_k + 24, full_v = empty_k + 24, empty_v = full_v + 24;
  // the rows are there; scores and dp are there, have been read; ds is there, its product is complete
  const uint32_t a_full = empty_v + 24, s_full = a_full + 8, s_free = s_full + 8, p_full = s_free + 8, p_done = p_full + 8;
  const uint32_t d_full = p_done + 8, tail = d_full + 8;      // the halves' sums of p dp are there
  volatile int* dead = (volatile int*)(smem_raw + (tail - base));
  uint32_t* tmem_slot = (uint32_t*)(smem_raw + (tail + 8 - base));
  float* sums = (float*)(smem_raw + (tail + 16 - base));      // [half][row]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    *dead = 0;
    for (int s = 0; s < 3; ++s) {
      mbar_init(full_k + 8 * s, 1);
      mbar_init(empty_k + 8 * s, 1);
      mbar_init(full_v + 8 * s, 1);
      mbar_init(empty_v + 8 * s, 1);
    }
    mbar_init(a_full, 1);
    mbar_init(s_full, 1);
    mbar_init(s_free, 8);
    mbar_init(p_full, 8);
    mbar_init(p_done, 1);
    mbar_init(d_full, 8);
    mbar_init_visible();
    tma_prefetch(&maps.q);
    tma_prefetch(&maps.k);
    tma_prefetch(&maps.v);
    tma_prefetch(&maps.dout);
  }
  if (warp == 9) tmem_alloc<1>(smem_addr(tmem_slot), 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  grid_trigger();
  grid_wait();
  fence_async_global();

  const int b = blockIdx.z, n = attn_length(p, b);
  const GradWork w(p, n, false, 128, BLOCK);
  const int h = w.head, g = h / p.share;
  // few blocks are walked twice: first for delta, then for ds
  const int blocks = w.count, first_pass = blocks * 128 <= kExactKeys ? blocks : 0, count = blocks + first_pass;
  auto block_of = [&](int k) { return k < first_pass ? k : k - first_pass; };
  // long sums as in the forward pass (there is one pass over so many keys): the sums taken out lie in the workspace.  600,000 keys
  // that are the values, float16: dq 1.1e-3 too small -> 4e-5
  const bool fold = LONG && count > kLongKeys / BLOCK;
  auto fresh = [&](int k) { return fold && k > 0 && k % kFoldKeys == 0; };

  if (warp == 8) {                         // loads
    const bool lead = elect_one();
    if (lead && count) {
      mbar_expect_tx(a_full, 2 * Shape::kTile);
      load_rows<D, 128>(base, &maps.q, w.row0, h, b, a_full);
      load_rows<D, 128>(base + Shape::kTile, &maps.dout, w.row0, h, b, a_full);
    }
    __syncwarp();
    int issued_k = 0, issued_v = 0;
    for (int k = 0; k < count; ++k) {
      const int sk = k % RK, sv = k % RV, t = w.first(block_of(k));
      if (!mbar_wait(empty_v + 8 * sv, (uint32_t)(k / RV + 1) & 1u, dead)) break;
      if (lead) {
        mbar_expect_tx(full_v + 8 * sv, Shape::kTile);
        load_rows<D, BLOCK>(ring_v + sv * Shape::kTile, &maps.v, t, g, b, full_v + 8 * sv);
      }
      __syncwarp();
      ++issued_v;
      if (!mbar_wait(empty_k + 8 * sk, (uint32_t)(k / RK + 1) & 1u, dead)) break;
      if (lead) {
        mbar_expect_tx(full_k + 8 * sk, Shape::kTile);
        load_rows<D, BLOCK>(ring_k + sk * Shape::kTile, &maps.k, t, g, b, full_k + 8 * sk);
      }
      __syncwarp();
      ++issued_k;
    }
    dead[1] = issued_k;
    dead[3] = issued_v;
  } else if (warp == 9) {                  // products
    const bool lead = elect_one();
    constexpr uint32_t kScores = attn_idesc<T>(BLOCK, false), kSums = attn_idesc<T>(D, true);
    const uint64_t a_desc = operand_desc(base, 16384), desc_k = operand_desc(ring_k, 16384), desc_v = operand_desc(ring_v, 16384);
    auto scores = [&](int k) {
      const int sk = k % RK, sv = k % RV;
      if (!mbar_wait(full_k + 8 * sk, (uint32_t)(k / RK) & 1u, dead)) return false;
      if (!mbar_wait(full_v + 8 * sv, (uint32_t)(k / RV) & 1u, dead)) return false;
      if (k && !mbar_wait(s_free, (uint32_t)(k - 1) & 1u, dead)) return false;
      tc_fence_after();
      if (lead) {
        const uint64_t bk = desc_k + (uint64_t)(sk * Shape::kTile >> 4), bv = desc_v + (uint64_t)(sv * Shape::kTile >> 4);
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int i = 0; i < D / 16; ++i) {
            const uint64_t step = (uint64_t)((i / 4) * 16384 + (i % 4) * 32) >> 4;
            mma_f16<1>(tmem + 128 * x, a_desc + (uint64_t)(x * Shape::kTile >> 4) + step, (x ? bv : bk) + step, kScores, i > 0);
          }
        mma_commit<1>(s_full);
        mma_commit<1>(empty_v + 8 * sv);
        if (k < first_pass) mma_commit<1>(empty_k + 8 * sk);
      }
      __syncwarp();
      return true;
    };
    bool ok = count > 0 && mbar_wait(a_full, 0, dead) && scores(0);
    for (int k = 0; ok && k < count; ++k) {
      if (k + 1 < count && !(ok = scores(k + 1))) break;      // as soon as these have been read
      if (k < first_pass) continue;
      const int sk = k % RK;
      if (!mbar_wait(p_full, (uint32_t)(k - first_pass) & 1u, dead)) break;
      tc_fence_after();
      if (lead) {
        const uint64_t bk = desc_k + (uint64_t)(sk * Shape::kTile >> 4);
#pragma unroll
        for (int i = 0; i < BLOCK / 16; ++i) {
          mma_f16_ts(tmem + 256, tmem + Shape::kDs + 8 * i, bk + i * (2048 >> 4), kSums, i > 0 || (k > first_pass && !fresh(k)));
          if (kTwo) mma_f16_ts(tmem + 256, tmem + Shape::kDs + 64 + 8 * i, bk + i * (2048 >> 4), kSums, 1);
        }
        mma_commit<1>(empty_k + 8 * sk);
        mma_commit<1>(p_done);
      }
      __syncwarp();
    }
  } else {                                 // half of a row a thread
    const int half = warp >> 2, row = (warp & 3) * 32 + lane, at = w.row0 + row;
    const uint32_t mine = tmem + ((uint32_t)((warp & 3) * 32) << 16), words = mine + Shape::kDs + 32 * half;
    const float c = p.scale * kLog2e, hold = count ? attn_grad_scale(p, b, g) : 1.f;
    float shift = 0.f, delta = 0.f, sum = 0.f;      // sum: of p dp
    float* part = p.part + ((((int64_t)b * p.heads + h) * gridDim.x + w.row0 / 128) * 128 + row) * D;
    bool ok = true;
    auto meet = [&] {                      // all rows' sums are in shared memory
      __syncwarp();
      if (lane == 0) mbar_arrive(d_full);
      return mbar_wait(d_full, 0, dead);
    };
    if constexpr (kTwo) {
      if (at < n) {
        shift = p.shift[attn_delta(p, b, h, at)];
        delta = p.delta[attn_delta(p, b, h, at)];
      }
    } else if (count) {                    // the two numbers of this row, while the first loads are under way
      if (at < n) shift = -kLog2e * attn_lse(p, b, h, at);
      if (half == 0 && at < p.padded) p.shift[attn_delta(p, b, h, at)] = shift;
      if (!first_pass) {                   // 16 lanes a row, 8 rows at a time
#pragma unroll 1
        for (int r0 = warp * 16; r0 < warp * 16 + 16; r0 += 8) {
          Pack<T, 8> x[4], y[4];
          float s[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int i = min(w.row0 + r0 + 2 * r + (lane >> 4), n - 1), col = min(8 * (lane & 15), p.dim - 8);
            x[r].load(head_row<const T>(p.out, b, i, h) + col);
            y[r].load(head_row<const T>(p.dout, b, i, h) + col);
          }
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            s[r] = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) s[r] = fmaf(to_f32(x[r].t[e]), to_f32(y[r].t[e]), s[r]);
            if (8 * (lane & 15) >= p.dim) s[r] = 0.f;
          }
          for (int o = 8; o; o >>= 1)
#pragma unroll
            for (int r = 0; r < 4; ++r) s[r] += __shfl_xor_sync(0xffffffffu, s[r], o);
          if ((lane & 15) == 0)
#pragma unroll
            for (int r = 0; r < 4; ++r) sums[r0 + 2 * r + (lane >> 4)] = s[r];
        }
        ok = ok && meet();
        delta = sums[row];
        if (half == 0 && at < p.padded) p.delta[attn_delta(p, b, h, at)] = at < n ? delta : 0.f;
      }
    }
    for (int k = 0; ok && k < count; ++k) {
      const int t = w.first(block_of(k)) + COLS * half;
      if (!mbar_wait(s_full, (uint32_t)k & 1u, dead)) {
        ok = false;
        break;
      }
      tc_fence_after();
      float x[COLS], y[COLS];
      tmem_fetch64(mine + COLS * half, x);
      tmem_fetch64(mine + 128 + COLS * half, y);
      tmem_loaded();
      tmem_use(x);
      tmem_use(y);
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(s_free);
      if (first_pass && k == first_pass) {      // delta is complete: the two halves of a row put it together
        sums[half * 128 + row] = sum;
        if (!(ok = meet())) break;
        delta = sum + sums[(half ^ 1) * 128 + row];
        if (half == 0 && at < p.padded) p.delta[attn_delta(p, b, h, at)] = at < n ? delta : 0.f;
      }
#pragma unroll
      for (int e = 0; e < COLS; ++e) {
        x[e] = exp2_fast(fmaf(x[e], c, shift)) * (k < first_pass ? y[e] : y[e] - delta);
        if (kTwo && k >= first_pass) x[e] *= hold;
      }
      const bool first = block_of(k) < w.keys.nfirst;
      if (first || t + COLS - 1 > w.row0 || t <= w.row0 + 127 - p.window) {
        // first tokens before the window: all queries see them; else key t + e is not behind query `at`, and is in its window or
        // one of the first tokens
#pragma unroll
        for (int i = 0; i < COLS; i += 32) {
          const uint32_t seen = first ? low_bits(w.keys.first - t - i)
                                      : low_bits(at - t + 1 - i) & (~low_bits(at - p.window + 1 - t - i) | low_bits(p.sinks - t - i));
#pragma unroll
          for (int e = 0; e < 32; ++e) x[i + e] = seen >> e & 1u ? x[i + e] : 0.f;
        }
      }
      if (k < first_pass) {
#pragma unroll
        for (int e = 0; e < COLS; e += 4) sum += (x[e] + x[e + 1]) + (x[e + 2] + x[e + 3]);
        continue;
      }
      // the product with the block before has read its ds
      if (k > first_pass && !mbar_wait(p_done, (uint32_t)(k - first_pass - 1) & 1u, dead)) {
        ok = false;
        break;
      }
      tc_fence_after();
      if (half == 0 && fresh(k))
#pragma unroll 1
        for (int col = 0; col < D; col += 32) add_sums(mine + 256 + col, part + col, k > kFoldKeys);
      uint32_t word[COLS / 2];
#pragma unroll
      for (int e = 0; e < COLS; e += 2) word[e / 2] = pack2<T>(x[e], x[e + 1]);
      tmem_store32(words, word);
      if (kTwo) {
#pragma unroll
        for (int e = 0; e < COLS; e += 2) {
          const float2 hi = __half22float2(reinterpret_cast<const __half2&>(word[e / 2]));
          word[e / 2] = pack2<T>(x[e] - hi.x, x[e + 1] - hi.y);
        }
        tmem_store32(words + 64, word);
      }
      tmem_stored();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(p_full);
    }
    if (ok && count) ok = mbar_wait(p_done, (uint32_t)(blocks - 1) & 1u, dead);
    tc_fence_after();
    if (!kTwo && !ok && at < p.padded) p.delta[attn_delta(p, b, h, at)] = NAN;      // which may not have been made: dk shows it
    const bool exists = at < p.tokens, real = at < n;
    if (half == 0) {
      T* to = head_row<T>(p.dq, b, exists ? at : 0, h);
      const float factor = ok ? p.scale / hold : NAN;   // a wait that ran out shows in the result
      bool bad = false;
      if (count) {
#pragma unroll
        for (int col = 0; col < D; col += 32) {
          float o[32];
          tmem_fetch32(mine + 256 + col, o);
          tmem_loaded();
          tmem_use(o);
          if (fold) add_to(o, part + col);
#pragma unroll
          for (int e = 0; e < 32; ++e) bad |= !isfinite(o[e]) && col + e < p.dim;
          if (real) put_columns(to, o, factor, col, p.dim);
        }
      }
      if (exists && !real) put_zeros(to, p.dim);
      __syncwarp();   // what follows may write the same rows
      unsigned again = __ballot_sync(0xffffffffu, bad && real && ok);
      for (; again; again &= again - 1) dq_row<T>(p, b, h, w.row0 + warp * 32 + __ffs(again) - 1, n);
    }
  }
  __syncthreads();
  if (*dead) {   // a wait ran out: loads and products may still be under way
    if (warp == 8 && count) {
      mbar_wait(a_full, 0, dead);
      rows_landed<RK>(full_k, dead[1], dead);
      rows_landed<RV>(full_v, dead[3], dead);
    }
    for (int i = 0; i < 200; ++i) __nanosleep(1000);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 9) {
    tc_fence_after();
    tmem_free<1>(tmem, 512);
  }
}

// dk and dv.  LONG: sums over more than kLongBlocks blocks.  grid: that of GradWork
template <typename T, int D, bool LONG>
__global__ void __launch_bounds__(kAttnThreads, 1) attn_dkv_kernel(const __grid_constant__ AttnMaps maps, const AttnArgs p) {
  constexpr bool kTwo = std::is_same<T, __half>::value;
  using Shape = DkvShape<D>;
  constexpr int STAGES = Shape::kStages;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_addr(smem_raw) + 1023u) & ~1023u;
  const uint32_t ring = base + 2 * Shape::kTile, bars = ring + STAGES * Shape::kStage;
  const uint32_t full = bars, empty = full + 8 * STAGES, a_full = empty + 8 * STAGES;
  // of each group: scores and dp are there; p and ds are there; the sums that it writes are complete
  const uint32_t s_full = a_full + 8, p_full = s_full + 16, o_full = p_full + 16, tail = o_full + 16;
  volatile int* dead = (volatile int*)(smem_raw + (tail - smem_addr(smem_raw)));
  uint32_t* tmem_slot = (uint32_t*)(smem_raw + (tail + 8 - smem_addr(smem_raw)));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    *dead = 0;
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(full + 8 * s, 1);
      mbar_init(empty + 8 * s, 1);
    }
    mbar_init(a_full, 1);
    for (int r = 0; r < 2; ++r) {
      mbar_init(o_full + 8 * r, 1);
      mbar_init(s_full + 8 * r, 1);
      mbar_init(p_full + 8 * r, 4);
    }
    mbar_init_visible();
    tma_prefetch(&maps.q);
    tma_prefetch(&maps.k);
    tma_prefetch(&maps.v);
    tma_prefetch(&maps.dout);
  }
  if (warp == 9) tmem_alloc<1>(smem_addr(tmem_slot), 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  grid_trigger();
  grid_wait();
  fence_async_global();

  const int b = blockIdx.z, n = attn_length(p, b);
  const GradWork w(p, n, true, 128, kBlock);
  const int g = w.head, count = w.count;
  // The first group takes dv out before block k's products where k is a multiple of kFoldBlocks, the second one dk before those
  // of the block behind it: each of them before it hands over its own block.
  const bool fold = LONG && count > kLongBlocks;
  auto fresh = [&](int k, int r) { return fold && k > r && k % kFoldBlocks == r; };

  if (warp == 8) {                         // loads
    const bool lead = elect_one();
    if (lead && count) {
      mbar_expect_tx(a_full, 2 * Shape::kTile);
      load_rows<D, 128>(base, &maps.k, w.row0, g, b, a_full);
      load_rows<D, 128>(base + Shape::kTile, &maps.v, w.row0, g, b, a_full);
    }
    __syncwarp();
    int s = 0, issued = 0;
    uint32_t ph = 0;
    for (int k = 0; k < count; ++k) {
      if (!mbar_wait(empty + 8 * s, ph ^ 1u, dead)) break;
      if (lead) {
        const uint32_t at = ring + s * Shape::kStage, bar = full + 8 * s;
        const int t = w.first(k), h = w.head_of(k, p);
        mbar_expect_tx(bar, 2 * Shape::kHalf + 2 * kBlock * 4);
        load_rows<D, kBlock>(at, &maps.q, t, h, b, bar);
        load_rows<D, kBlock>(at + Shape::kHalf, &maps.dout, t, h, b, bar);
        bulk_load(at + 2 * Shape::kHalf, p.shift + attn_delta(p, b, h, t), kBlock * 4, bar);
        bulk_load(at + 2 * Shape::kHalf + kBlock * 4, p.delta + attn_delta(p, b, h, t), kBlock * 4, bar);
      }
      __syncwarp();
      ++issued;
      if (++s == STAGES) {
        s = 0;
        ph ^= 1u;
      }
    }
    dead[1] = issued;
  } else if (warp == 9) {                  // products
    const bool lead = elect_one();
    constexpr uint32_t kScores = attn_idesc<T>(kBlock, false), kSums = attn_idesc<T>(D, true);
    const uint64_t a_desc = operand_desc(base, kBlock * 128), ring_desc = operand_desc(ring, kBlock * 128);
    bool ok = count == 0 || mbar_wait(a_full, 0, dead);
    auto scores = [&](int k) {
      const int s = k % STAGES;
      if (!mbar_wait(full + 8 * s, (uint32_t)(k / STAGES) & 1u, dead)) return false;
      tc_fence_after();
      if (lead) {
        const uint64_t db = ring_desc + (uint64_t)(s * Shape::kStage >> 4);
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int i = 0; i < D / 16; ++i)
            mma_f16<1>(tmem + 128 * (k & 1) + 64 * x,
                       a_desc + (uint64_t)((x * Shape::kTile + (i / 4) * 16384 + (i % 4) * 32) >> 4),
                       db + (uint64_t)((x * Shape::kHalf + (i / 4) * 8192 + (i % 4) * 32) >> 4), kScores, i > 0);
        mma_commit<1>(s_full + 8 * (k & 1));
      }
      __syncwarp();
      return true;
    };
    for (int k = 0; ok && k < 2 && k < count; ++k) ok = scores(k);
    for (int k = 0; ok && k < count; ++k) {
      const int s = k % STAGES, r = k & 1;
      if (!(ok = mbar_wait(p_full + 8 * r, (uint32_t)(k >> 1) & 1u, dead))) break;
      tc_fence_after();
      if (lead) {
        const uint64_t db = ring_desc + (uint64_t)(s * Shape::kStage >> 4);
        const uint32_t a_p = tmem + 128 * r, a_ds = a_p + 64;
#pragma unroll
        for (int i = 0; i < kBlock / 16; ++i) {
          const uint64_t b1 = db + (uint64_t)(2048 * i >> 4), b2 = b1 + (Shape::kHalf >> 4);
          mma_f16_ts(tmem + 256, a_p + 8 * i, b2, kSums, i > 0 || (k > 0 && !fresh(k, 0)));
          mma_f16_ts(tmem + 256 + D, a_ds + 8 * i, b1, kSums, i > 0 || (k > 0 && !fresh(k, 1)));
          if (kTwo) mma_f16_ts(tmem + 256 + D, a_ds + 32 + 8 * i, b1, kSums, 1);
        }
        mma_commit<1>(empty + 8 * s);
        if (k + 1 < count)
          for (int x = 0; x < 2; ++x)
            if (fresh(k + 1, x)) mma_commit<1>(o_full + 8 * x);
      }
      __syncwarp();
      if (k + 2 < count) ok = scores(k + 2);
    }
    if (lead && ok) {      // else who waits for the sums gives up too
      mma_commit<1>(o_full);
      mma_commit<1>(o_full + 8);
    }
    __syncwarp();
  } else {                                 // a row a thread; the groups take the blocks by turns
    const int r = warp >> 2, row = (warp & 3) * 32 + lane, at = w.row0 + row;
    const uint32_t mine = tmem + ((uint32_t)((warp & 3) * 32) << 16), cells = mine + 128 * r;
    const float c = p.scale * kLog2e, hold = count ? attn_grad_scale(p, b, g) : 1.f;
    const uint32_t result = mine + 256 + D * r;      // the first group has dv, the second one dk
    auto sums = [&] { return p.part + w.part_of(p, b, r, 128, D) + row * D; };
    uint32_t phase = 0, folds = 0;
    bool ok = true;
    for (int k = r; k < count; k += 2) {
      if (fresh(k, r)) {
        if (!mbar_wait(o_full + 8 * r, folds & 1u, dead)) {
          ok = false;
          break;
        }
        tc_fence_after();
#pragma unroll 1
        for (int col = 0; col < D; col += 32) add_sums(result + col, sums() + col, folds > 0);
        ++folds;
      }
      const int s = k % STAGES;
      // a block's numbers were copied by the asynchronous proxy: their own barrier makes them visible
      if (!mbar_wait(full + 8 * s, (uint32_t)(k / STAGES) & 1u, dead) || !mbar_wait(s_full + 8 * r, phase, dead)) {
        ok = false;
        break;
      }
      phase ^= 1u;
      tc_fence_after();
      float x[kBlock], y[kBlock];
      tmem_fetch64(cells, x);
      tmem_fetch64(cells + 64, y);
      tmem_loaded();
      tmem_use(x);
      tmem_use(y);
      // the queries' numbers, read ahead of their use
      const uint32_t numbers = ring + s * Shape::kStage + 2 * Shape::kHalf;
      float4 sh = lds_f32x4(numbers), de = lds_f32x4(numbers + kBlock * 4);
#pragma unroll
      for (int e = 0; e < kBlock; e += 4) {
        const float shifts[4] = {sh.x, sh.y, sh.z, sh.w}, deltas[4] = {de.x, de.y, de.z, de.w};
        if (e + 4 < kBlock) {
          sh = lds_f32x4(numbers + 4 * (e + 4));
          de = lds_f32x4(numbers + 4 * (kBlock + e + 4));
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[e + i] = exp2_fast(fmaf(x[e + i], c, shifts[i]));
          y[e + i] = x[e + i] * (y[e + i] - deltas[i]);
          if (kTwo) y[e + i] *= hold;
        }
      }
      const int t = w.first(k);
      // query t + e: not before key `at`, before the end, in the key's window or the key one of the first tokens
      if (t < w.row0 + 127 || t + kBlock > n || (t + kBlock > w.row0 + p.window && w.row0 + 127 >= p.sinks)) {
        const int to = at < p.sinks || p.window > n - at ? n - t : at + p.window - t;
#pragma unroll
        for (int i = 0; i < kBlock; i += 32) {
          const uint32_t seen = low_bits(to - i) & ~low_bits(at - t - i);
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            x[i + e] = seen >> e & 1u ? x[i + e] : 0.f;
            y[i + e] = seen >> e & 1u ? y[i + e] : 0.f;
          }
        }
      }
      uint32_t word[kBlock / 2];
#pragma unroll
      for (int e = 0; e < kBlock; e += 2) word[e / 2] = kTwo ? pack2<T>(x[e] * kWeightUp, x[e + 1] * kWeightUp) : pack2<T>(x[e], x[e + 1]);
      tmem_store32(cells, word);
#pragma unroll
      for (int e = 0; e < kBlock; e += 2) word[e / 2] = pack2<T>(y[e], y[e + 1]);
      tmem_store32(cells + 64, word);
      if (kTwo) {
#pragma unroll
        for (int e = 0; e < kBlock; e += 2) {
          const float2 hi = __half22float2(reinterpret_cast<const __half2&>(word[e / 2]));
          word[e / 2] = pack2<T>(y[e] - hi.x, y[e + 1] - hi.y);
        }
        tmem_store32(cells + 96, word);
      }
      tmem_stored();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(p_full + 8 * r);
    }
    if (ok && count) ok = mbar_wait(o_full + 8 * r, folds & 1u, dead);
    tc_fence_after();
    const bool exists = at < p.tokens, real = at < n;
    T* to = head_row<T>(r ? p.dk : p.dv, b, exists ? at : 0, g);
    const float factor = !ok ? NAN : r ? p.scale / hold : kTwo ? 1.f / kWeightUp : 1.f;   // a wait that ran out shows in the result
    float* part = w.piece >= 0 || (LONG && folds) ? sums() : nullptr;
    bool bad = false;
    if (count) {
#pragma unroll
      for (int col = 0; col < D; col += 32) {
        float o[32];
        tmem_fetch32(result + col, o);
        tmem_loaded();
        tmem_use(o);
        if (LONG && folds) add_to(o, part + col);
        if (w.piece >= 0) {
#pragma unroll
          for (int e = 0; e < 32; e += 4)
            *reinterpret_cast<float4*>(part + col + e) = make_float4(o[e] * factor, o[e + 1] * factor, o[e + 2] * factor, o[e + 3] * factor);
        } else {
#pragma unroll
          for (int e = 0; e < 32; ++e) bad |= !isfinite(o[e]) && col + e < p.dim;
          if (real) put_columns(to, o, factor, col, p.dim);
        }
      }
    } else if (w.piece >= 0) {
      for (int col = 0; col < D; col += 4) *reinterpret_cast<float4*>(part + col) = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    if (exists && !real && w.piece < 0) put_zeros(to, p.dim);
    __syncwarp();   // what follows may write the same rows
    unsigned again = __ballot_sync(0xffffffffu, bad && real && ok);
    for (; again; again &= again - 1) dkv_row<T>(p, b, g, w.row0 + (warp & 3) * 32 + __ffs(again) - 1, n, r == 1, r == 0);
  }
  __syncthreads();
  if (*dead) {   // a wait ran out: loads and products may still be under way
    if (warp == 8 && count) {
      mbar_wait(a_full, 0, dead);
      rows_landed<STAGES>(full, dead[1], dead);
    }
    for (int i = 0; i < 200; ++i) __nanosleep(1000);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 9) {
    tc_fence_after();
    tmem_free<1>(tmem, 512);
  }
}

}  // namespace brace
