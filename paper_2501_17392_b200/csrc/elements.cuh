// Element types of the operators' tensors and their conversions.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace brace {

enum { kTypeF32 = 0, kTypeBF16 = 1, kTypeF16 = 2, kTypeBits = 3 };

template <int TYPE>
struct Elem { using T = float; };
template <>
struct Elem<kTypeBF16> { using T = __nv_bfloat16; };
template <>
struct Elem<kTypeF16> { using T = __half; };

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
template <typename T>
__device__ __forceinline__ T from_f32(float x);
template <>
__device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <>
__device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }

template <int BYTES>
struct WideWord;
template <>
struct WideWord<16> { using T = uint4; };
template <>
struct WideWord<8> { using T = uint2; };
template <>
struct WideWord<4> { using T = uint32_t; };
template <>
struct WideWord<2> { using T = unsigned short; };

// V consecutive elements as wide words (V * sizeof(T) bytes, at most 16 at a time).
template <typename T, int V>
struct Pack {
  static constexpr int kBytes = V * (int)sizeof(T);
  using W = typename WideWord<(kBytes >= 16 ? 16 : kBytes)>::T;
  static constexpr int kWords = kBytes / (int)sizeof(W);
  alignas(16) T t[V];
  // Ordinary loads, not those of the read-only path: a kernel here may start before the one that wrote its input has
  // ended (it waits on the device), and what it reads and writes may be one buffer.
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < kWords; ++i) reinterpret_cast<W*>(t)[i] = reinterpret_cast<const W*>(p)[i];
  }
  __device__ __forceinline__ void store_plain(T* p) const {
#pragma unroll
    for (int i = 0; i < kWords; ++i) reinterpret_cast<W*>(p)[i] = reinterpret_cast<const W*>(t)[i];
  }
  __device__ __forceinline__ void store_stream(T* p) const {
#pragma unroll
    for (int i = 0; i < kWords; ++i) __stcs(reinterpret_cast<W*>(p) + i, reinterpret_cast<const W*>(t)[i]);
  }
};

}  // namespace brace
