// Launches of the windowed attention's kernels in float32 arithmetic.
#include <algorithm>

#include "attention_float.cuh"
#include "attention_host.cuh"

namespace brace {

namespace {

// Calls f with the head's dimension in tiles of 64, 128 or 256.
template <typename F>
cudaError_t with_tile(int dim, F&& f) {
  using std::integral_constant;
  return dim <= 64 ? f(integral_constant<int, 64>{}) : dim <= 128 ? f(integral_constant<int, 128>{}) : f(integral_constant<int, 256>{});
}

unsigned tiles_of(int tokens) { return (unsigned)(((int64_t)tokens + kFloatRows - 1) / kFloatRows); }

template <typename T, int D, bool DKV>
cudaError_t launch_grad(const AttnArgs& a, cudaStream_t st) {
  static std::atomic<uint64_t> granted{0};
  auto* kernel = attn_grad_float_kernel<T, D, DKV>;
  const cudaError_t err = grant_smem((const void*)kernel, granted, FloatShape<D>::kGrad);
  if (err != cudaSuccess) return err;
  const unsigned tiles = tiles_of(a.tokens);
  const dim3 grid(DKV ? a.first_tiles * a.pieces + tiles - a.first_tiles : tiles, (unsigned)(DKV ? a.kv_heads : a.heads), (unsigned)a.batch);
  return launch(kernel, grid, kFloatThreads, FloatShape<D>::kGrad, 1, st, a);
}

}  // namespace

cudaError_t attn_forward_float(int type, const AttnArgs& a, cudaStream_t st) {
  return with_type(type, [&](auto t) {
    return with_tile(a.dim, [&](auto d) {
      using T = decltype(t);
      constexpr int D = decltype(d)::value;
      static std::atomic<uint64_t> granted{0};
      auto* kernel = attn_forward_float_kernel<T, D>;
      const cudaError_t err = grant_smem((const void*)kernel, granted, FloatShape<D>::kForward);
      if (err != cudaSuccess) return err;
      return launch(kernel, dim3(tiles_of(a.tokens), (unsigned)a.heads, (unsigned)a.batch), kFloatThreads, FloatShape<D>::kForward, 1, st, a);
    });
  });
}

cudaError_t attn_grad_float(int type, const AttnArgs& a, cudaStream_t st) {
  return with_type(type, [&](auto t) {
    return with_tile(a.dim, [&](auto d) {
      using T = decltype(t);
      constexpr int D = decltype(d)::value;
      cudaError_t err = launch(attn_prepare_float_kernel<T>, dim3((unsigned)(a.padded / 8), (unsigned)a.heads, (unsigned)a.batch), 256, 0, 1, st, a);
      // dq first: dk and dv take the delta that it may have made
      if (err == cudaSuccess) err = launch_grad<T, D, false>(a, st);
      if (err == cudaSuccess) err = launch_grad<T, D, true>(a, st);
      if (err == cudaSuccess && a.first_tiles)
        err = launch(attn_join_kernel<T, D, kFloatRows>, dim3((unsigned)(a.first_tiles * (kFloatRows / 4)), (unsigned)a.kv_heads, (unsigned)a.batch),
                     128, 0, 1, st, a);
      return err;
    });
  });
}

}  // namespace brace
