// What the host sides of the operators share: sizes and alignment of arguments, launches, the tensor-map encoder.
#pragma once

#include "brace.h"

#include <cuda.h>
#include <cuda_runtime.h>

#include <atomic>

#include "elements.cuh"

namespace brace {

int cuda_fail_no_ctx(cudaError_t err);   // brace.cu: keeps the error for brace_last_cuda_error(NULL)

inline int64_t round_up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }
inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

inline int elem_bytes(int type) { return type == BRACE_TYPE_F32 || type == BRACE_TYPE_BITS ? 4 : 2; }
inline bool float_type(int t) { return t == BRACE_TYPE_F32 || t == BRACE_TYPE_BF16 || t == BRACE_TYPE_F16; }

inline bool typed(const void* p, int type) { return p && aligned(p, (size_t)elem_bytes(type)); }
inline bool typed_or_null(const void* p, int type) { return !p || aligned(p, (size_t)elem_bytes(type)); }

// Rows and matrices whose 8-element groups are whole 16-byte words.
inline bool wide_rows(const void* p, int type, int64_t ld, int64_t s1, int64_t s2 = 0) {
  const int64_t per = 16 / elem_bytes(type);
  return aligned(p, 16) && ld % per == 0 && s1 % per == 0 && s2 % per == 0;
}

inline int sm_count() {
  static std::atomic<int> cached[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 148;
  int n = cached[dev].load(std::memory_order_relaxed);
  if (n == 0) {
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) n = 148;
    cached[dev].store(n, std::memory_order_relaxed);
  }
  return n;
}

// Every kernel here waits on the device for the one before it (griddepcontrol.wait) and may be set up while that one
// drains.  `cluster`: CTAs per cluster.
struct LaunchConfig {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  LaunchConfig(dim3 grid, int block, size_t smem, int cluster, cudaStream_t st) {
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
  }
  LaunchConfig(const LaunchConfig&) = delete;   // cfg points into it
};

template <typename... KArgs, typename... Args>
cudaError_t launch(void (*kernel)(KArgs...), dim3 grid, int block, size_t smem, int cluster, cudaStream_t st,
                   const Args&... args) {
  const LaunchConfig at(grid, block, smem, cluster, st);
  return cudaLaunchKernelEx(&at.cfg, kernel, args...);
}

// Calls f with a value of the element type.
template <typename F>
cudaError_t with_type(int type, F&& f) {
  if (type == BRACE_TYPE_F32) return f(float{});
  if (type == BRACE_TYPE_BF16) return f(__nv_bfloat16{});
  return f(__half{});
}

// Lets a kernel use its shared memory on the current device (once per device and kernel).
inline cudaError_t grant_smem(const void* kernel, std::atomic<uint64_t>& granted, int bytes) {
  int dev = 0;
  cudaError_t err = cudaGetDevice(&dev);
  if (err != cudaSuccess) return err;
  const uint64_t bit = 1ull << (dev & 63);
  if (granted.load(std::memory_order_relaxed) & bit) return cudaSuccess;
  err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (err == cudaSuccess) granted.fetch_or(bit, std::memory_order_relaxed);
  return err;
}

using EncodeFn = decltype(&cuTensorMapEncodeTiled);
inline EncodeFn encode_fn() {
  static std::atomic<void*> fn{nullptr};
  void* f = fn.load(std::memory_order_acquire);
  if (!f) {
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess)
      return nullptr;
    fn.store(f, std::memory_order_release);
  }
  return (EncodeFn)f;
}

}  // namespace brace
