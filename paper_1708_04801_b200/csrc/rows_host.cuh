// What the host code of the operators on rows shares (wpsgd_rows.cu, wpsgd_nodes.cu, wpsgd_delta.cu): launches with all of an SM's shared memory and in
// clusters, checks of memory that must not overlap.
#pragma once

#include <cuda.h>

#include <atomic>

#include "context.cuh"

namespace wpsgd {

// All of an SM's shared memory for a kernel (see allow_all_smem), asked for once per device: the call takes part of a microsecond.
template <auto Kernel>
cudaError_t allow_smem(const wpsgd_ctx* c) {
  static std::atomic<uint64_t> done{0};  // a bit per device
  const uint64_t bit = c->device < 64 ? 1ull << c->device : 0;
  if (done.load(std::memory_order_acquire) & bit) return cudaSuccess;
  cudaFuncAttributes at;
  cudaError_t e = cudaFuncGetAttributes(&at, Kernel);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(Kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(kSmemMax - at.sharedSizeBytes));
  if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_release);
  return e;
}

// launch() of clusters of `cluster` blocks
template <typename... P, typename... A>
cudaError_t launch_clusters(void (*kern)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t stream, unsigned cluster, A&&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = cluster;
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kern, std::forward<A>(args)...);
}

// The driver's encoder of tensor maps, asked for by name: the library does not link against the driver.
inline decltype(&cuTensorMapEncodeTiled) tensor_map_encoder() {
  static const auto fn = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) {
      cudaGetLastError();
      f = nullptr;
    }
    return (decltype(&cuTensorMapEncodeTiled))f;
  }();
  return fn;
}
inline bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  return (uintptr_t)a < (uintptr_t)b + nb && (uintptr_t)b < (uintptr_t)a + na;
}

// Rows of `width` bytes, `stride` apart
struct Region {
  const void* p;
  long long width, stride, n;
};
// Whether two sets of rows share a byte. One may lie in the padding of the other (scales behind the codes of each row).
inline bool meet(const Region& a, const Region& b) {
  if (a.n < 1 || b.n < 1 || a.width < 1 || b.width < 1) return false;
  const uintptr_t a0 = (uintptr_t)a.p, b0 = (uintptr_t)b.p;
  if (a0 + (a.n - 1) * a.stride + a.width <= b0 || b0 + (b.n - 1) * b.stride + b.width <= a0) return false;
  if (a.stride == b.stride) {  // each row of one at the same place of a row of the other: no need to go through them
    const uintptr_t place = b0 >= a0 ? (b0 - a0) % a.stride : (a.stride - (a0 - b0) % a.stride) % a.stride;
    if (place >= (uintptr_t)a.width && place + b.width <= (uintptr_t)a.stride) return false;
  }
  const Region &few = a.n <= b.n ? a : b, &many = a.n <= b.n ? b : a;
  const uintptr_t m0 = (uintptr_t)many.p;
  for (long long i = 0; i < few.n; ++i) {
    const uintptr_t lo = (uintptr_t)few.p + i * few.stride, hi = lo + few.width;
    if (hi <= m0) continue;
    const long long last = std::min<long long>((hi - 1 - m0) / many.stride, many.n - 1);  // the last row of `many` that starts before hi
    if (m0 + last * many.stride + many.width > lo) return true;
  }
  return false;
}

inline size_t element_size(wpsgd_xtype t) { return t == WPSGD_X_F32 ? 4 : 2; }
inline bool known(wpsgd_xtype t) { return t == WPSGD_X_F32 || t == WPSGD_X_BF16; }

}  // namespace wpsgd
