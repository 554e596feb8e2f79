// The context behind the C ABI (include/wpsgd.h) and what the host code of every entry point shares: error texts, device guard,
// buffers that grow, kernel launches.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <string>
#include <utility>
#include <vector>

#include "../../include/wpsgd.h"
#include "common.cuh"

struct wpsgd_ctx {
  int device = 0;
  cudaStream_t stream = nullptr;
  int k = 0;
  long long d = 0;
  // models
  float* W = nullptr;       // [k, d]
  double* scale = nullptr;  // [k] (sparse path: w_j = scale_j * W[j])
  bool scaled = false;
  // per-launch tables on the device: one buffer laid out by TableLayout(k), and where its parts are
  unsigned char* tables = nullptr;
  long long *t_shard_off = nullptr, *t_steps = nullptr, *t_first = nullptr, *t_idx_off = nullptr;
  int* t_order = nullptr;
  std::vector<unsigned char> h_tables;
  double* t_weights = nullptr;       // [k]
  uint32_t* idx = nullptr;
  size_t idx_cap = 0;  // entries
  bool streams_read = false;  // every stream kernel so far has been followed by a launch of chains
  wpsgd::DevStatus* status = nullptr;
  double* part = nullptr;  // objective partial sums
  size_t part_cap = 0;     // doubles
  unsigned* ticket = nullptr;  // blocks of the running objective kernel that have finished (zero between launches)
  void* rows_ws = nullptr;  // workspace of the operators on whole sets of rows (RowsLayout)
  // staging of the host-buffer entry point
  void* st_X = nullptr;
  size_t st_X_cap = 0;
  float* st_y = nullptr;
  size_t st_y_cap = 0;
  float* st_v = nullptr;   // [d]
  long long* st_rp = nullptr;  // CSR staging of the host-buffer entry point
  size_t st_rp_cap = 0;
  int* st_ci = nullptr;
  size_t st_ci_cap = 0;
  float* st_va = nullptr;
  size_t st_va_cap = 0;
  float* st_w0 = nullptr;  // [d]
  // state of the chains
  bool have_run = false;
  std::vector<long long> steps_done;
  std::vector<int> node_ids;
  std::vector<long long> last_steps;    // step counts of the launch being prepared
  std::vector<long long> steps_sorted;  // step counts that the estimates of a launch go by, largest first (see estimate_for)
  double steps_sum = 0.0;
  float eta0 = 0.f, lambda = 0.f;
  int sched = 0, loss = 0;
  uint64_t seed = 0;
  // options
  int opt_stages = 0;
  int opt_variant = 0, opt_prefetch = 0, opt_threads = 0, opt_cluster = 0;
  int opt_block_samples = 0;   // tensor-core cluster kernel: samples per block (0: chosen here, 8 or 16)
  int opt_sparse_variant = 0;  // 0: chosen here, 1: one step per round trip, 2: blocks of steps through a shared-memory cache
  long long opt_spin_limit = 1ll << 20;
  long long opt_drop_block = -1;
  int opt_sampling = 0;  // 0: i.i.d. draws, 1: one shuffle per node, cycled
  int opt_timing = 0;
  int opt_host_pipeline = 1;  // host-buffer entry point: copy the shards in groups and start chains as they arrive
  cudaStream_t copy_stream = nullptr;
  cudaEvent_t ev_fork = nullptr, ev_group[4] = {nullptr, nullptr, nullptr, nullptr};
  cudaEvent_t ev0 = nullptr, ev1 = nullptr;
  bool ev_valid = false;
  long long launches = 0;
  std::string err;
};

namespace wpsgd {

inline std::string g_err;  // last error of context-free calls

struct DeviceGuard {
  int prev = -1;
  explicit DeviceGuard(int dev) {
    if (cudaGetDevice(&prev) != cudaSuccess) prev = -1;
    if (prev != dev) cudaSetDevice(dev);
    else prev = -1;
  }
  ~DeviceGuard() {
    if (prev >= 0) cudaSetDevice(prev);
  }
};

inline wpsgd_status fail(wpsgd_ctx* c, wpsgd_status s, const std::string& msg) {
  if (c) c->err = msg;
  else g_err = msg;
  return s;
}

#define CU_TRY(ctx, expr)                                                                          \
  do {                                                                                             \
    cudaError_t e_ = (expr);                                                                       \
    if (e_ != cudaSuccess) {                                                                       \
      cudaGetLastError(); /* reported here, and not by the next call's look at the last error too */ \
      const bool oom_ = (e_ == cudaErrorMemoryAllocation);                                         \
      return fail(ctx, oom_ ? WPSGD_ERR_ALLOC : WPSGD_ERR_CUDA,                                    \
                  std::string(#expr) + ": " + cudaGetErrorString(e_));                             \
    }                                                                                              \
  } while (0)

template <typename T>
wpsgd_status grow(wpsgd_ctx* c, T** p, size_t* cap, size_t need) {
  if (need <= *cap) return WPSGD_OK;
  if (*p) {
    CU_TRY(c, cudaStreamSynchronize(c->stream));
    CU_TRY(c, cudaFree(*p));
    *p = nullptr;
    *cap = 0;
  }
  const size_t want = need + need / 8;
  void* q = nullptr;
  CU_TRY(c, cudaMalloc(&q, want * sizeof(T)));
  *p = (T*)q;
  *cap = want;
  return WPSGD_OK;
}

// Kernel launch that may start while the kernel before it on the stream ends (see kernel_started in common.cuh).
template <typename... P, typename... A>
cudaError_t launch(void (*kern)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t stream, A&&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, std::forward<A>(args)...);
}

inline bool aligned16(const void* p) { return (uintptr_t)p % 16 == 0; }

inline int grid_for(long long work_items, int block, int cap = 148 * 16) {
  long long g = (work_items + block - 1) / block;
  return (int)std::max(1ll, std::min<long long>(g, cap));
}

// Lets a kernel take up to all of an SM's shared memory. The limit belongs to the function and so to every thread and context of
// the process: set to the size of the launch at hand, a thread with a small ring lowered it between another's call and its
// launch, which was then refused. It is therefore only ever set to this one value; a launch names its own size.
constexpr size_t kSmemMax = 227 * 1024;
template <typename Kernel>
cudaError_t allow_all_smem(Kernel kern) {
  return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemMax);
}

}  // namespace wpsgd
