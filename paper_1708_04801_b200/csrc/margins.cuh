// Margins of many models on many rows, both 8-bit with a scale for each block of 128 columns:
//   Z[i, m] = sum_b s_i,b t_m,b sum_{c in block b} q_i,c p_m,c
#pragma once

#include <cuda_fp8.h>

#include "common.cuh"
#include "gradient.cuh"

namespace wpsgd {

template <typename OT>
__device__ __forceinline__ OT narrow_to(float v);
template <>
__device__ __forceinline__ float narrow_to<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 narrow_to<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// 64 x 64 margins per block of 256 threads, 4 x 4 per thread, the columns in blocks of 128.
template <typename OT>
__global__ void __launch_bounds__(256) margins_kernel(const uint8_t* __restrict__ Q, long long ld_q, const float* __restrict__ qs, long long ld_qs, long long n_rows,
                                                      const uint8_t* __restrict__ M, long long ld_m, const float* __restrict__ ms, long long ld_ms, long long n_models,
                                                      long long d, OT* __restrict__ Z, long long ld_z) {
  extern __shared__ float sh[];  // [2][64][129]
  kernel_started();
  kernel_inputs_ready();
  float* a = sh;
  float* b = sh + 64 * 129;
  const long long i0 = (long long)blockIdx.x * 64, m0 = (long long)blockIdx.y * 64;
  const int ti = threadIdx.x / 16, tm = threadIdx.x % 16;
  float acc[4][4] = {};
  for (long long c0 = 0; c0 < d; c0 += Q_BLOCK) {
    for (int e = threadIdx.x; e < 64 * Q_BLOCK; e += 256) {
      const int r = e / Q_BLOCK, c = e % Q_BLOCK;
      a[r * 129 + c] = i0 + r < n_rows && c0 + c < d ? RowUnit<Row8>::pair(Q[(i0 + r) * ld_q + c0 + c]).x : 0.0f;
      b[r * 129 + c] = m0 + r < n_models && c0 + c < d ? RowUnit<Row8>::pair(M[(m0 + r) * ld_m + c0 + c]).x : 0.0f;
    }
    __syncthreads();
    float dot[4][4] = {};
    for (int c = 0; c < Q_BLOCK; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int m = 0; m < 4; ++m) dot[i][m] = fmaf(a[(ti + 16 * i) * 129 + c], b[(tm + 16 * m) * 129 + c], dot[i][m]);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        const long long r = i0 + ti + 16 * i, n = m0 + tm + 16 * m;
        if (r < n_rows && n < n_models) acc[i][m] = fmaf(dot[i][m], qs[r * ld_qs + c0 / Q_BLOCK] * ms[n * ld_ms + c0 / Q_BLOCK], acc[i][m]);
      }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const long long r = i0 + ti + 16 * i, n = m0 + tm + 16 * m;
      if (r < n_rows && n < n_models) Z[r * ld_z + n] = narrow_to<OT>(acc[i][m]);
    }
}

}  // namespace wpsgd
