// Rows packed to 8 bits: e4m3 with a scale for each block of 128 columns.
//
//   a = max(2^-100, max |x_c| over the block),  q_c = e4m3(x_c * fl(448 / a)),  scale = fl(a / 448),   x_c ~ q_c * scale
//
// 448 is the largest e4m3 value, so the largest magnitude of a block uses the whole range. The lower limit of `a` keeps 448 / a
// finite for blocks of zeros or of subnormal numbers. Each q is rounded twice, to 24 bits by the product (2^-24 of it) and to
// e4m3's 4 bits (2^-4): the product instead of a division moves a value across a rounding border of e4m3 in about one of 2^20
// cases, and costs one instruction where the division costs ten. An infinity makes the scale infinite and its block NaN or 0
// (0 * infinity is NaN again in every margin); a NaN stays a NaN and does not enter `a`.
// Bound by memory: reads 4 or 2 bytes per element, writes 1.
#pragma once

#include <cuda_fp8.h>

#include "common.cuh"

namespace wpsgd {

constexpr int Q_BLOCK = 128;            // columns that share a scale
constexpr float Q_MAX = 448.0f;         // largest e4m3 value
constexpr float Q_AMAX_MIN = 0x1p-100f;

// two fp32 -> two e4m3 (lo in the low byte), nearest even; beyond 448 (by the rounding of the product only) -> 448, NaN -> NaN
__device__ __forceinline__ uint32_t to_e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}

// A group of 128 / V lanes per block, each lane V elements of it: one 16-byte load and one store of V bytes. VEC = false (rows that do
// not start on 16 bytes, or whose last 16 bytes are not whole): the same lanes and elements, loaded one by one.
template <typename XT, bool VEC, int U>
__global__ void __launch_bounds__(256) quantize_rows_kernel(const XT* __restrict__ X, long long ld, long long n_rows, long long d, int nb,
                                                            uint8_t* __restrict__ Q, long long ld_q, float* __restrict__ scales, long long ld_s) {
  kernel_started();
  kernel_inputs_ready();
  constexpr int V = XVec<XT>::V, G = Q_BLOCK / V, PER_WARP = 32 / G;
  const int lane = threadIdx.x & 31, gl = lane % G;
  const long long warps = (long long)gridDim.x * 8, total = n_rows * nb;
  for (long long t0 = ((long long)blockIdx.x * 8 + (threadIdx.x >> 5)) * (PER_WARP * U); t0 < total; t0 += warps * (PER_WARP * U)) {
    float x[U][V];
    long long row[U], c[U];
    bool in[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long t = t0 + u * PER_WARP + lane / G;
      in[u] = t < total;
      row[u] = in[u] ? row_of(t, nb) : 0;
      c[u] = (t - row[u] * nb) * Q_BLOCK + gl * V;
      if constexpr (VEC) {
        XVec<XT>::widen(ld_stream16_if(X + row[u] * ld + c[u], in[u] && c[u] < d), x[u]);
      } else {
#pragma unroll
        for (int e = 0; e < V; ++e) x[u][e] = in[u] && c[u] + e < d ? widen_scalar<XT>(X[row[u] * ld + c[u] + e]) : 0.0f;
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float a = Q_AMAX_MIN;
#pragma unroll
      for (int e = 0; e < V; ++e) a = fmaxf(a, fabsf(x[u][e]));
#pragma unroll
      for (int o = G / 2; o > 0; o >>= 1) a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, o));
      const float inv = Q_MAX / a;
      uint32_t q[V / 4];
#pragma unroll
      for (int e = 0; e < V; e += 4) {
        const uint32_t lo = to_e4m3x2(x[u][e] * inv, x[u][e + 1] * inv), hi = to_e4m3x2(x[u][e + 2] * inv, x[u][e + 3] * inv);
        q[e / 4] = lo | hi << 16;
      }
      if (in[u] && c[u] < d) {
        uint8_t* dst = Q + row[u] * ld_q + c[u];
        if (VEC || c[u] + V <= d) {
          if constexpr (V == 8) *(uint2*)dst = make_uint2(q[0], q[1]);
          else *(uint32_t*)dst = q[0];
        } else {
#pragma unroll
          for (int e = 0; e < V; ++e)
            if (c[u] + e < d) dst[e] = (uint8_t)(q[e / 4] >> 8 * (e % 4));
        }
        if (gl == 0) scales[row[u] * ld_s + c[u] / Q_BLOCK] = a / Q_MAX;
      }
    }
  }
}

}  // namespace wpsgd
