// Rows packed to 8 bits: e4m3 with a scale for each block of 128 columns.
//
//   a = max(2^-100, max |x_c| over the block),  q_c = e4m3(x_c * fl(448 / a)),  scale = fl(a / 448),   x_c ~ q_c * scale
//
// 448 is the largest e4m3 value, so the largest magnitude of a block uses the whole range. The lower limit of `a` keeps 448 / a
// finite for blocks of zeros or of subnormal numbers. Each q is rounded twice, to 24 bits by the product (2^-24 of it) and to
// e4m3's 4 bits (2^-4): the product instead of a division costs one instruction instead of ten and moves a value across a rounding border of
// e4m3 in one of 2 million codes of fp32 rows, and in one of 4100 of bf16 rows, whose quotients are exact ties in 0.5 % of the cases (counted on
// 16.8 million normal values). The quotient 448 / a is the nearest fp32; 448 times a rounded 1 / a would miss that in a quarter of the blocks and change
// 0.08 % of the codes of bf16 rows. An infinity makes the scale infinite and its block NaN or 0
// (0 * infinity is NaN again in every margin); a NaN stays a NaN and does not enter `a`.
// Bound by memory: reads 4 or 2 bytes per element, writes 1. 131072 bf16 rows of 4096 columns: 311 us, 5.3 TB/s.
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

// Largest magnitude of a 16-byte unit, NaNs left out; bf16 two at a time
__device__ __forceinline__ float abs_max(const uint4& raw, float) {
  return fmaxf(fmaxf(fabsf(__uint_as_float(raw.x)), fabsf(__uint_as_float(raw.y))), fmaxf(fabsf(__uint_as_float(raw.z)), fabsf(__uint_as_float(raw.w))));
}
__device__ __forceinline__ float abs_max(const uint4& raw, __nv_bfloat16) {
  auto pair = [](uint32_t w) { return __habs2(*(const __nv_bfloat162*)&w); };
  const __nv_bfloat162 m = __hmax2(__hmax2(pair(raw.x), pair(raw.y)), __hmax2(pair(raw.z), pair(raw.w)));
  return fmaxf(__low2float(m), __high2float(m));
}

// U blocks at a time per group of G lanes: lane g < U divides 448 / a of block g, lane U + g the scale a / 448, so that two divisions of ten
// instructions are done once and not by every lane. `a` is left in all lanes of the group.
template <int U, int G>
__device__ __forceinline__ void block_scales(float (&a)[U], float (&inv)[U], float& scale, int gl) {
  static_assert(2 * U <= G, "a lane for each division");
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int o = G / 2; o > 0; o >>= 1) a[u] = fmaxf(a[u], __shfl_xor_sync(0xffffffffu, a[u], o));
  float own = a[0];
#pragma unroll
  for (int u = 1; u < U; ++u) own = gl % U == u ? a[u] : own;
  scale = gl < U ? Q_MAX / own : own / Q_MAX;
#pragma unroll
  for (int u = 0; u < U; ++u) inv[u] = __shfl_sync(0xffffffffu, scale, u, G);
}

// The blocks (row, block of columns) first, first + apart, .. first + (U - 1) apart of all rows' blocks, and on by `stride` each step,
// without a division per step.
template <int U>
struct BlockWalk {
  long long row[U], rows_per_step;
  int block[U], blocks_per_step;
  __device__ __forceinline__ BlockWalk(long long first, int apart, long long stride, int nb) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      row[u] = row_of(first + u * apart, nb);
      block[u] = (int)(first + u * apart - row[u] * nb);
    }
    rows_per_step = row_of(stride, nb);
    blocks_per_step = (int)(stride - rows_per_step * nb);
  }
  __device__ __forceinline__ void step(int nb) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      row[u] += rows_per_step;
      block[u] += blocks_per_step;
      if (block[u] >= nb) { block[u] -= nb; ++row[u]; }
    }
  }
};

// Rows that start on 16 bytes: a group of 128 / V lanes per block, each lane V elements of it in one 16-byte load and one store of V
// bytes. U blocks in flight per group.
template <typename XT, int U>
__global__ void __launch_bounds__(256) quantize_rows_kernel(const XT* __restrict__ X, long long ld, long long n_rows, long long d, int nb,
                                                            uint8_t* __restrict__ Q, long long ld_q, float* __restrict__ scales, long long ld_s) {
  kernel_started();
  kernel_inputs_ready();
  constexpr int V = XVec<XT>::V, G = Q_BLOCK / V, PER_WARP = 32 / G;
  const int lane = threadIdx.x & 31, gl = lane % G;
  BlockWalk<U> at(((long long)blockIdx.x * 8 + (threadIdx.x >> 5)) * (PER_WARP * U) + lane / G, PER_WARP, (long long)gridDim.x * 8 * (PER_WARP * U), nb);
  for (; __any_sync(0xffffffffu, at.row[0] < n_rows); at.step(nb)) {
    uint4 raw[U];
    bool in[U];  // this lane has a part of a row
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c = at.block[u] * Q_BLOCK + gl * V;
      in[u] = at.row[u] < n_rows && c < d;
      raw[u] = ld_stream16_if(X + at.row[u] * ld + c, in[u]);
    }
    float a[U], inv[U], scale;
#pragma unroll
    for (int u = 0; u < U; ++u) a[u] = fmaxf(Q_AMAX_MIN, abs_max(raw[u], XT()));
    block_scales<U, G>(a, inv, scale, gl);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float x[V];
      XVec<XT>::widen(raw[u], x);
      uint32_t q[V / 4];
#pragma unroll
      for (int e = 0; e < V; e += 4) {
        const uint32_t lo = to_e4m3x2(x[e] * inv[u], x[e + 1] * inv[u]), hi = to_e4m3x2(x[e + 2] * inv[u], x[e + 3] * inv[u]);
        q[e / 4] = lo | hi << 16;
      }
      if (in[u]) {
        uint8_t* dst = Q + at.row[u] * ld_q + at.block[u] * Q_BLOCK + gl * V;
        if constexpr (V == 8) *(uint2*)dst = make_uint2(q[0], q[1]);
        else *(uint32_t*)dst = q[0];
      }
      if (gl == U + u && at.row[u] < n_rows) scales[at.row[u] * ld_s + at.block[u]] = scale;
    }
  }
}

// Any other rows: a warp per block, lane l the columns l, l + 32, l + 64, l + 96 (neighbouring lanes load neighbouring elements), whose
// codes it exchanges for those of columns 4 l to 4 l + 3.
template <typename XT, int U>
__global__ void __launch_bounds__(256) quantize_elements_kernel(const XT* __restrict__ X, long long ld, long long n_rows, long long d, int nb,
                                                                uint8_t* __restrict__ Q, long long ld_q, float* __restrict__ scales, long long ld_s) {
  kernel_started();
  kernel_inputs_ready();
  const int lane = threadIdx.x & 31;
  BlockWalk<U> at(((long long)blockIdx.x * 8 + (threadIdx.x >> 5)) * U, 1, (long long)gridDim.x * 8 * U, nb);
  for (; at.row[0] < n_rows; at.step(nb)) {
    float x[U][4], a[U], inv[U], scale;
    int left[U];  // columns of the block
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long rest = d - (long long)at.block[u] * Q_BLOCK;
      left[u] = at.row[u] < n_rows ? (int)(rest < Q_BLOCK ? rest : Q_BLOCK) : 0;
      a[u] = Q_AMAX_MIN;
      const XT* src = X + at.row[u] * ld + at.block[u] * Q_BLOCK + lane;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[u][e] = lane + 32 * e < left[u] ? widen_scalar<XT>(src[32 * e]) : 0.0f;
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) a[u] = fmaxf(a[u], fabsf(x[u][e]));
    block_scales<U, 32>(a, inv, scale, lane);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t q = to_e4m3x2(x[u][0] * inv[u], x[u][1] * inv[u]) | to_e4m3x2(x[u][2] * inv[u], x[u][3] * inv[u]) << 16;
      uint32_t w = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) w |= (__shfl_sync(0xffffffffu, q, lane % 8 * 4 + i) >> lane / 8 * 8 & 0xffu) << 8 * i;
      uint8_t* dst = Q + at.row[u] * ld_q + at.block[u] * Q_BLOCK + 4 * lane;
      if (4 * lane + 4 <= left[u]) {
        *(uint32_t*)dst = w;
      } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
          if (4 * lane + i < left[u]) dst[i] = (uint8_t)(w >> 8 * i);
      }
      if (lane == U + u && left[u] > 0) scales[at.row[u] * ld_s + at.block[u]] = scale;
    }
  }
}

}  // namespace wpsgd
