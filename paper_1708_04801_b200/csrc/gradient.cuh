// Objective of Eq. 3-4, 0/1 error, and the gradient of the objective over all rows:
//
//   z_i = w . x_i,   out = { lambda / 2 |w|^2 + mean_i L(y_i, z_i),  share of rows with sign(z_i) != sign(y_i) },
//   grad = lambda w + mean_i L'(y_i, z_i) x_i.
//
// Rows fp32, bf16, or 8-bit with a scale for each block of 128 columns (x = scale q, as quantize.cuh makes them).
//
// One pass over the rows (gradient_rows_kernel): a group of threads holds R rows in registers, each thread its columns of them; the
// margins are summed over the group, and the same registers are then added, times L', to the thread's columns of the gradient. A group is a
// part of a warp for narrow rows and up to 16 warps for wide ones, so that a thread holds one to four 16-byte units of a row; the next R
// rows are requested before the present ones are worked on. Rows wider than that take two passes
// (gradient_margins_kernel, gradient_columns_kernel). Either way each block leaves a partial gradient, and
// gradient_finish_kernel adds those up in fp64 in block order. Nothing depends on timing.
//
// Hinge losses and signs jump: L' where y z = 1, the error where z = 0. The fp32 sum of a margin is off by at most
//   terms 2^-24 sum_c |w_c x_c|  <=  terms 2^-24 |w| |x|          (terms: length of the chain of additions a product takes part in)
// so a row whose margin is nearer than that to a jump has its margin formed again in fp64. |x|^2 costs one more multiply-add per
// element. The decisions are then those of exact products summed in fp64.
#pragma once

#include <cuda_fp8.h>

#include <type_traits>

#include "common.cuh"
#include "quantize.cuh"

namespace wpsgd {

constexpr int GRAD_THREADS = 256;
constexpr int GRAD_FINISH_WARPS = 16;

struct GradParams {
  const void* X;
  long long ld;          // elements of a row's storage
  const float* scales;   // 8-bit rows: [n_rows, ld_s]
  long long ld_s;
  const float* y;
  const float* w;
  long long n_rows, d;
  int loss;
  float* part;           // [blocks, d] partial gradients
  double* sums;          // [blocks, 2] losses and errors
};

// 16 bytes of a row, widened
struct Row8 {};  // tag of 8-bit rows
template <typename RT>
struct RowUnit {
  static constexpr int V = XVec<RT>::V;
  using Scalar = RT;
  __device__ __forceinline__ static void widen(const uint4& raw, float (&f)[V]) { XVec<RT>::widen(raw, f); }
};
template <>
struct RowUnit<Row8> {
  static constexpr int V = 16;
  using Scalar = uint8_t;
  __device__ __forceinline__ static float2 pair(uint32_t two) {  // exact: e4m3 is a subset of fp16
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)two));
    return __half22float2(*(const __half2*)&h);
  }
  __device__ __forceinline__ static void widen(const uint4& raw, float (&f)[16]) {
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 a = pair(w[i] & 0xffffu), b = pair(w[i] >> 16);
      f[4 * i] = a.x; f[4 * i + 1] = a.y; f[4 * i + 2] = b.x; f[4 * i + 3] = b.y;
    }
  }
};
template <typename RT>
__device__ __forceinline__ float row_element(const GradParams& p, long long row, long long c) {
  if constexpr (std::is_same<RT, Row8>::value) {
    const float2 v = RowUnit<Row8>::pair(((const uint8_t*)p.X)[row * p.ld + c]);
    return v.x * p.scales[row * p.ld_s + c / Q_BLOCK];
  } else {
    return widen_scalar<RT>(((const RT*)p.X)[row * p.ld + c]);
  }
}
// w_c x_c, exact for fp32 and bf16 rows; for 8-bit rows rounded once to fp64
template <typename RT>
__device__ __forceinline__ double exact_product(const GradParams& p, long long row, long long c) {
  if constexpr (std::is_same<RT, Row8>::value) {
    const float2 v = RowUnit<Row8>::pair(((const uint8_t*)p.X)[row * p.ld + c]);
    return (double)p.w[c] * ((double)v.x * (double)p.scales[row * p.ld_s + c / Q_BLOCK]);
  } else {
    return (double)p.w[c] * (double)widen_scalar<RT>(((const RT*)p.X)[row * p.ld + c]);
  }
}

// Bound of the fp32 margin's error, see above. 1.01: the norms are fp32 sums themselves; 2^-120: products below fp32's range.
__device__ __forceinline__ float margin_error(float terms, float w_norm, float x_squares) {
  return w_norm > 0.0f ? fmaf(terms * 0x1p-24f * 1.01f * w_norm, sqrtf(x_squares), 0x1p-120f) : 0.0f;
}
// Whether an error of `err` in z could move the row across a jump of the loss's derivative or of the sign.
__device__ __forceinline__ bool near_jump(int loss, float y, float z, float err) {
  if (fabsf(z) < err) return true;
  return loss == LOSS_HINGE && fabsf(1.0f - y * z) < fmaf(fabsf(y), err, 0x1p-22f);
}
// A margin that is not a number gives a derivative and a loss that are none, whatever the loss.
__device__ __forceinline__ float loss_derivative_f64(int loss, float y, double z) {
  if (isnan(z)) return (float)z;
  if (loss == LOSS_HINGE) return (double)y * z < 1.0 ? -y : 0.0f;
  return loss_derivative(loss, y, (float)z);
}

// |w| by a block, to every thread (any block size of whole warps up to 512)
__device__ __forceinline__ float block_w_norm(const float* __restrict__ w, long long d, double* sh) {
  double s = 0.0;
  for (long long c = threadIdx.x; c < d; c += blockDim.x) s = fma((double)w[c], (double)w[c], s);
  s = warp_sum_f64(s);
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = s;
  __syncthreads();
  double t = 0.0;
  for (int i = 0; i < (int)blockDim.x / 32; ++i) t += sh[i];
  __syncthreads();
  return (float)sqrt(t) * 1.0001f;
}

// ---- rows of any width: two passes ---------------------------------------------------------------------------------------
// Rows row0 .. row0 + count - 1: their L' to coef, losses and errors to sums (added to what is there unless `first`). A warp per row.
template <typename RT>
__global__ void __launch_bounds__(GRAD_THREADS) gradient_margins_kernel(const GradParams p, long long row0, long long count, bool first,
                                                                        float* __restrict__ coef) {
  __shared__ double sh[2][GRAD_THREADS / 32];
  kernel_started();
  kernel_inputs_ready();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const float w_norm = block_w_norm(p.w, p.d, sh[0]);
  const float terms = (float)((p.d + 31) / 32 + 8);
  double loss = 0.0, wrong = 0.0;
  for (long long i = (long long)blockIdx.x * (GRAD_THREADS / 32) + warp; i < count; i += (long long)gridDim.x * (GRAD_THREADS / 32)) {
    const long long row = row0 + i;
    float z = 0.0f, xx = 0.0f;
#pragma unroll 8
    for (long long c = lane; c < p.d; c += 32) {
      const float x = row_element<RT>(p, row, c);
      z = fmaf(p.w[c], x, z);
      xx = fmaf(x, x, xx);
    }
    z = warp_sum(z);
    xx = warp_sum(xx);
    const float y = p.y[row];
    double zd = z;
    if (near_jump(p.loss, y, z, margin_error(terms, w_norm, xx))) {
      zd = 0.0;
      for (long long c = lane; c < p.d; c += 32) zd += exact_product<RT>(p, row, c);
      zd = warp_sum_f64(zd);
    }
    if (lane == 0) {
      coef[i] = loss_derivative_f64(p.loss, y, zd);
      loss += isnan(zd) ? zd : loss_value(p.loss, y, zd);
      wrong += (zd >= 0.0) != (y >= 0.0f) ? 1.0 : 0.0;
    }
  }
  if (lane == 0) { sh[0][warp] = loss; sh[1][warp] = wrong; }
  __syncthreads();
  if (threadIdx.x < 2) {
    double t = 0.0;
    for (int i = 0; i < GRAD_THREADS / 32; ++i) t += sh[threadIdx.x][i];
    double* to = p.sums + 2 * blockIdx.x + threadIdx.x;
    *to = first ? t : *to + t;
  }
}

// Partial gradient `blockIdx.y` of the same rows: those of its share, a thread per column.
template <typename RT>
__global__ void __launch_bounds__(GRAD_THREADS) gradient_columns_kernel(const GradParams p, long long row0, long long count, bool first,
                                                                        const float* __restrict__ coef) {
  kernel_started();
  kernel_inputs_ready();
  const long long c = (long long)blockIdx.x * GRAD_THREADS + threadIdx.x;
  if (c >= p.d) return;
  const long long i0 = count * blockIdx.y / gridDim.y, i1 = count * (blockIdx.y + 1) / gridDim.y;
  float acc = 0.0f;
#pragma unroll 8
  for (long long i = i0; i < i1; ++i) acc = fmaf(coef[i], row_element<RT>(p, row0 + i, c), acc);
  float* to = p.part + blockIdx.y * p.d + c;
  *to = first ? acc : *to + acc;
}

// grad = lambda w + (sum of the partial gradients) / n, and the measures. A block owns 32 columns, its warps split the partials; the warps'
// sums are added in warp order. Block 0 also forms |w|^2 and adds up the blocks' losses and errors.
__global__ void __launch_bounds__(32 * GRAD_FINISH_WARPS) gradient_finish_kernel(const float* __restrict__ part, int parts, const double* __restrict__ sums, int n_sums,
                                                                                 const float* __restrict__ w, long long d, long long n_rows, float lambda,
                                                                                 float* __restrict__ grad, float* __restrict__ out) {
  __shared__ double sh[GRAD_FINISH_WARPS][33];
  kernel_started();
  kernel_inputs_ready();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long c = (long long)blockIdx.x * 32 + lane;
  double t = 0.0;
  if (c < d) {
#pragma unroll 4
    for (int i = warp; i < parts; i += GRAD_FINISH_WARPS) t += (double)__ldcg(part + (long long)i * d + c);
  }
  sh[warp][lane] = t;
  __syncthreads();
  const double n = n_rows > 0 ? (double)n_rows : 1.0;
  if (warp == 0 && c < d) {
    t = 0.0;
    for (int i = 0; i < GRAD_FINISH_WARPS; ++i) t += sh[i][lane];
    grad[c] = (float)fma((double)lambda, (double)w[c], t / n);
  }
  if (blockIdx.x != 0) return;
  __syncthreads();
  double ww = 0.0, loss = 0.0, wrong = 0.0;
  for (long long i = threadIdx.x; i < d; i += 32 * GRAD_FINISH_WARPS) ww = fma((double)w[i], (double)w[i], ww);
  for (int i = threadIdx.x; i < n_sums; i += 32 * GRAD_FINISH_WARPS) {
    loss += __ldcg(sums + 2 * i);
    wrong += __ldcg(sums + 2 * i + 1);
  }
  ww = warp_sum_f64(ww); loss = warp_sum_f64(loss); wrong = warp_sum_f64(wrong);
  if (lane == 0) { sh[warp][0] = ww; sh[warp][1] = loss; sh[warp][2] = wrong; }
  __syncthreads();
  if (threadIdx.x == 0) {
    ww = loss = wrong = 0.0;
    for (int i = 0; i < GRAD_FINISH_WARPS; ++i) { ww += sh[i][0]; loss += sh[i][1]; wrong += sh[i][2]; }
    out[0] = (float)(0.5 * (double)lambda * ww + loss / n);
    out[1] = (float)(wrong / n);
  }
}

}  // namespace wpsgd
