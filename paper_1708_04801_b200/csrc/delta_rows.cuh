// Chains whose labels are vectors, row by row (gated delta rule, see include/wpsgd.h): W <- e^g W, W <- W - beta (W k - v) k^T, o = scale W q.
//
// The models of a chain are heads_v dv rows of dk features that know nothing of each other, so heads are not looked at: model R
// = head dv + j has features and queries of its head, a label of its own, and dk numbers. Eight lanes have a model: lane s of them the features 4 (s + 8 i) to
// 4 (s + 8 i) + 3. The margin and the answer come from the same pass over the old model, o = e^g (w q) + delta (k q) with
// delta = beta (v - e^g (w k)), so one reduction over eight lanes (three sums together) is all that is serial.
#pragma once

#include "common.cuh"

namespace wpsgd {

constexpr int DELTA_MAX_D = 128;   // features and labels of a head at most
constexpr float DELTA_MIN_G = -128.0f;

struct DeltaRowsParams {
  const void *q, *k, *v, *g, *beta;
  long long ld_q, ld_k, ld_v, ld_g, ld_beta, ld_out;
  void* out;
  const float* W0;  // NULL: zeros
  float* W;         // may be NULL in a run of chains
  long long n_rows;
  const long long* shard_off;  // chains
  int n_chains;
  const int* slots;  // single rows
  long long n_slots;
  int hk, hv, dk, dv;
  float scale;
  int vec;  // features and models can be loaded four at a time
  DevStatus* status;
};

// four features from column c on, zeros behind dk
template <typename XT>
__device__ __forceinline__ void features4(const XT* row, int c, int dk, int vec, float (&f)[4]) {
  if (vec) {
    if (c < dk) {
      if constexpr (sizeof(XT) == 4) {
        const float4 r = __ldg((const float4*)(row + c));
        f[0] = r.x, f[1] = r.y, f[2] = r.z, f[3] = r.w;
      } else {
        const uint2 r = __ldg((const uint2*)(row + c));
        f[0] = __uint_as_float(r.x << 16), f[1] = __uint_as_float(r.x & 0xffff0000u), f[2] = __uint_as_float(r.y << 16), f[3] = __uint_as_float(r.y & 0xffff0000u);
      }
    } else {
      f[0] = f[1] = f[2] = f[3] = 0.0f;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = c + e < dk ? widen_scalar<XT>(row[c + e]) : 0.0f;
  }
}
template <typename XT>
__device__ __forceinline__ XT narrow_scalar(float v) {
  if constexpr (sizeof(XT) == 4) return v;
  else return __float2bfloat16_rn(v);
}
// models: read and written by the same thread, plain loads
__device__ __forceinline__ void model4(const float* row, int c, int dk, int vec, float* w) {
  if (vec) {
    float4 r = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (c < dk) r = *(const float4*)(row + c);
    w[0] = r.x, w[1] = r.y, w[2] = r.z, w[3] = r.w;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = c + e < dk ? row[c + e] : 0.0f;
  }
}
__device__ __forceinline__ void put_model4(float* row, int c, int dk, int vec, const float* w) {
  if (vec) {
    if (c < dk) *(float4*)(row + c) = make_float4(w[0], w[1], w[2], w[3]);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (c + e < dk) row[c + e] = w[e];
  }
}

__device__ __forceinline__ float sum8(float v) {
  v += __shfl_xor_sync(0xffffffffu, v, 1);
  v += __shfl_xor_sync(0xffffffffu, v, 2);
  return v + __shfl_xor_sync(0xffffffffu, v, 4);
}

// One row of one model: updates w (4 NJ features of this lane) and returns the answer (in all eight lanes).
template <int NJ>
__device__ __forceinline__ float delta_one_row(float (&w)[4 * NJ], const float (&k)[4 * NJ], const float (&q)[4 * NJ], float v, float g, float beta) {
  const float a = expf(g < DELTA_MIN_G ? DELTA_MIN_G : g);
  float wk = 0.0f, wq = 0.0f, kq = 0.0f;
#pragma unroll
  for (int e = 0; e < 4 * NJ; ++e) {
    w[e] *= a;
    wk = fmaf(w[e], k[e], wk);
    wq = fmaf(w[e], q[e], wq);
    kq = fmaf(k[e], q[e], kq);
  }
  wk = sum8(wk), wq = sum8(wq), kq = sum8(kq);
  const float delta = beta * (v - wk);
#pragma unroll
  for (int e = 0; e < 4 * NJ; ++e) w[e] = fmaf(delta, k[e], w[e]);
  return fmaf(delta, kq, wq);
}

// ---- chains, row by row ---------------------------------------------------------------------------------------------------------
// A warp has four models of a chain in registers and goes over the chain's rows. Bounds: the latency of a row (sums over eight lanes, about
// 150 cycles); the loads of the next rows are under way meanwhile.
constexpr int DELTA_WARPS = 4;

template <typename XT, int NJ>
__global__ void __launch_bounds__(32 * DELTA_WARPS) delta_rows_kernel(const __grid_constant__ DeltaRowsParams p) {
  constexpr int AHEAD = 4;  // rows whose loads are under way
  kernel_started();
  kernel_inputs_ready();
  const int lane = threadIdx.x & 31, s = lane & 7, models = p.hv * p.dv;
  const int groups = (models + 4 * DELTA_WARPS - 1) / (4 * DELTA_WARPS);
  const long long chain = blockIdx.x / groups;
  const int R = ((int)(blockIdx.x % groups) * DELTA_WARPS + (threadIdx.x >> 5)) * 4 + (lane >> 3);
  const bool there = R < models;
  const int h = there ? R / p.dv : 0, hk = h / (p.hv / p.hk);
  const long long first = p.shard_off[chain], end = p.shard_off[chain + 1];
  if (first < 0 || end < first || end > p.n_rows) {  // the same for the whole block; other chains may be in order, and run
    if (threadIdx.x == 0) set_status(p.status, DEV_BOUNDS, 22, chain);
    return;
  }
  float w[4 * NJ];
  const long long at = (chain * models + (there ? R : 0)) * p.dk;
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    if (p.W0 && there) model4(p.W0 + at, 4 * (s + 8 * j), p.dk, p.vec, w + 4 * j);
    else w[4 * j] = w[4 * j + 1] = w[4 * j + 2] = w[4 * j + 3] = 0.0f;
  }
  struct Row {
    float k[4 * NJ], q[4 * NJ], v, g, beta;
  } rows[AHEAD];
  auto load = [&](Row& r, long long t) {
    if (t >= end) return;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      float f[4];
      features4((const XT*)p.k + t * p.ld_k + hk * p.dk, 4 * (s + 8 * j), p.dk, p.vec, f);
      r.k[4 * j] = f[0], r.k[4 * j + 1] = f[1], r.k[4 * j + 2] = f[2], r.k[4 * j + 3] = f[3];
      features4((const XT*)p.q + t * p.ld_q + hk * p.dk, 4 * (s + 8 * j), p.dk, p.vec, f);
      r.q[4 * j] = f[0], r.q[4 * j + 1] = f[1], r.q[4 * j + 2] = f[2], r.q[4 * j + 3] = f[3];
    }
    r.v = widen_scalar<XT>(((const XT*)p.v)[t * p.ld_v + (there ? R : 0)]);
    r.g = widen_scalar<XT>(((const XT*)p.g)[t * p.ld_g + h]);
    r.beta = widen_scalar<XT>(((const XT*)p.beta)[t * p.ld_beta + h]);
  };
#pragma unroll
  for (int a = 0; a < AHEAD; ++a) load(rows[a], first + a);
  for (long long t = first; t < end; t += AHEAD) {
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
      if (t + a >= end) break;
      const float o = delta_one_row<NJ>(w, rows[a].k, rows[a].q, rows[a].v, rows[a].g, rows[a].beta);
      if (s == 0 && there) ((XT*)p.out)[(t + a) * p.ld_out + R] = narrow_scalar<XT>(p.scale * o);
      load(rows[a], t + a + AHEAD);
    }
  }
  if (p.W && there)
#pragma unroll
    for (int j = 0; j < NJ; ++j) put_model4(p.W + at, 4 * (s + 8 * j), p.dk, p.vec, w + 4 * j);
}

// ---- one row for each of many chains ------------------------------------------------------------------------------------------------
// A block has 32 RI models of a chain, all on their way from memory before the first is used. Bounds: bytes, the models once in and once out.
// A slot that an earlier row has is left to that row: every block looks through the slots before its own, which come from L2 while its models come from memory.
constexpr int STEP_THREADS = 256;

template <typename XT, int NJ, int RI>
__global__ void __launch_bounds__(STEP_THREADS) delta_step_kernel(const __grid_constant__ DeltaRowsParams p) {
  kernel_started();
  kernel_inputs_ready();
  const int lane = threadIdx.x & 31, s = lane & 7, models = p.hv * p.dv;
  const int groups = (models + 32 * RI - 1) / (32 * RI);
  const long long row = blockIdx.x / groups;
  const int R0 = (int)(blockIdx.x % groups) * 32 * RI + (threadIdx.x >> 5) * 4 + (lane >> 3);
  const long long slot = p.slots ? p.slots[row] : row;
  const bool valid = slot >= 0 && slot < p.n_slots;
  float w[RI][4 * NJ];
#pragma unroll
  for (int i = 0; i < RI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      w[i][4 * j] = w[i][4 * j + 1] = w[i][4 * j + 2] = w[i][4 * j + 3] = 0.0f;
      if (valid && R0 + 32 * i < models) model4(p.W + (slot * models + R0 + 32 * i) * p.dk, 4 * (s + 8 * j), p.dk, p.vec, w[i] + 4 * j);
    }
  int twice = 0;
  if (p.slots) {
    if (valid)
      for (long long r = threadIdx.x; r < row; r += STEP_THREADS) twice |= p.slots[r] == slot;
    twice = __syncthreads_or(twice);
  }
  if (!valid || twice) {
    if (threadIdx.x == 0 && (twice || slot >= p.n_slots)) set_status(p.status, DEV_BOUNDS, 23, row);
    return;
  }
#pragma unroll
  for (int i = 0; i < RI; ++i) {
    const int R = R0 + 32 * i;
    const bool there = R < models;
    const int h = there ? R / p.dv : 0, hk = h / (p.hv / p.hk);
    float k[4 * NJ], q[4 * NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      float f[4];
      features4((const XT*)p.k + row * p.ld_k + hk * p.dk, 4 * (s + 8 * j), p.dk, p.vec, f);
      k[4 * j] = f[0], k[4 * j + 1] = f[1], k[4 * j + 2] = f[2], k[4 * j + 3] = f[3];
      features4((const XT*)p.q + row * p.ld_q + hk * p.dk, 4 * (s + 8 * j), p.dk, p.vec, f);
      q[4 * j] = f[0], q[4 * j + 1] = f[1], q[4 * j + 2] = f[2], q[4 * j + 3] = f[3];
    }
    const float v = widen_scalar<XT>(((const XT*)p.v)[row * p.ld_v + (there ? R : 0)]);
    const float g = widen_scalar<XT>(((const XT*)p.g)[row * p.ld_g + h]), beta = widen_scalar<XT>(((const XT*)p.beta)[row * p.ld_beta + h]);
    const float o = delta_one_row<NJ>(w[i], k, q, v, g, beta);
    if (there) {
      if (s == 0) ((XT*)p.out)[row * p.ld_out + R] = narrow_scalar<XT>(p.scale * o);
#pragma unroll
      for (int j = 0; j < NJ; ++j) put_model4(p.W + (slot * models + R) * p.dk, 4 * (s + 8 * j), p.dk, p.vec, w[i] + 4 * j);
    }
  }
}

}  // namespace wpsgd
