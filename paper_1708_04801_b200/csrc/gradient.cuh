// Objective of Eq. 3-4, 0/1 error, and the gradient of the objective over all rows:
//
//   z_i = w . x_i,   out = { lambda / 2 |w|^2 + mean_i L(y_i, z_i),  share of rows with sign(z_i) != sign(y_i) },
//   grad = lambda w + mean_i L'(y_i, z_i) x_i.
//
// Rows fp32, bf16, or 8-bit with a scale for each block of 128 columns (x = scale q, as quantize.cuh makes them).
//
// One pass over the rows (gradient_rows_kernel): a group of threads takes R rows at a time from shared memory, each thread its columns of them;
// the margins are summed over the group, and the rows are then read again and added, times L', to the gradient, whose columns each
// thread keeps in registers. A group is a part of a warp for narrow rows and up to 16 warps for wide ones, so that a thread has one to
// four 16-byte units of a row; the rows after the next are requested while the present ones are worked on. Rows wider than that (16384 columns, fp32 8192) take two passes
// (gradient_margins_kernel, gradient_columns_kernel). Either way each block leaves a partial gradient, and
// gradient_finish_kernel adds those up in fp64 in block order. Nothing depends on timing.
//
// Bound by the read of the rows as far as the instructions allow: two packed multiply-adds per pair of elements for the margin and its
// bound, one for the gradient, and the widening of bf16 and 8-bit values, twice, because widened rows would not fit the registers.
// 131072 fp32 rows of 4096 columns 335 us (6.4 TB/s), 262144 bf16 rows 402 to 450 us (5.3 to 4.8 TB/s, the less the longer the GPU has been at work), 131072 8-bit rows of 999 columns
// 62 us (2.2 TB/s: about 160 instructions per 16 elements).
//
// Hinge losses and signs jump: L' where y z = 1, the error where z = 0. The fp32 sum of a margin is off by at most
//   terms 2^-24 sum_c |w_c x_c|  <=  terms 2^-24 |w| |x|          (terms: length of the chain of additions a product takes part in)
// so a row whose margin is nearer than that to a jump has its margin formed again in fp64. |x|^2 costs one more multiply-add per
// element. The decisions are then those of exact products summed in fp64.
#pragma once

#include <cuda_fp8.h>

#include <algorithm>
#include <type_traits>

#include "async.cuh"
#include "common.cuh"
#include "quantize.cuh"

namespace wpsgd {

constexpr int GRAD_THREADS = 256;
constexpr int GRAD_FINISH_WARPS = 16;
constexpr int GRAD_LAST_BLOCK = 8192;  // up to so many elements of partial gradients, the block that finishes last adds them up

struct GradParams {
  const void* X;
  long long ld;          // elements of a row's storage
  const float* scales;   // 8-bit rows: [n_rows, ld_s]
  long long ld_s;
  const float* y;
  const float* w;
  long long n_rows, d;
  int loss;
  float lambda;
  float* grad;           // [d]
  float* out;            // [2]
  float* part;           // [blocks, d] partial gradients
  double* sums;          // [blocks, 2] losses and errors
  unsigned* ticket;      // blocks that have finished (zero between launches); null: gradient_finish_kernel follows
  int slots;             // of a ring (FEED_BULK)
  long long spin_limit, drop_block;
  DevStatus* status;
};

// 16 bytes of a row, widened to pairs
struct Row8 {};  // tag of 8-bit rows
template <typename RT>
struct RowUnit {
  static constexpr int V = XVec<RT>::V;
  using Scalar = RT;
  __device__ __forceinline__ static void widen(const uint4& raw, uint64_t (&f)[V / 2]) {
    float x[V];
    XVec<RT>::widen(raw, x);
#pragma unroll
    for (int i = 0; i < V / 2; ++i) f[i] = pair_of(__float_as_uint(x[2 * i]), __float_as_uint(x[2 * i + 1]));
  }
};
template <>
struct RowUnit<Row8> {  // (never element by element)
  static constexpr int V = 16;
  using Scalar = uint8_t;
  __device__ __forceinline__ static float2 pair(uint32_t two) {  // exact: e4m3 is a subset of fp16
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)two));
    return __half22float2(*(const __half2*)&h);
  }
  __device__ __forceinline__ static void widen(const uint4& raw, uint64_t (&f)[8]) {
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 a = pair(w[i] & 0xffffu), b = pair(w[i] >> 16);
      f[2 * i] = pair_of(__float_as_uint(a.x), __float_as_uint(a.y));
      f[2 * i + 1] = pair_of(__float_as_uint(b.x), __float_as_uint(b.y));
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

// Bound of the fp32 margin's error, see above. 1.01: the norms are fp32 sums themselves, and the root may be off by 2^-10;
// 2^-110: squares below fp32's range, of which each loses 2^-150 at most (2^40 of them); 2^-120: products below it.
__device__ __forceinline__ float margin_error(float terms, float w_norm, float x_squares) {
  float root;
  asm("sqrt.approx.f32 %0, %1;" : "=f"(root) : "f"(x_squares + 0x1p-110f));
  return w_norm > 0.0f ? fmaf(terms * 0x1p-24f * 1.01f * w_norm, root, 0x1p-120f) : 0.0f;
}
// Whether an error of `err` in z could move the row across a jump of the loss's derivative or of the sign, or its sum has left fp32
// on the way (the margin itself may lie within).
__device__ __forceinline__ bool near_jump(int loss, float y, float z, float err) {
  if (!(fabsf(z) >= err && fabsf(z) < INFINITY)) return true;
  return loss == LOSS_HINGE && fabsf(1.0f - y * z) < fmaf(fabsf(y), err, 0x1p-22f);
}
// A margin or label that is not a number gives a derivative and a loss that are none, whatever the loss.
__device__ __forceinline__ double loss_of(int loss, float y, double z) {
  return isnan(z + (double)y) ? z + (double)y : loss_value(loss, y, z);
}
// L' of a row whose margin no rounding can move across a jump
__device__ __forceinline__ float row_derivative(int loss, float y, float z) {
  const float t = y * z;
  if (loss == LOSS_HINGE) return t < 1.0f ? -y : t >= 1.0f ? 0.0f : t;
  if (loss == LOSS_LOGISTIC) return __fdividef(-y, 1.0f + expf(t));  // off by 2^-22 at most, and 0 instead of values below 2^-126
  return z - y;
}
// and by the margin in fp64
__device__ __forceinline__ float row_derivative(int loss, float y, double z) {
  if (loss != LOSS_HINGE) return row_derivative(loss, y, (float)z);
  const double t = (double)y * z;
  return t < 1.0 ? -y : t >= 1.0 ? 0.0f : (float)t;
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

// grad = lambda w + (sum of the partial gradients) / n for columns 32 slab and on, and for slab 0 the measures. The block's warps split
// the partials, the warps' sums are added in warp order: the same result whichever block does it.
template <int WARPS>
__device__ __forceinline__ void gradient_finish(const GradParams& p, int parts, int n_sums, int slab, double (*sh)[33]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long c = (long long)slab * 32 + lane;
  double t = 0.0;
  if (c < p.d) {
#pragma unroll 8
    for (int i = warp; i < parts; i += WARPS) t += (double)__ldcg(p.part + (long long)i * p.d + c);
  }
  __syncthreads();
  sh[warp][lane] = t;
  __syncthreads();
  const double n = p.n_rows > 0 ? (double)p.n_rows : 1.0;
  if (warp == 0 && c < p.d) {
    t = 0.0;
    for (int i = 0; i < WARPS; ++i) t += sh[i][lane];
    p.grad[c] = (float)fma((double)p.lambda, (double)p.w[c], t / n);
  }
  if (slab != 0) return;
  __syncthreads();
  double ww = 0.0, loss = 0.0, wrong = 0.0;
  for (long long i = threadIdx.x; i < p.d; i += 32 * WARPS) ww = fma((double)p.w[i], (double)p.w[i], ww);
  for (int i = threadIdx.x; i < n_sums; i += 32 * WARPS) {
    loss += __ldcg(p.sums + 2 * i);
    wrong += __ldcg(p.sums + 2 * i + 1);
  }
  ww = warp_sum_f64(ww); loss = warp_sum_f64(loss); wrong = warp_sum_f64(wrong);
  if (lane == 0) { sh[warp][0] = ww; sh[warp][1] = loss; sh[warp][2] = wrong; }
  __syncthreads();
  if (threadIdx.x == 0) {
    ww = loss = wrong = 0.0;
    for (int i = 0; i < WARPS; ++i) { ww += sh[i][0]; loss += sh[i][1]; wrong += sh[i][2]; }
    p.out[0] = (float)(0.5 * (double)p.lambda * ww + loss / n);
    p.out[1] = (float)(wrong / n);
  }
}
// The same by one block of WARPS warps for all of few columns: slabs side by side, one barrier.
template <int WARPS>
__device__ __forceinline__ void gradient_finish_small(const GradParams& p, int parts, int n_sums, double (*sh)[36]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int slabs = (int)((p.d + 31) / 32), per_slab = WARPS / slabs > 1 ? WARPS / slabs : 1, first = warp / per_slab, step = WARPS / per_slab;
  const double n = p.n_rows > 0 ? (double)p.n_rows : 1.0;
  double ww = 0.0, loss = 0.0, wrong = 0.0;
  for (long long i = threadIdx.x; i < p.d; i += 32 * WARPS) ww = fma((double)p.w[i], (double)p.w[i], ww);
  for (int i = threadIdx.x; i < n_sums; i += 32 * WARPS) {
    loss += __ldcg(p.sums + 2 * i);
    wrong += __ldcg(p.sums + 2 * i + 1);
  }
  for (int slab = first; slab < slabs; slab += step) {  // more than once only where a warp has a slab to itself
    const long long c = (long long)slab * 32 + lane;
    double t = 0.0;
    if (c < p.d) {
#pragma unroll 8
      for (int i = warp % per_slab; i < parts; i += per_slab) t += (double)__ldcg(p.part + (long long)i * p.d + c);
      if (per_slab == 1) p.grad[c] = (float)fma((double)p.lambda, (double)p.w[c], t / n);
    }
    sh[warp][lane] = t;
  }
  ww = warp_sum_f64(ww); loss = warp_sum_f64(loss); wrong = warp_sum_f64(wrong);
  if (lane == 0) { sh[warp][32] = ww; sh[warp][33] = loss; sh[warp][34] = wrong; }
  __syncthreads();
  if (per_slab > 1 && warp % per_slab == 0 && first < slabs) {
    const long long c = (long long)first * 32 + lane;
    double t = 0.0;
    for (int i = 0; i < per_slab; ++i) t += sh[warp + i][lane];
    if (c < p.d) p.grad[c] = (float)fma((double)p.lambda, (double)p.w[c], t / n);
  }
  if (threadIdx.x == 0) {
    ww = loss = wrong = 0.0;
    for (int i = 0; i < WARPS; ++i) { ww += sh[i][32]; loss += sh[i][33]; wrong += sh[i][34]; }
    p.out[0] = (float)(0.5 * (double)p.lambda * ww + loss / n);
    p.out[1] = (float)(wrong / n);
  }
}
__global__ void __launch_bounds__(32 * GRAD_FINISH_WARPS) gradient_finish_kernel(const __grid_constant__ GradParams p, int parts, int n_sums) {
  __shared__ double sh[GRAD_FINISH_WARPS][33];
  kernel_started();
  kernel_inputs_ready();
  gradient_finish<GRAD_FINISH_WARPS>(p, parts, n_sums, blockIdx.x, sh);
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
      coef[i] = row_derivative(p.loss, y, zd);
      loss += loss_of(p.loss, y, zd);
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

// ---- rows that a group of threads holds in registers: one pass ----------------------------------------------------------------
// Sums over the lanes of each row group of R rows at a time: halves the rows a lane answers for at every step, so that R sums over L lanes take
// about R + log2(L / R) exchanges. Lane l of its L ends with the sum of row (l / (L / R)).
template <int R, int L>
__device__ __forceinline__ float transpose_sum(float (&v)[R], int l) {
  static_assert(R <= L, "a lane for each row");
#pragma unroll
  for (int o = L / 2, n = R / 2; o > 0; o >>= 1, n >>= 1) {
    if (n > 0) {
      const bool upper = (l & o) != 0;
#pragma unroll
      for (int i = 0; i < R / 2; ++i)
        if (i < n) {
          const float mine = upper ? v[i + n] : v[i], other = upper ? v[i] : v[i + n];
          v[i] = mine + __shfl_xor_sync(0xffffffffu, other, o);
        }
    } else {
      v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
    }
  }
  return v[0];
}

// How rows reach the threads that work on them.
enum RowFeed {
  FEED_ELEMENTS = 0,  // element by element into registers: rows that do not start on 16 bytes
  FEED_UNITS = 1,     // each thread its own 16-byte units (cp.async), with their scales: 8-bit rows, and others whose last unit is not whole
  FEED_BULK = 2       // whole rows in bulk copies. 65536 bf16 rows of 4096 columns: by units 109 us without any work on them, in bulk 94
};

// G threads per row, each CH units of 16 bytes of it (or the same number of single elements); R rows at a time.
template <typename RT, int FEED, int G, int CH, int R>
struct GradShape {
  static constexpr int V = RowUnit<RT>::V;
  static constexpr bool scaled = std::is_same<RT, Row8>::value;
  static constexpr int threads = G > GRAD_THREADS ? G : GRAD_THREADS;
  static constexpr int per_sm = threads > GRAD_THREADS ? 1 : 2;
  static constexpr int groups = threads / G;       // of a block
  static constexpr int lanes = G < 32 ? G : 32;    // of a warp that work on the same rows
  static constexpr int warps = G < 32 ? 1 : G / 32;
  static constexpr int budget = 110 * 1024 * 2 / per_sm;  // of shared memory: three slots of 32 KB (with two, 131072 fp32 rows of 4096 columns take 414 us, not 335)
  // FEED_UNITS: slots of R rows, each thread's part of them its own
  static constexpr int unit_slot_bytes = threads * R * CH * (scaled ? 20 : 16);
  static constexpr int unit_slots = budget / unit_slot_bytes;
  // FEED_BULK: rings of slots of `rows` rows, a ring per group, or per warp where groups are smaller; 16 zeros in front
  static constexpr int rings = threads / 32 / warps, rows = R * (32 / lanes);
  static int bulk_slots(long long row_bytes) { return (int)std::min<long long>(8, (budget - 16) / (rings * rows * row_bytes)); }
  static constexpr int fold_bytes = groups > 1 ? threads * CH * V * 4 : 0;
  static constexpr int finish_bytes = threads / 32 * 36 * 8;
  static int smem(long long row_bytes) {
    const int ring = FEED == FEED_UNITS ? unit_slots * unit_slot_bytes : FEED == FEED_BULK ? 16 + (int)(bulk_slots(row_bytes) * rings * rows * row_bytes) : 0;
    return std::max({ring, fold_bytes, finish_bytes});
  }
};

template <typename RT, int FEED, int G, int CH, int R>
__global__ void __launch_bounds__(GradShape<RT, FEED, G, CH, R>::threads, GradShape<RT, FEED, G, CH, R>::per_sm)
gradient_rows_kernel(const __grid_constant__ GradParams p) {
  using Shape = GradShape<RT, FEED, G, CH, R>;
  constexpr int V = Shape::V, L = Shape::lanes, W = Shape::warps, E = CH * V, T = Shape::threads;
  constexpr bool SCALED = Shape::scaled, VEC = FEED != FEED_ELEMENTS, BULK = FEED == FEED_BULK;
  extern __shared__ __align__(16) unsigned char grad_smem[];
  __shared__ float2 cross[2][T / 32][R];  // a warp's sums of w x and x x of each row
  __shared__ double cross64[T / 32];
  __shared__ double sums[2][T / 32];
  __shared__ unsigned long long bars[BULK ? Shape::rings * 8 : 1];
  __shared__ bool gave_up[2][BULK && W > 1 ? Shape::groups : 1];  // in an even or odd round, by a warp of the group
  kernel_started();
  if constexpr (BULK) {
    if (threadIdx.x == 0) {
      for (int i = 0; i < Shape::rings * 8; ++i) mbar_init(&bars[i], 1);
      mbar_fence_init();
    }
    if (threadIdx.x < 4) ((uint32_t*)grad_smem)[threadIdx.x] = 0u;
    if (W > 1 && threadIdx.x < 2 * Shape::groups) (&gave_up[0][0])[threadIdx.x] = false;
    __syncthreads();
  }
  kernel_inputs_ready();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int group = threadIdx.x / G, gl = threadIdx.x % G, l = lane % L;
  const int units = (int)(VEC ? (p.d + V - 1) / V : p.d);
  auto group_barrier = [&]() {
    if constexpr (W > 1) asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(G) : "memory");
  };
  // column of element i: VEC (unit gl + j G) V + e, else gl + i G
  auto column = [&](int i) { return VEC ? (gl + i / V * G) * V + i % V : gl + i * G; };
  auto has = [&](int i) { return column(i) < p.d; };

  const long long stride = (long long)gridDim.x * Shape::groups * R;  // rows that all groups take at a time
  const long long first = ((long long)blockIdx.x * Shape::groups + group) * R;
  // ---- FEED_UNITS: rows through this thread's slots. What lies behind a row's end arrives as zeros.
  constexpr int S = FEED == FEED_UNITS ? Shape::unit_slots : 2;
  const uint32_t slots = (uint32_t)__cvta_generic_to_shared(grad_smem) + threadIdx.x * 16;
  const uint32_t slot_scales = (uint32_t)__cvta_generic_to_shared(grad_smem) + S * T * R * CH * 16 + threadIdx.x * 4;
  const long long row_bytes = VEC ? p.ld * (16 / V) : 0;
  const char* from = VEC ? (const char*)p.X + (first < p.n_rows ? first : 0) * row_bytes : nullptr;  // the next rows to request
  const float* from_scale = SCALED ? p.scales + (first < p.n_rows ? first : 0) * p.ld_s : nullptr;
  long long left = p.n_rows - first;  // rows from there on
  int bytes[CH], offset[CH];  // of unit j: bytes of the row, place in it (the row's start for units behind its end: nothing is read there)
#pragma unroll
  for (int j = 0; j < CH; ++j) {
    const long long b = (p.d - (long long)(gl + j * G) * V) * (16 / V);
    bytes[j] = b < 0 ? 0 : b > 16 ? 16 : (int)b;
    offset[j] = b > 0 ? (gl + j * G) * 16 : 0;
  }
  auto request_units = [&](int slot) {
    const char* row = from;
    const float* row_scale = from_scale;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const bool yes = r < left;
#pragma unroll
      for (int j = 0; j < CH; ++j) {
        const int at = (slot * R + r) * CH + j;
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(slots + at * (T * 16)), "l"(row + offset[j]), "r"(yes ? bytes[j] : 0) : "memory");
        if constexpr (SCALED)
          asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(slot_scales + at * (T * 4)), "l"(row_scale + offset[j] / Q_BLOCK), "r"(yes && bytes[j] ? 4 : 0) : "memory");
      }
      if (r + 1 < left) {  // never beyond the last row
        row += row_bytes;
        if constexpr (SCALED) row_scale += p.ld_s;
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    if (left > stride) {
      from += stride * row_bytes;
      if constexpr (SCALED) from_scale += stride * p.ld_s;
    }
    left -= stride;
  };
  // ---- FEED_BULK: the ring of this group or warp. Rows behind the last are zeros.
  int dead = -1;  // round in which a wait ran out: go on without waiting and without new requests. The same in a warp, and in a group after a round's barrier
  const int ring_slots = p.slots, ring = warp / W, bulk_row = (int)(p.d * (16 / V)), bulk_slot = Shape::rows * bulk_row;
  unsigned char* ring_base = grad_smem + 16 + (size_t)ring * ring_slots * bulk_slot;
  const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring_base) + (L < 32 ? lane / L * (R * bulk_row) : 0) + gl * 16;  // this thread's first unit
  const uint32_t zeros_at = (uint32_t)__cvta_generic_to_shared(grad_smem);
  const long long ring_first = ((long long)blockIdx.x * Shape::rings + ring) * Shape::rows;  // the warp's first row
  unsigned long long* full = bars + ring * 8;
  auto request_rows = [&](int slot, long long row0, long long round) {  // by one warp
    if (row0 >= p.n_rows || round == p.drop_block || dead >= 0) return;
    const int rows = p.n_rows - row0 < Shape::rows ? (int)(p.n_rows - row0) : Shape::rows;
    unsigned char* to = ring_base + (size_t)slot * bulk_slot;
    const char* src = (const char*)p.X + row0 * row_bytes;
    for (int i = rows * bulk_row + lane * 16; i < bulk_slot; i += 512) *(uint4*)(to + i) = make_uint4(0u, 0u, 0u, 0u);
    __syncwarp();
    if (lane == 0) mbar_arrive_expect_tx(&full[slot], rows * bulk_row);
    if (row_bytes == bulk_row) {
      if (lane == 0) bulk_copy_g2s(to, src, rows * bulk_row, &full[slot]);
    } else {
      __syncwarp();
      for (int r = lane; r < rows; r += 32) bulk_copy_g2s(to + r * bulk_row, src + r * row_bytes, bulk_row, &full[slot]);
    }
  };
  // ---- else: rows through registers, the next R on their way
  using Scalar = typename RowUnit<RT>::Scalar;  // kept as loaded: a conversion would wait for the load
  Scalar next[VEC ? 1 : R][VEC ? 1 : E];
  auto load = [&](long long row0) {
    if constexpr (!VEC) {
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < E; ++i) next[r][i] = row0 + r < p.n_rows && has(i) ? ((const Scalar*)p.X)[(row0 + r) * p.ld + column(i)] : Scalar(0.0f);
    }
  };
  if constexpr (BULK) {
    if (W == 1 || warp % W == 0)
      for (int i = 0; i < ring_slots; ++i) request_rows(i, ring_first + i * stride, i);
  } else if constexpr (VEC) {
#pragma unroll 1
    for (int i = 0; i < S - 1; ++i) request_units(i);
  } else {
    load(first);
  }

  uint64_t w[E / 2], acc[E / 2];
#pragma unroll
  for (int i = 0; i < E; i += 2) {
    w[i / 2] = pair_of(__float_as_uint(has(i) ? p.w[column(i)] : 0.0f), __float_as_uint(has(i + 1) ? p.w[column(i + 1)] : 0.0f));
    acc[i / 2] = 0;
  }
  float w_norm;  // |w|
  if constexpr (W > 1) {
    w_norm = block_w_norm(p.w, p.d, cross64);
  } else {  // narrow rows: from the group's registers
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < E / 2; ++i) {
      const float2 h = halves(w[i]);
      s = fma((double)h.x, (double)h.x, fma((double)h.y, (double)h.y, s));
    }
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    w_norm = (float)sqrt(s) * 1.0001f;
  }
  constexpr float terms = E + W + 8;  // additions a product takes part in: the thread's, 5 in the warp, W over the warps; 3 roundings for scales

  // losses: their margins wait, a lane each, until the warp has a full set to evaluate side by side
  double loss = 0.0;
  float z_held = 0.0f, y_held = 0.0f;
  int held = 0, wrong = 0;
  bool in_held = false;
  auto evaluate = [&]() {
    if (lane < held && in_held) loss += loss_of(p.loss, y_held, z_held);
    held = 0;
  };

  int round = 0, slot = 0;
  uint32_t parity = 0;
  const int own = l / (L / R);  // of the R rows, the one whose sums this lane ends with
  float y_next = first + own < p.n_rows ? p.y[first + own] : 0.0f;
  // groups within a warp go round together (shuffles over the warp)
  for (long long row0 = first; L < 32 ? __any_sync(0xffffffffu, row0 < p.n_rows) : row0 < p.n_rows; row0 += stride, ++round) {
    const bool in = row0 + own < p.n_rows;
    const float y = y_next;
    y_next = row0 + stride + own < p.n_rows ? p.y[row0 + stride + own] : 0.0f;
    Scalar plain[VEC ? 1 : R][VEC ? 1 : E];
    const int cur = slot;
    if constexpr (BULK) {
      if (dead < 0 && !__all_sync(0xffffffffu, mbar_wait_bounded(&full[cur], parity, p.spin_limit))) {  // (the lanes' waits may end differently)
        dead = round;
        if (W > 1) gave_up[round & 1][group] = true;
        if (lane == 0) set_status(p.status, DEV_TIMEOUT, 51, blockIdx.x);
      }
      if (++slot == ring_slots) { slot = 0; parity ^= 1; }
    } else if constexpr (VEC) {
      asm volatile("cp.async.wait_group %0;" ::"n"(S - 2) : "memory");
      request_units(slot == 0 ? S - 1 : slot - 1);  // into the slot of one round ago
      slot = slot == S - 1 ? 0 : slot + 1;
    } else {
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < E; ++i) plain[r][i] = next[r][i];
      load(row0 + stride);
    }
    // read from the slot both for the margin and for the gradient; widened values of all R rows would not fit the registers
    auto values = [&](int r, int j, uint64_t (&x)[V / 2]) {
      if constexpr (VEC) {
        uint32_t at = slots + ((cur * R + r) * CH + j) * (T * 16);
        if constexpr (BULK) at = gl + j * G < units ? ring_at + cur * bulk_slot + r * bulk_row + j * (G * 16) : zeros_at;
        uint4 raw;
        asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(raw.x), "=r"(raw.y), "=r"(raw.z), "=r"(raw.w) : "r"(at));
        RowUnit<RT>::widen(raw, x);
      } else {
#pragma unroll
        for (int e = 0; e < V / 2; ++e) x[e] = pair_of(__float_as_uint(widen_scalar<Scalar>(plain[r][j * V + 2 * e])), __float_as_uint(widen_scalar<Scalar>(plain[r][j * V + 2 * e + 1])));
      }
    };
    auto scale_of = [&](int r, int j) {
      float v;
      asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(slot_scales + ((cur * R + r) * CH + j) * (T * 4)));
      return v;
    };

    float z[R], xx[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      uint64_t z2 = 0, x2 = 0;
      z[r] = xx[r] = 0.0f;
#pragma unroll
      for (int j = 0; j < CH; ++j) {
        uint64_t x[V / 2];
        values(r, j, x);
#pragma unroll
        for (int e = 0; e < V / 2; ++e) {
          z2 = fma2(w[j * (V / 2) + e], x[e], z2);
          if constexpr (!SCALED) x2 = fma2(x[e], x[e], x2);
        }
        if constexpr (SCALED) {
          const float2 h = halves(z2);
          const float scale = scale_of(r, j);
          z[r] = fmaf(scale, h.x + h.y, z[r]);
          xx[r] = fmaf(scale * (V * Q_MAX * Q_MAX), scale, xx[r]);  // a bound: no |q| is above 448
          z2 = 0;
        }
      }
      if constexpr (!SCALED) {
        const float2 h = halves(z2), q = halves(x2);
        z[r] = h.x + h.y;
        xx[r] = q.x + q.y;
      }
    }
    float zs = transpose_sum<R, L>(z, l), xs = transpose_sum<R, L>(xx, l);
    if constexpr (W > 1) {  // every warp of the group adds up and goes on alike: one barrier a round
      if (l % (L / R) == 0) cross[round & 1][warp][own] = make_float2(zs, xs);
      group_barrier();
      if constexpr (BULK) {  // the rows of one round ago are done with
        if (dead < 0 && gave_up[round & 1][group]) dead = round;  // (a warp that is ahead by a round writes the other flag)
        if (round > 0 && round % W == warp - group * W) request_rows(cur == 0 ? ring_slots - 1 : cur - 1, row0 + (ring_slots - 1) * stride, round + ring_slots - 1ll);
      }
      zs = xs = 0.0f;
#pragma unroll
      for (int i = 0; i < W; ++i) {
        const float2 c = cross[round & 1][group * W + i][own];
        zs += c.x;
        xs += c.y;
      }
    }
    float g = in ? row_derivative(p.loss, y, zs) : 0.0f;
    bool positive = zs >= 0.0f;
    // the same in all lanes that hold the row, and in all warps of the group
    const unsigned redo = __ballot_sync(0xffffffffu, in && near_jump(p.loss, y, zs, margin_error(terms, w_norm, xs)));
    if (redo) {
#pragma unroll 1
      for (int r = 0; r < R; ++r) {
        if (!__any_sync(0xffffffffu, own == r && (redo >> lane & 1))) continue;
        double s = 0.0;  // this thread's columns once more, with exact products
        if constexpr (VEC) {
#pragma unroll
          for (int j = 0; j < CH; ++j) {
            uint64_t x[V / 2];
            values(r, j, x);
            const double scale = SCALED ? (double)scale_of(r, j) : 1.0;
#pragma unroll
            for (int e = 0; e < V / 2; ++e) {
              const float2 xe = halves(x[e]), we = halves(w[j * (V / 2) + e]);
              s += (double)we.x * (scale * (double)xe.x) + (double)we.y * (scale * (double)xe.y);
            }
          }
        } else if (row0 + r < p.n_rows) {
#pragma unroll
          for (int i = 0; i < E; ++i)
            if (has(i)) s += exact_product<RT>(p, row0 + r, column(i));
        }
#pragma unroll
        for (int o = L / 2; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        if constexpr (W > 1) {
          group_barrier();
          if (lane == 0) cross64[warp] = s;
          group_barrier();
          s = 0.0;
#pragma unroll 1
          for (int i = 0; i < W; ++i) s += cross64[group * W + i];
        }
        if (own == r && in) {
          g = row_derivative(p.loss, y, s);
          positive = s >= 0.0;
          zs = (float)s;
        }
      }
    }
    if (W == 1 || round % W == warp - group * W) {  // the warps of a group take turns with the losses
      constexpr int N = R * (32 / L);               // rows of the warp; row i's margin is in lane i L / R
      wrong += __popc(__ballot_sync(0xffffffffu, in && l % (L / R) == 0 && positive != (y >= 0.0f)));
      if (held + N > 32) evaluate();
      const int from_lane = (lane - held) * (L / R) & 31;
      const float zv = __shfl_sync(0xffffffffu, zs, from_lane), yv = __shfl_sync(0xffffffffu, y, from_lane);
      const unsigned inside = __ballot_sync(0xffffffffu, in);
      if (lane >= held && lane < held + N) { z_held = zv; y_held = yv; in_held = inside >> from_lane & 1; }
      held += N;
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const float gr = __shfl_sync(0xffffffffu, g, r * (L / R), L);
#pragma unroll
      for (int j = 0; j < CH; ++j) {
        uint64_t x[V / 2];
        values(r, j, x);
        float gs = gr;
        if constexpr (SCALED) gs *= scale_of(r, j);
        const uint64_t g2 = pair_of(__float_as_uint(gs), __float_as_uint(gs));
#pragma unroll
        for (int e = 0; e < V / 2; ++e) acc[j * (V / 2) + e] = fma2(g2, x[e], acc[j * (V / 2) + e]);
      }
    }
    if constexpr (BULK && W == 1) {
      __syncwarp();
      request_rows(cur, row0 - first + ring_first + ring_slots * stride, round + (long long)ring_slots);
    }
  }
  if constexpr (BULK) {
    if (dead >= 0 && lane == 0 && (W == 1 || warp % W == 0)) {  // copies in flight land before the block ends
      const int requested = dead + ring_slots - (W > 1 && dead > 0 ? 1 : 0);  // rounds; larger groups request in the round after
      for (int i = dead; i < requested; ++i)
        if (ring_first + i * stride < p.n_rows && i != p.drop_block) mbar_wait_bounded(&full[i % ring_slots], i / ring_slots & 1, DRAIN_LIMIT);
    }
  }
  evaluate();

  loss = warp_sum_f64(loss);
  if (lane == 0) { sums[0][warp] = loss; sums[1][warp] = wrong; }
  auto own_sum = [&](int i) { return i % 2 ? halves(acc[i / 2]).y : halves(acc[i / 2]).x; };
  float* fold = (float*)grad_smem;
  if constexpr (FEED == FEED_UNITS) asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();  // the slots are done with
  if constexpr (Shape::groups > 1) {
#pragma unroll
    for (int i = 0; i < E; ++i) fold[(i * Shape::groups + group) * G + gl] = own_sum(i);
  }
  __syncthreads();
  if (threadIdx.x < 2) {
    double t = 0.0;
    for (int i = 0; i < T / 32; ++i) t += sums[threadIdx.x][i];
    p.sums[2 * blockIdx.x + threadIdx.x] = t;
  }
  float* to = p.part + (long long)blockIdx.x * p.d;
  if constexpr (Shape::groups > 1) {
    for (int c = threadIdx.x; c < E * G; c += T) {  // element c / G of thread c % G of every group
      const int i = c / G, t = c % G;
      const int col = VEC ? (t + i / V * G) * V + i % V : t + i * G;
      if (col < p.d) {
        float s = 0.0f;
#pragma unroll
        for (int g = 0; g < Shape::groups; ++g) s += fold[(i * Shape::groups + g) * G + t];
        to[col] = s;
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (has(i)) to[column(i)] = own_sum(i);
  }
  if (!p.ticket) return;
  __shared__ bool last;
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) {
    last = atomicAdd(p.ticket, 1u) == gridDim.x - 1;
    if (last) *p.ticket = 0u;
  }
  __syncthreads();
  if (!last) return;
  __threadfence();
  gradient_finish_small<T / 32>(p, gridDim.x, gridDim.x, (double (*)[36])grad_smem);
}

}  // namespace wpsgd
