// Global norm of a list of gradients and clipping:  N = sqrt(sum over all tensors and elements of g^2),
// out = g * f with f = max_norm / N where N > max_norm, else 1.
//
// Two launches (short lists: one, clip_small_kernel): block sums of g^2, then the scaled copies, each block of which adds the block sums up again in the same order (so
// no result depends on timing, and no block waits for another). The list travels as a kernel argument: nothing is copied before
// the launch and nothing is kept after it.
// Sums: the squares of a batch of 16-byte units in fp32, the batches in fp64. Where a batch's sum leaves the range in which fp32
// squares are exact to rounding (elements below 2^-40 alone, above 2^60, not finite) it is formed again in fp64, so that norms of
// very small and very large gradients come out right.
// Bound by memory: reads the gradients once for the norm and once more, from L2 as far as they fit, for the copies. The second
// pass therefore goes through each block's part backwards, latest read first, and all but the last 72 MB of the first pass, and
// all of the second, is marked to leave L2 first (64 tensors of 2^20 fp32 elements: 140.8 us without the marks, 138.5 with them). The
// norm alone takes 45.7 us there, 5.9 TB/s, the second pass 92, 5.8 TB/s of reads and writes.
#pragma once

#include "common.cuh"

namespace wpsgd {

constexpr int CLIP_CHUNK = 8192;   // elements per unit of work
constexpr int CLIP_BLOCKS = 148 * 8;
constexpr int CLIP_THREADS = 128;
constexpr long long CLIP_KEEP = 72ll << 20;  // bytes that the first pass leaves in L2 for the second

// N tensors at most. elems_type = elements * 2 + (1: bf16, 0: fp32); first_chunk[i]: chunks of the tensors before i.
template <int N>
struct TensorList {
  const void* src[N];
  void* dst[N];
  long long elems_type[N];
  int first_chunk[N + 1];
  int n;
  uint16_t start[CLIP_BLOCKS];  // tensor that holds the first chunk of each block's share
};

// Elements of a tensor as 16-byte units of the source: `head` elements before the first aligned address, whole units, the rest.
struct TensorParts {
  long long head, units, n;
  __device__ __forceinline__ TensorParts(const void* src, long long n_, int es) : n(n_) {
    const long long h = (16 - ((uintptr_t)src & 15)) % 16 / es;
    head = h < n ? h : n;
    units = (n - head) / (16 / es);
  }
};

template <typename T>
__device__ __forceinline__ float batch_squares(const uint4* raw, int count) {
  constexpr int V = XVec<T>::V;
  float s = 0.0f;
#pragma unroll
  for (int u = 0; u < count; ++u) {
    float x[V];
    XVec<T>::widen(raw[u], x);
#pragma unroll
    for (int e = 0; e < V; ++e) s = fmaf(x[e], x[e], s);
  }
  return s;
}
template <typename T, int U>
__device__ __forceinline__ double batch_squares_f64(const uint4 (&raw)[U]) {
  constexpr int V = XVec<T>::V;
  double s = 0.0;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float x[V];
    XVec<T>::widen(raw[u], x);
#pragma unroll
    for (int e = 0; e < V; ++e) s = fma((double)x[e], (double)x[e], s);
  }
  return s;
}

// this thread's share of the squares of chunk `chunk` (of its tensor)
template <typename T>
__device__ __forceinline__ double chunk_squares(const T* src, long long n, int chunk, bool keep) {
  constexpr int V = XVec<T>::V, UNITS = CLIP_CHUNK / V, U = 4;
  const TensorParts tp(src, n, sizeof(T));
  const uint4* body = (const uint4*)(src + tp.head);
  double sum = 0.0;
  const long long u0 = (long long)chunk * UNITS, u1 = u0 + UNITS < tp.units ? u0 + UNITS : tp.units;
  for (long long u = u0 + threadIdx.x; u < u1; u += U * CLIP_THREADS) {
    uint4 raw[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      raw[i] = make_uint4(0u, 0u, 0u, 0u);
      if (u + i * CLIP_THREADS < u1) raw[i] = keep ? body[u + i * CLIP_THREADS] : __ldcs(body + u + i * CLIP_THREADS);  // (ordinary loads: clip_small_kernel writes in place)
    }
    const float s = batch_squares<T>(raw, U);
    if (s > 0x1p-80f && s < 0x1p120f) sum += (double)s;
    else {
      uint32_t any = 0;
#pragma unroll
      for (int i = 0; i < U; ++i) any |= raw[i].x | raw[i].y | raw[i].z | raw[i].w;
      if (any) sum += batch_squares_f64<T, U>(raw);
    }
  }
  if (chunk == 0) {  // the elements before and behind the whole units: fewer than 2 V
    const long long ends = n - tp.units * V;
    if (threadIdx.x < ends) {
      const double x = widen_scalar<T>(src[threadIdx.x < tp.head ? threadIdx.x : threadIdx.x + tp.units * V]);
      sum = fma(x, x, sum);
    }
  }
  return sum;
}

// scaled copy of chunk `chunk`
template <typename T>
__device__ __forceinline__ T scaled(float x, float f);
template <>
__device__ __forceinline__ float scaled<float>(float x, float f) { return x * f; }
template <>
__device__ __forceinline__ __nv_bfloat16 scaled<__nv_bfloat16>(float x, float f) { return __float2bfloat16_rn(x * f); }
__device__ __forceinline__ uint4 scaled_unit(const uint4& raw, float f, float) {
  return make_uint4(__float_as_uint(__uint_as_float(raw.x) * f), __float_as_uint(__uint_as_float(raw.y) * f),
                    __float_as_uint(__uint_as_float(raw.z) * f), __float_as_uint(__uint_as_float(raw.w) * f));
}
__device__ __forceinline__ uint4 scaled_unit(const uint4& raw, float f, __nv_bfloat16) {
  float x[8];
  XVec<__nv_bfloat16>::widen(raw, x);
  uint32_t w[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(x[2 * e] * f, x[2 * e + 1] * f);
    w[e] = *(const uint32_t*)&p;
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
template <typename T>
__device__ __forceinline__ void chunk_scale(const T* src, T* dst, long long n, int chunk, float f) {
  constexpr int V = XVec<T>::V, UNITS = CLIP_CHUNK / V, U = 4;
  const TensorParts tp(src, n, sizeof(T));
  const uint4* body = (const uint4*)(src + tp.head);
  T* to = dst + tp.head;
  const bool whole = ((uintptr_t)to & 15) == 0;
  const long long u0 = (long long)chunk * UNITS, u1 = u0 + UNITS < tp.units ? u0 + UNITS : tp.units;
  for (long long u = u0 + threadIdx.x; u < u1; u += U * CLIP_THREADS) {
    uint4 raw[U];
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (u + i * CLIP_THREADS < u1) raw[i] = __ldcs(body + u + i * CLIP_THREADS);
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (u + i * CLIP_THREADS >= u1) continue;
      if (whole) {
        __stcs((uint4*)to + u + i * CLIP_THREADS, scaled_unit(raw[i], f, T()));
      } else {
        float x[V];
        XVec<T>::widen(raw[i], x);
#pragma unroll
        for (int e = 0; e < V; ++e) to[(u + i * CLIP_THREADS) * V + e] = scaled<T>(x[e], f);
      }
    }
  }
  if (chunk == 0) {
    const long long ends = n - tp.units * V;
    if (threadIdx.x < ends) {
      const long long i = threadIdx.x < tp.head ? threadIdx.x : threadIdx.x + tp.units * V;
      dst[i] = scaled<T>(widen_scalar<T>(src[i]), f);
    }
  }
}

// The same by a factor that has no normal fp32 (gradients of 1e38 brought down to a norm of 1 and less): products in fp64.
template <typename T>
__device__ __forceinline__ void chunk_scale_f64(const T* src, T* dst, long long n, int chunk, double q) {
  const long long i0 = (long long)chunk * CLIP_CHUNK, i1 = i0 + CLIP_CHUNK < n ? i0 + CLIP_CHUNK : n;
  for (long long i = i0 + threadIdx.x; i < i1; i += CLIP_THREADS) dst[i] = scaled<T>((float)((double)widen_scalar<T>(src[i]) * q), 1.0f);
}
// out = g q, q = max_norm / N or 1
template <int N>
__device__ __forceinline__ void scale_chunk_of(const TensorList<N>& list, int i, int chunk, double q) {
  const long long n = list.elems_type[i] >> 1;
  const bool bf16 = list.elems_type[i] & 1;
  if (q < 0x1p-126 && q > 0.0) {
    if (bf16) chunk_scale_f64((const __nv_bfloat16*)list.src[i], (__nv_bfloat16*)list.dst[i], n, chunk, q);
    else chunk_scale_f64((const float*)list.src[i], (float*)list.dst[i], n, chunk, q);
  } else {
    if (bf16) chunk_scale((const __nv_bfloat16*)list.src[i], (__nv_bfloat16*)list.dst[i], n, chunk, (float)q);
    else chunk_scale((const float*)list.src[i], (float*)list.dst[i], n, chunk, (float)q);
  }
}

// The chunks of a block's even share of all, first to last or last to first: f(tensor, chunk of it, chunks to go)
template <int N, typename F>
__device__ __forceinline__ void for_own_chunks(const TensorList<N>& list, bool backwards, F f) {
  const int total = list.first_chunk[list.n];
  const int c0 = (int)((long long)total * blockIdx.x / gridDim.x), c1 = (int)((long long)total * (blockIdx.x + 1) / gridDim.x);
  if (c0 >= c1) return;
  const int start = backwards ? c1 - 1 : c0;
  int i = list.start[blockIdx.x];
  for (int k = 0; k < c1 - c0; ++k) {
    const int c = backwards ? start - k : start + k;
    while (c >= list.first_chunk[i + 1]) ++i;
    while (c < list.first_chunk[i]) --i;
    f(i, c - list.first_chunk[i], c1 - c0 - k);
  }
}

__device__ __forceinline__ double block_sum_f64(double v, double* sh) {  // of all CLIP_THREADS threads, to every thread
  v = warp_sum_f64(v);
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
  __syncthreads();
  double t = 0.0;
#pragma unroll
  for (int i = 0; i < CLIP_THREADS / 32; ++i) t += sh[i];
  return t;
}

// part[block] = squares of the block's share (added to what the launches before it found, where the list takes several)
template <int N>
__global__ void __launch_bounds__(CLIP_THREADS, 8) squares_kernel(const __grid_constant__ TensorList<N> list, bool first, double* __restrict__ part) {
  __shared__ double sh[CLIP_THREADS / 32];
  kernel_started();
  kernel_inputs_ready();
  double sum = 0.0;
  const int kept = (int)(CLIP_KEEP / (CLIP_CHUNK * 4) / gridDim.x);  // of a block's chunks, the last: the second pass starts with them
  for_own_chunks(list, false, [&](int i, int chunk, int to_go) {
    const long long n = list.elems_type[i] >> 1;
    sum += list.elems_type[i] & 1 ? chunk_squares((const __nv_bfloat16*)list.src[i], n, chunk, to_go <= kept) : chunk_squares((const float*)list.src[i], n, chunk, to_go <= kept);
  });
  sum = block_sum_f64(sum, sh);
  if (threadIdx.x == 0) part[blockIdx.x] = first ? sum : part[blockIdx.x] + sum;
}

// N from the block sums, the same in every block
__device__ __forceinline__ double norm_of_parts(const double* part, int parts, double* sh) {
  double v = 0.0;
  for (int i = threadIdx.x; i < parts; i += CLIP_THREADS) v += __ldcg(part + i);
  return sqrt(block_sum_f64(v, sh));
}

__global__ void __launch_bounds__(CLIP_THREADS) norm_kernel(const double* __restrict__ part, int parts, float* __restrict__ norm_out) {
  __shared__ double sh[CLIP_THREADS / 32];
  kernel_started();
  kernel_inputs_ready();
  const double norm = norm_of_parts(part, parts, sh);
  if (threadIdx.x == 0) *norm_out = (float)norm;
}

template <int N>
__global__ void __launch_bounds__(CLIP_THREADS, 8) scale_kernel(const __grid_constant__ TensorList<N> list, const double* __restrict__ part, int parts,
                                                             double max_norm, bool in_place, float* __restrict__ norm_out) {
  __shared__ double sh[CLIP_THREADS / 32];
  kernel_started();
  kernel_inputs_ready();
  const double norm = norm_of_parts(part, parts, sh);
  if (blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)norm;
  const bool clips = norm > max_norm;
  if (!clips && in_place) return;  // times 1
  const double q = clips ? max_norm / norm : 1.0;
  for_own_chunks(list, true, [&](int i, int chunk, int) { scale_chunk_of(list, i, chunk, q); });
}

// Both steps of a short list in one launch: a cluster of blocks that give each other their sums through distributed shared memory.
// Times of one launch and of two, fp32, apart (in a graph): 8 tensors of 1024 elements 4.1 and 4.6 us (3.3 and 4.9), 16 of 1024 5.4 and 5.5 (4.3 and 5.0), 17 of 1024
// 6.5 and 5.5, 8 of 8192 6.6 and 8.0, 16 of 8192 9.8 and 8.2. The limit of 16 chunks suits lists of short tensors; whole chunks pay up to 8.
constexpr int CLIP_CLUSTER = 8;
constexpr int CLIP_SMALL_CHUNKS = 2 * CLIP_CLUSTER;
template <int N>
__global__ void __cluster_dims__(CLIP_CLUSTER, 1, 1) __launch_bounds__(CLIP_THREADS)
clip_small_kernel(const __grid_constant__ TensorList<N> list, bool scale, double max_norm, bool in_place, float* __restrict__ norm_out) {
  __shared__ double sh[CLIP_THREADS / 32];
  __shared__ double sums[CLIP_CLUSTER];
  asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");  // start-up, waited for below
  kernel_started();
  kernel_inputs_ready();
  double sum = 0.0;
  const int kept = (int)(CLIP_KEEP / (CLIP_CHUNK * 4) / gridDim.x);  // of a block's chunks, the last: the second pass starts with them
  for_own_chunks(list, false, [&](int i, int chunk, int to_go) {
    const long long n = list.elems_type[i] >> 1;
    sum += list.elems_type[i] & 1 ? chunk_squares((const __nv_bfloat16*)list.src[i], n, chunk, to_go <= kept) : chunk_squares((const float*)list.src[i], n, chunk, to_go <= kept);
  });
  sum = block_sum_f64(sum, sh);
  asm volatile("barrier.cluster.wait;" ::: "memory");  // every block of the cluster runs, so its shared memory is there
  if (threadIdx.x < CLIP_CLUSTER) {
    uint32_t to;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"((uint32_t)__cvta_generic_to_shared(sums + blockIdx.x)), "r"(threadIdx.x));
    asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(to), "d"(sum) : "memory");
  }
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  double all = 0.0;
#pragma unroll
  for (int i = 0; i < CLIP_CLUSTER; ++i) all += sums[i];
  const double norm = sqrt(all);
  if (blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)norm;
  const bool clips = norm > max_norm;
  if (!scale || (!clips && in_place)) return;
  const double q = clips ? max_norm / norm : 1.0;
  for_own_chunks(list, true, [&](int i, int chunk, int) { scale_chunk_of(list, i, chunk, q); });
}

}  // namespace wpsgd
