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
  int new_out;  // answers of rows outside the chains are set to zeros
  DevStatus* status;
};

// Four features from column c on, zeros behind dk, as loaded: what is converted on arrival is waited for on arrival
template <typename XT>
struct Features4;
template <>
struct Features4<float> {
  float4 r;
  __device__ __forceinline__ void load(const float* row, int c, int dk, int vec) {
    r = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (vec) {
      if (c < dk) r = __ldg((const float4*)(row + c));
    } else {
      if (c < dk) r.x = row[c];
      if (c + 1 < dk) r.y = row[c + 1];
      if (c + 2 < dk) r.z = row[c + 2];
      if (c + 3 < dk) r.w = row[c + 3];
    }
  }
  __device__ __forceinline__ void widen(float* f) const { f[0] = r.x, f[1] = r.y, f[2] = r.z, f[3] = r.w; }
};
template <>
struct Features4<__nv_bfloat16> {
  uint2 r;
  __device__ __forceinline__ void load(const __nv_bfloat16* row, int c, int dk, int vec) {
    r = make_uint2(0u, 0u);
    if (vec) {
      if (c < dk) r = __ldg((const uint2*)(row + c));
    } else {
      const unsigned short* at = (const unsigned short*)row;
      unsigned short e[4] = {0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (c + i < dk) e[i] = at[c + i];
      r = make_uint2(e[0] | (unsigned)e[1] << 16, e[2] | (unsigned)e[3] << 16);
    }
  }
  __device__ __forceinline__ void widen(float* f) const {
    f[0] = __uint_as_float(r.x << 16), f[1] = __uint_as_float(r.x & 0xffff0000u), f[2] = __uint_as_float(r.y << 16), f[3] = __uint_as_float(r.y & 0xffff0000u);
  }
};
// What a row brings for one model, as loaded
template <typename XT, int NJ>
struct DeltaRow {
  Features4<XT> k[NJ], q[NJ];
  XT v, g, beta;
  __device__ __forceinline__ void load(const XT* pk, const XT* pq, const XT* pv, const XT* pg, const XT* pb, int s, int dk, int vec) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      k[j].load(pk, 4 * (s + 8 * j), dk, vec);
      q[j].load(pq, 4 * (s + 8 * j), dk, vec);
    }
    v = *pv;
    g = *pg;
    beta = *pb;
  }
};
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

// One row of one model: updates w (4 NJ features of this lane) and returns the answer (in all eight lanes). Operations on pairs of fp32: half the instructions.
template <typename XT, int NJ>
__device__ __forceinline__ float delta_one_row(float (&w)[4 * NJ], const DeltaRow<XT, NJ>& row) {
  const float g = widen_scalar<XT>(row.g), a = expf(g < DELTA_MIN_G ? DELTA_MIN_G : g);
  uint64_t wk = 0, wq = 0, kq = 0, w2[2 * NJ], k2[2 * NJ];
  auto pair = [](float x, float y) { return pair_of(__float_as_uint(x), __float_as_uint(y)); };
  auto both = [](uint64_t v) {
    const float2 h = halves(v);
    return h.x + h.y;
  };
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    float k[4], q[4];
    row.k[j].widen(k);
    row.q[j].widen(q);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int i = 2 * j + e;
      const uint64_t q2 = pair(q[2 * e], q[2 * e + 1]);
      k2[i] = pair(k[2 * e], k[2 * e + 1]);
      w2[i] = pair(w[2 * i], w[2 * i + 1]);
      wk = fma2(w2[i], k2[i], wk);
      wq = fma2(w2[i], q2, wq);
      kq = fma2(k2[i], q2, kq);
    }
  }
  const float sk = sum8(both(wk)), sq = sum8(both(wq)), skq = sum8(both(kq));
  const float delta = widen_scalar<XT>(row.beta) * fmaf(-a, sk, widen_scalar<XT>(row.v));
  const uint64_t a2 = pair(a, a), d2 = pair(delta, delta);
#pragma unroll
  for (int i = 0; i < 2 * NJ; ++i) {
    const float2 h = halves(fma2(d2, k2[i], mul2(a2, w2[i])));
    w[2 * i] = h.x, w[2 * i + 1] = h.y;
  }
  return fmaf(a, sq, delta * skq);
}

// ---- chains, row by row ---------------------------------------------------------------------------------------------------------
// A block has 16 models of a chain, four to a warp, in registers and goes over the chain's rows, fp32. Features, queries, labels and gates of the next `batch` rows come to
// shared memory by asynchronous copies of all threads while it works on this batch; a row's are read a row ahead. Bounds: issue of one warp per scheduler and
// the latency of a row (sums over eight lanes and the step that depends on them). (Each lane bringing what it needs itself: 200 instructions a row and 820 cycles.)
constexpr int DELTA_WARPS = 4, ROWS_MODELS = 4 * DELTA_WARPS, ROWS_BATCH = 16;

// Heads of features that 16 neighbouring models can have, and floats of a row in shared memory: features and queries of those heads, a label, decay and step of each model
__host__ __device__ constexpr int rows_heads(int hk, int hv, int dv) {
  const int shared = hv / hk * dv, most = (ROWS_MODELS - 1 + shared - 1) / shared + 1;
  return most < hk ? most : hk;
}
template <int NJ>
__host__ __device__ constexpr int rows_floats(int heads) { return 2 * heads * 32 * NJ + 3 * ROWS_MODELS; }

__device__ __forceinline__ void copy4(const void* to, const void* from, bool yes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from), "r"(yes ? 4 : 0) : "memory");
}
__device__ __forceinline__ void copy_features(const float* to, const float* row, int c, int dk, int vec) {
  if (vec) {
    const bool yes = c < dk;
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(yes ? row + c : row), "r"(yes ? 16 : 0) : "memory");
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) copy4(to + e, c + e < dk ? row + c + e : row, c + e < dk);
  }
}

// A model whose chain is left out ends as it started; eight threads have it
__device__ __noinline__ void keep_model(const DeltaRowsParams& p, long long model, int s) {
  for (long long i = model * p.dk + s; i < (model + 1) * p.dk; i += 8) p.W[i] = p.W0 ? p.W0[i] : 0.0f;
}

// Answers of the rows before the first chain and behind the last set to zeros, a block's 16 columns of them. (Apart, as keep_model: written out in the kernel they cost
// 333 rows of 4 heads 0.5 of 17.7 us by other registers for the rows' loop.)
__device__ __noinline__ void clear_outside_columns(const DeltaRowsParams& p, long long chain, long long first, long long end, int R0, int models) {
  const int col = R0 + (threadIdx.x & 15);
  auto clear = [&](long long begin, long long stop) {
    for (long long r = begin + (threadIdx.x >> 4); r < stop; r += 2 * DELTA_WARPS)
      if (col < models) ((float*)p.out)[r * p.ld_out + col] = 0.0f;
  };
  if (chain == 0) clear(0, first);
  if (chain + 1 == p.n_chains) clear(end, p.n_rows);
}

template <int NJ>
__global__ void __launch_bounds__(32 * DELTA_WARPS) delta_rows_kernel(const __grid_constant__ DeltaRowsParams p, int batch) {
  constexpr int UNITS = 8 * NJ;  // of four features
  extern __shared__ __align__(16) float batch_smem[];
  kernel_inputs_ready();
  const int tid = threadIdx.x, lane = tid & 31, s = lane & 7, models = p.hv * p.dv, more = p.hv / p.hk;
  const int groups = (models + ROWS_MODELS - 1) / ROWS_MODELS;
  const long long chain = blockIdx.x / groups;
  const int R0 = (int)(blockIdx.x % groups) * ROWS_MODELS, mine = tid >> 3, R = R0 + mine;  // a model has eight threads
  const bool there = R < models;
  const int hk0 = R0 / p.dv / more, hk = there ? R / p.dv / more : hk0, heads = (min(R0 + ROWS_MODELS, models) - 1) / p.dv / more - hk0 + 1;
  const long long first = p.shard_off[chain], end = p.shard_off[chain + 1];
  if (first < 0 || end < first || end > p.n_rows) {  // the same for the whole block; other chains may be in order, and run
    if (tid == 0) set_status(p.status, DEV_BOUNDS, 22, chain);
    if (p.W && there) keep_model(p, chain * models + R, s);
    return;
  }
  const int floats = rows_floats<NJ>(rows_heads(p.hk, p.hv, p.dv)), labels_at = 2 * heads * 32 * NJ;
  auto bring = [&](long long t0, float* to) {  // rows t0 to t0 + batch - 1, as far as there are
    const int n = (int)min((long long)batch, end - t0);
    for (int u = tid; u < n * heads * 2 * UNITS; u += 32 * DELTA_WARPS) {
      const int c = u % UNITS * 4, which = u / UNITS % 2, rest = u / (2 * UNITS), row = rest / heads, head = rest - row * heads;
      const float* from = which ? (const float*)p.q + (t0 + row) * p.ld_q : (const float*)p.k + (t0 + row) * p.ld_k;
      copy_features(to + row * floats + (2 * head + which) * 32 * NJ + c, from + (hk0 + head) * p.dk, c, p.dk, p.vec);
    }
    for (int u = tid; u < n * ROWS_MODELS; u += 32 * DELTA_WARPS) {
      const int m = u % ROWS_MODELS, row = u / ROWS_MODELS, r = min(R0 + m, models - 1), h = r / p.dv;
      float* at = to + row * floats + labels_at + m;
      copy4(at, (const float*)p.v + (t0 + row) * p.ld_v + r, true);
      copy4(at + ROWS_MODELS, (const float*)p.g + (t0 + row) * p.ld_g + h, true);
      copy4(at + 2 * ROWS_MODELS, (const float*)p.beta + (t0 + row) * p.ld_beta + h, true);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  float* buffers[2] = {batch_smem, batch_smem + batch * floats};
  if (first < end) bring(first, buffers[0]);
  float w[4 * NJ];
  const long long at = (chain * models + (there ? R : 0)) * p.dk;
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    if (p.W0 && there) model4(p.W0 + at, 4 * (s + 8 * j), p.dk, p.vec, w + 4 * j);
    else w[4 * j] = w[4 * j + 1] = w[4 * j + 2] = w[4 * j + 3] = 0.0f;
  }
  float* out = (float*)p.out + first * p.ld_out + R;
  const int own = 2 * (hk - hk0) * 32 * NJ + 4 * s;
  int which = 0;
  for (long long t0 = first; t0 < end; t0 += batch, which ^= 1) {
    if (t0 + batch < end) {
      bring(t0 + batch, buffers[which ^ 1]);
      asm volatile("cp.async.wait_group 1;" ::: "memory");
    } else {
      asm volatile("cp.async.wait_group 0;" ::: "memory");
    }
    __syncthreads();
    const int n = (int)min((long long)batch, end - t0);
    const float* from = which ? buffers[1] : buffers[0];
    auto read = [&](DeltaRow<float, NJ>& row) {
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        row.k[j].r = *(const float4*)(from + own + 32 * j);
        row.q[j].r = *(const float4*)(from + own + 32 * NJ + 32 * j);
      }
      row.v = from[labels_at + mine], row.g = from[labels_at + ROWS_MODELS + mine], row.beta = from[labels_at + 2 * ROWS_MODELS + mine];
      from += floats;
    };
    DeltaRow<float, NJ> now, next;
    read(now);
#pragma unroll 2
    for (int i = 0; i < n; ++i) {
      if (i + 1 < n) read(next);
      const float o = delta_one_row<float, NJ>(w, now);
      if (s == 0 && there) *out = p.scale * o;
      out += p.ld_out;
      now = next;
    }
    __syncthreads();
  }
  kernel_started();  // not before: blocks of the next call that wait would share the schedulers of some (34 us a call instead of 17.6 for 333 rows of 4 heads)
  if (p.W && there)
#pragma unroll
    for (int j = 0; j < NJ; ++j) put_model4(p.W + at, 4 * (s + 8 * j), p.dk, p.vec, w + 4 * j);
  if (p.new_out) clear_outside_columns(p, chain, first, end, R0, models);
}

// ---- one row for each of many chains ------------------------------------------------------------------------------------------------
// A block has 32 models of a row at a time; they and what the row brings are on their way from memory together. Bounds: bytes, the models once in and once
// out (85 % of the copy rate for heads of 128 x 128; 131072 rows of one head of 16 x 16: 13 %, a block each of which half has no model). (Four models for each
// group of eight lanes, 128 a block: 266 us instead of 178 for 256 rows of 32 heads of 128 x 128; two: 191.)
// A slot that an earlier row has is left to that row. With few rows every block looks through the slots before its own, which come from L2 while its models come from memory; that is
// n^2 / 2 slots for each 32 models. With more, a block has a run of rows, and looks through the slots before them once for all: they are kept in a hash table in shared memory.
constexpr int STEP_THREADS = 256, STEP_RUN = 2048;  // rows of a run at most; the table has twice as many places and more

template <typename XT, int NJ>
__global__ void __launch_bounds__(STEP_THREADS) delta_step_kernel(const __grid_constant__ DeltaRowsParams p) {
  kernel_started();
  kernel_inputs_ready();
  const int lane = threadIdx.x & 31, s = lane & 7, models = p.hv * p.dv;
  const int groups = (models + 31) / 32;
  const long long row = blockIdx.x / groups;
  const int R = (int)(blockIdx.x % groups) * 32 + (threadIdx.x >> 5) * 4 + (lane >> 3);
  const bool there = R < models;
  const long long slot = p.slots ? p.slots[row] : row;
  const bool valid = slot >= 0 && slot < p.n_slots;
  float w[4 * NJ] = {};
  float* model = p.W + (valid && there ? (slot * models + R) * p.dk : 0);
  if (valid && there)
#pragma unroll
    for (int j = 0; j < NJ; ++j) model4(model, 4 * (s + 8 * j), p.dk, p.vec, w + 4 * j);
  const int h = there ? R / p.dv : 0, hk = h / (p.hv / p.hk);
  DeltaRow<XT, NJ> brought;
  brought.load((const XT*)p.k + row * p.ld_k + hk * p.dk, (const XT*)p.q + row * p.ld_q + hk * p.dk, (const XT*)p.v + row * p.ld_v + (there ? R : 0), (const XT*)p.g + row * p.ld_g + h,
               (const XT*)p.beta + row * p.ld_beta + h, s, p.dk, p.vec);
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
  const float o = delta_one_row<XT, NJ>(w, brought);
  if (there) {
    if (s == 0) ((XT*)p.out)[row * p.ld_out + R] = narrow_scalar<XT>(p.scale * o);
#pragma unroll
    for (int j = 0; j < NJ; ++j) put_model4(model, 4 * (s + 8 * j), p.dk, p.vec, w + 4 * j);
  }
}

// Many rows with slots: a block has `run` of them, one behind the other. table: 2^lg slots (twice `run` at least), -1 where there is none; first: the first row of
// the run that has the slot, -1 where an earlier run has it.
template <typename XT, int NJ>
__global__ void __launch_bounds__(STEP_THREADS) delta_step_runs_kernel(const __grid_constant__ DeltaRowsParams p, int run, int lg) {
  const int places = 1 << lg;
  extern __shared__ int step_smem[];
  int *table = step_smem, *first = table + places, *slots = first + places;  // slots: [run]
  const int tid = threadIdx.x, models = p.hv * p.dv, groups = (models + 31) / 32;
  const long long row0 = (long long)blockIdx.x * run;
  const int n = (int)min((long long)run, p.n_rows - row0);
  kernel_started();
  for (int i = tid; i < places; i += STEP_THREADS) table[i] = -1, first[i] = run;
  kernel_inputs_ready();
  __syncthreads();
  auto place = [&](int slot) { return (int)((unsigned)slot * 2654435769u >> (32 - lg)); };  // the high bits: slots that lie equally far apart spread too
  for (int i = tid; i < n; i += STEP_THREADS) {
    const int slot = p.slots[row0 + i];
    slots[i] = slot;
    if (slot < 0 || slot >= p.n_slots) continue;
    int at = place(slot);
    for (;; at = (at + 1) & (places - 1)) {  // ends: half of the places stay empty
      const int there = atomicCAS(table + at, -1, slot);
      if (there == -1 || there == slot) break;
    }
    atomicMin(first + at, i);
  }
  __syncthreads();
  auto look = [&](int slot) {  // of an earlier run
    for (int at = place(slot); table[at] != -1; at = (at + 1) & (places - 1))
      if (table[at] == slot) {
        first[at] = -1;
        break;
      }
  };
  constexpr int AHEAD = 8;
  for (long long r0 = tid; r0 < row0; r0 += STEP_THREADS * AHEAD) {
    int slot[AHEAD];
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) slot[a] = r0 + a * STEP_THREADS < row0 ? p.slots[r0 + a * STEP_THREADS] : -1;
#pragma unroll
    for (int a = 0; a < AHEAD; ++a)
      if (slot[a] >= 0) look(slot[a]);
  }
  __syncthreads();
  for (int i = tid; i < n; i += STEP_THREADS) {  // slots[i]: -1 from here on where the row has no models to step
    const int slot = slots[i];
    if (slot < 0) continue;
    bool mine = slot < p.n_slots;
    if (mine) {
      int at = place(slot);
      while (table[at] != slot) at = (at + 1) & (places - 1);
      mine = first[at] == i;
    }
    if (!mine) {
      set_status(p.status, DEV_BOUNDS, 23, row0 + i);
      slots[i] = -1;
    }
  }
  __syncthreads();
  const int s = tid & 7;
  for (int i = 0; i < n; ++i) {
    if (slots[i] < 0) continue;
    const long long row = row0 + i, model0 = (long long)slots[i] * models;
    for (int R = tid >> 3; R < groups * 32; R += 32) {  // all lanes go round: they add up together
      const bool there = R < models;
      float w[4 * NJ] = {};
      float* model = p.W + (model0 + (there ? R : 0)) * p.dk;
      if (there)
#pragma unroll
        for (int j = 0; j < NJ; ++j) model4(model, 4 * (s + 8 * j), p.dk, p.vec, w + 4 * j);
      const int h = there ? R / p.dv : 0, hk = h / (p.hv / p.hk);
      DeltaRow<XT, NJ> brought;
      brought.load((const XT*)p.k + row * p.ld_k + hk * p.dk, (const XT*)p.q + row * p.ld_q + hk * p.dk, (const XT*)p.v + row * p.ld_v + (there ? R : 0), (const XT*)p.g + row * p.ld_g + h,
                   (const XT*)p.beta + row * p.ld_beta + h, s, p.dk, p.vec);
      const float o = delta_one_row<XT, NJ>(w, brought);
      if (!there) continue;
      if (s == 0) ((XT*)p.out)[row * p.ld_out + R] = narrow_scalar<XT>(p.scale * o);
#pragma unroll
      for (int j = 0; j < NJ; ++j) put_model4(model, 4 * (s + 8 * j), p.dk, p.vec, w + 4 * j);
    }
  }
}

}  // namespace wpsgd
