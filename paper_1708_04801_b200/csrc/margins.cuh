// Margins of many models on many rows, both 8-bit with a scale for each block of 128 columns:
//
//   Z[i, m] = sum_b s_i,b t_m,b D_b[i, m],   D_b[i, m] = sum_{c in block b} q_i,c p_m,c
//
// D_b is a product of 8-bit matrices, formed by the tensor cores (tcgen05.mma kind::f8f6f4, fp32 sums in tensor memory) for a tile of 128
// rows and BN models, one block of 128 columns at a time; the scales differ from block to block on both sides, so each D_b is read
// back and added to fp32 registers with its scales while the tensor cores form the next ones in other buffers.
//
// One persistent CTA per SM, a role per warp: warp 0 brings the tiles of Q and M into a ring of stages (TMA, 128-byte swizzle; what lies outside
// the matrices arrives as zeros), warp 1 issues the products, warp 2 brings the scales of a block's 128 rows and BN models (cp.async) into a
// ring of its own, warp 3 owns the tensor memory, the warps from 4 on add up: thread = row, 128 rows per four warps. The margins
// leave through a staging buffer of each warp, so that stores cover 64 bytes of a row.
// Every wait is bounded. When one runs out it is recorded in the status word, all roles leave, the copies and products in flight are waited
// for (bounded again), and the tensor memory is given back.
#pragma once

#include <cuda.h>

#include "async.cuh"
#include "common.cuh"
#include "quantize.cuh"

namespace wpsgd {

constexpr int MG_ROWS = 128;       // of a tile: the lanes of tensor memory
constexpr int MG_SCALE_SLOTS = 8;  // blocks whose scales are in shared memory at a time

template <int BN>
struct MarginsShape {
  static constexpr int groups = BN >= 64 ? 2 : 1;     // of four adding warps: each takes BN / groups models
  static constexpr int cols = BN / groups;
  static constexpr int threads = 128 + 128 * groups;
  static constexpr int buffers = BN == 256 ? 2 : 4;   // of D_b in tensor memory
  static constexpr int tmem_cols = buffers * BN;      // a power of two, 64 .. 512
  static constexpr int stage_bytes = (MG_ROWS + BN) * Q_BLOCK;
  static constexpr int slot_bytes = (MG_ROWS + BN) * 4;
  static constexpr int staging_bytes = 4 * groups * 32 * 80;
  static constexpr int fixed_bytes = 1024 + MG_SCALE_SLOTS * slot_bytes + staging_bytes + 512;  // 1024: alignment of the ring
  static constexpr int stages = (227 * 1024 - fixed_bytes) / stage_bytes < 10 ? (227 * 1024 - fixed_bytes) / stage_bytes : 10;
  static constexpr int smem = fixed_bytes + stages * stage_bytes;
};

struct MarginsParams {
  const float* q_scales;
  long long ld_qs;
  const float* m_scales;
  long long ld_ms;
  void* Z;
  long long ld_z;
  int n_rows, n_models, blocks;   // blocks of 128 columns
  int tiles_m, tiles;             // tiles of models per tile of rows, tiles in all
  bool vector;                    // 16-byte stores reach every row's margins
  long long spin_limit;
  long long drop_block;           // test hook: this block of columns is never requested (-1: none)
  DevStatus* status;
};

// ---- tcgen05 ---------------------------------------------------------------------------------------------------------------
// Shared-memory operand, rows of 128 bytes with 128-byte swizzle, 8 rows (1024 bytes) to the next group of rows
__device__ __forceinline__ uint64_t mma_operand(uint32_t addr) {
  return (uint64_t)((addr & 0x3ffff) >> 4) | 1ull << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
// D fp32, A and B e4m3, both with contiguous k, M = 128
template <int BN>
__host__ __device__ constexpr uint32_t mma_shape() { return 1u << 4 | (uint32_t)(BN >> 3) << 17 | (uint32_t)(MG_ROWS >> 4) << 24; }
__device__ __forceinline__ void mma_e4m3(uint32_t d, uint64_t a, uint64_t b, uint32_t shape, bool add) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b),
               "r"(shape), "r"((uint32_t)add)
               : "memory");
}
__device__ __forceinline__ void mma_commit(unsigned long long* bar) {  // the barrier is arrived at when all products issued so far are done
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"((uint32_t)__cvta_generic_to_shared(bar)) : "memory");
}
__device__ __forceinline__ void tmem_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_alloc(uint32_t* to, uint32_t cols) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "r"(cols) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free(uint32_t addr, uint32_t cols) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols) : "memory");
}
// 16 columns of this warp's 32 lanes, a lane per thread
__device__ __forceinline__ void tmem_load16(uint32_t addr, uint32_t (&v)[16]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]),
                 "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
               : "r"(addr));
}
__device__ __forceinline__ void tmem_wait_load(uint32_t (&v)[16]) {  // names the registers, so that no use of them moves before the wait
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]), "+r"(v[9]), "+r"(v[10]),
                 "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15])::"memory");
}
__device__ __forceinline__ void tma_load_2d(void* dst, const CUtensorMap* map, int x, int y, unsigned long long* bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"((uint32_t)__cvta_generic_to_shared(dst)),
               "l"(map), "r"(x), "r"(y), "r"((uint32_t)__cvta_generic_to_shared(bar))
               : "memory");
}
__device__ __forceinline__ void cp_async4_or_zero(uint32_t dst, const float* src, bool yes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(yes ? 4 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_arrive(unsigned long long* bar) {  // one of the expected arrivals, when this thread's copies so far have landed
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"((uint32_t)__cvta_generic_to_shared(bar)) : "memory");
}
__device__ __forceinline__ void mbar_arrive_one(unsigned long long* bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"((uint32_t)__cvta_generic_to_shared(bar)) : "memory");
}
// pairs of fp32 in one instruction
__device__ __forceinline__ uint64_t pair_of(uint32_t lo, uint32_t hi) { return (uint64_t)hi << 32 | lo; }
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint4 lds16(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
  return v;
}
__device__ __forceinline__ void sts16(uint32_t a, uint4 v) {
  asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(a), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// A wait that gives up: after its own limit, or when another role has (dead). False: leave.
struct MarginsWait {
  long long limit;
  volatile int* dead;
  DevStatus* status;
  __device__ __forceinline__ bool operator()(unsigned long long* bar, uint32_t parity, int where) const {
    for (long long i = 0; i < limit; ++i) {
      if (mbar_try_wait(bar, parity)) return true;
      if (*dead) return false;
    }
    *dead = 1;
    set_status(status, DEV_TIMEOUT, where, blockIdx.x);
    return false;
  }
};

template <typename OT, int BN>
__global__ void __launch_bounds__(MarginsShape<BN>::threads, 1)
margins_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_m, const __grid_constant__ MarginsParams p) {
  using Shape = MarginsShape<BN>;
  constexpr int S = Shape::stages, NB = Shape::buffers, SS = MG_SCALE_SLOTS, COLS = Shape::cols;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* ring = (unsigned char*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  float* scales = (float*)(ring + S * Shape::stage_bytes);
  unsigned char* staging = (unsigned char*)(scales + SS * (MG_ROWS + BN));
  unsigned long long* bars = (unsigned long long*)(staging + Shape::staging_bytes);
  unsigned long long *full = bars, *empty = full + S, *acc_full = empty + S, *acc_empty = acc_full + NB, *sc_full = acc_empty + NB, *sc_empty = sc_full + SS,
                     *drained = sc_empty + SS;
  static_assert(8 * (2 * S + 2 * NB + 2 * SS + 1) + 8 <= 512, "barriers, tensor memory address and flag must fit");
  uint32_t& tmem_base = *(uint32_t*)(drained + 1);  // (no static shared memory: the dynamic part may be all of the SM's)
  volatile int* dead_flag = (volatile int*)(drained + 1) + 1;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  kernel_started();
  if (threadIdx.x == 0) {
    for (int i = 0; i < S; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], 1); }
    for (int i = 0; i < NB; ++i) { mbar_init(&acc_full[i], 1); mbar_init(&acc_empty[i], 4 * Shape::groups); }
    for (int i = 0; i < SS; ++i) { mbar_init(&sc_full[i], 32); mbar_init(&sc_empty[i], 4 * Shape::groups); }
    mbar_init(drained, 1);
    *dead_flag = 0;
    mbar_fence_init();
  }
  if (warp == 3) tmem_alloc(&tmem_base, Shape::tmem_cols);
  tmem_fence_before();
  __syncthreads();
  tmem_fence_after();
  const uint32_t tmem = tmem_base;
  kernel_inputs_ready();
  const MarginsWait wait{p.spin_limit, dead_flag, p.status};
  const int nk = p.blocks;

  if (warp == 0) {
    if (lane == 0) {
      uint32_t it = 0;
      bool ok = true;
      for (int t = blockIdx.x; t < p.tiles && ok; t += gridDim.x) {
        const int row0 = t / p.tiles_m * MG_ROWS, m0 = t % p.tiles_m * BN;
        for (int k = 0; k < nk; ++k, ++it) {
          const uint32_t s = it % S;
          if (!(ok = wait(&empty[s], (it / S & 1) ^ 1, 41))) break;
          if (k == p.drop_block) continue;
          unsigned char* stage = ring + s * Shape::stage_bytes;
          mbar_arrive_expect_tx(&full[s], Shape::stage_bytes);
          tma_load_2d(stage, &map_q, k * Q_BLOCK, row0, &full[s]);
          tma_load_2d(stage + MG_ROWS * Q_BLOCK, &map_m, k * Q_BLOCK, m0, &full[s]);
        }
      }
      if (!ok)  // copies in flight land before the block ends: the last S requests
        for (uint32_t j = it > S ? it - S : 0; j < it; ++j) mbar_wait_bounded(&full[j % S], j / S & 1, p.spin_limit);
    }
  } else if (warp == 1) {
    if (lane == 0) {
      uint32_t it = 0;
      bool ok = true;
      for (int t = blockIdx.x; t < p.tiles && ok; t += gridDim.x) {
        for (int k = 0; k < nk; ++k, ++it) {
          const uint32_t s = it % S, b = it % NB;
          if (!(ok = wait(&acc_empty[b], (it / NB & 1) ^ 1, 42) && wait(&full[s], it / S & 1, 43))) break;
          tmem_fence_after();
          const uint32_t a = (uint32_t)__cvta_generic_to_shared(ring + s * Shape::stage_bytes), m = a + MG_ROWS * Q_BLOCK;
#pragma unroll
          for (int j = 0; j < Q_BLOCK / 32; ++j)  // 32 columns a product
            mma_e4m3(tmem + b * BN, mma_operand(a + 32 * j), mma_operand(m + 32 * j), mma_shape<BN>(), j > 0);
          mma_commit(&empty[s]);
          mma_commit(&acc_full[b]);
        }
      }
      if (!ok) {  // products in flight end before tensor memory is given back
        mma_commit(drained);
        mbar_wait_bounded(drained, 0, p.spin_limit);
      }
    }
  } else if (warp == 2) {
    uint32_t it = 0;
    bool ok = true;
    for (int t = blockIdx.x; t < p.tiles && ok; t += gridDim.x) {
      const int row0 = t / p.tiles_m * MG_ROWS, m0 = t % p.tiles_m * BN;
      for (int k = 0; k < nk; ++k, ++it) {
        const uint32_t q = it % SS;
        if (!(ok = wait(&sc_empty[q], (it / SS & 1) ^ 1, 44))) break;
        const uint32_t dst = (uint32_t)__cvta_generic_to_shared(scales + q * (MG_ROWS + BN));
#pragma unroll
        for (int i = 0; i < MG_ROWS / 32; ++i) {
          const int r = row0 + 32 * i + lane;
          const bool in = r < p.n_rows;
          cp_async4_or_zero(dst + (32 * i + lane) * 4, p.q_scales + (in ? r : 0) * p.ld_qs + k, in);
        }
#pragma unroll
        for (int i = 0; i < (BN + 31) / 32; ++i) {
          const int m = m0 + 32 * i + lane;
          const bool in = m < p.n_models;
          if (32 * i + lane < BN) cp_async4_or_zero(dst + (MG_ROWS + 32 * i + lane) * 4, p.m_scales + (in ? m : 0) * p.ld_ms + k, in);
        }
        cp_async_arrive(&sc_full[q]);
      }
      ok = __all_sync(0xffffffffu, ok);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
  } else if (warp >= 4) {
    const int quarter = warp & 3, group = (warp - 4) >> 2;  // a warp reads the 32 lanes of tensor memory of its number modulo 4
    const uint32_t my_tmem = tmem + ((uint32_t)(32 * quarter) << 16) + group * COLS;
    const uint32_t my_staging = (uint32_t)__cvta_generic_to_shared(staging + (warp - 4) * 32 * 80);
    const uint32_t scales_at = (uint32_t)__cvta_generic_to_shared(scales);
    uint32_t it = 0;
    bool ok = true;
    for (int t = blockIdx.x; t < p.tiles; t += gridDim.x) {
      const int row0 = t / p.tiles_m * MG_ROWS + 32 * quarter, m0 = t % p.tiles_m * BN + group * COLS;
      uint64_t acc[COLS / 2];
#pragma unroll
      for (int i = 0; i < COLS / 2; ++i) acc[i] = 0;
      for (int k = 0; k < nk; ++k, ++it) {
        const uint32_t b = it % NB, q = it % SS;
        ok = wait(&sc_full[q], it / SS & 1, 45) && wait(&acc_full[b], it / NB & 1, 46);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        tmem_fence_after();
        const uint32_t slot = scales_at + q * Shape::slot_bytes;
        float rs;
        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(rs) : "r"(slot + (32 * quarter + lane) * 4));
        const uint64_t rs2 = pair_of(__float_as_uint(rs), __float_as_uint(rs));
        const uint32_t cs = slot + (MG_ROWS + group * COLS) * 4;
#pragma unroll
        for (int c = 0; c < COLS; c += 16) {
          uint32_t v[16];
          tmem_load16(my_tmem + b * BN + c, v);
          tmem_wait_load(v);
#pragma unroll
          for (int e = 0; e < 16; e += 4) {
            const uint4 w = lds16(cs + (c + e) * 4);
            acc[(c + e) / 2] = fma2(pair_of(v[e], v[e + 1]), mul2(rs2, pair_of(w.x, w.y)), acc[(c + e) / 2]);
            acc[(c + e) / 2 + 1] = fma2(pair_of(v[e + 2], v[e + 3]), mul2(rs2, pair_of(w.z, w.w)), acc[(c + e) / 2 + 1]);
          }
        }
        tmem_fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive_one(&acc_empty[b]);
          mbar_arrive_one(&sc_empty[q]);
        }
      }
      if (!ok) break;
      // 16 words of each row at a time: 16 fp32 margins, or 32 of bf16
      constexpr int PER_WORD = sizeof(OT) == 4 ? 1 : 2, STEP = 16 * PER_WORD < COLS ? 16 * PER_WORD : COLS, WORDS = STEP / PER_WORD;
#pragma unroll
      for (int c = 0; c < COLS; c += STEP) {
        __syncwarp();
#pragma unroll
        for (int e = 0; e < WORDS; e += 4) {
          uint32_t w[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if constexpr (PER_WORD == 1) {
              const uint64_t a = acc[(c + e + i) / 2];
              w[i] = (e + i) % 2 ? (uint32_t)(a >> 32) : (uint32_t)a;
            } else {
              const uint64_t a = acc[c / 2 + e + i];
              const __nv_bfloat162 h = __floats2bfloat162_rn(__uint_as_float((uint32_t)a), __uint_as_float((uint32_t)(a >> 32)));
              w[i] = *(const uint32_t*)&h;
            }
          }
          sts16(my_staging + lane * 80 + e * 4, make_uint4(w[0], w[1], w[2], w[3]));
        }
        __syncwarp();
        if (p.vector) {
          constexpr int LANES = WORDS / 4;  // that cover a row
#pragma unroll
          for (int j = 0; j < LANES; ++j) {
            const int r = j * (32 / LANES) + lane / LANES, e = lane % LANES * 4, m = m0 + c + e * PER_WORD;
            const uint4 w = lds16(my_staging + r * 80 + e * 4);
            if (row0 + r >= p.n_rows) continue;
            OT* to = (OT*)p.Z + (long long)(row0 + r) * p.ld_z + m;
            if (m + 4 * PER_WORD <= p.n_models) {
              *(uint4*)to = w;
            } else {
              const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
              for (int i = 0; i < 4 * PER_WORD; ++i)
                if (m + i < p.n_models) {
                  if constexpr (PER_WORD == 1) ((uint32_t*)to)[i] = x[i];
                  else ((uint16_t*)to)[i] = (uint16_t)(x[i / 2] >> 16 * (i % 2));
                }
            }
          }
        } else {
          constexpr int LANES = STEP < 32 ? STEP : 32;  // a margin each
#pragma unroll 4
          for (int r0 = 0; r0 < 32; r0 += 32 / LANES) {
            const int r = r0 + lane / LANES, e = lane % LANES, m = m0 + c + e;
            uint32_t w;
            asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w) : "r"(my_staging + r * 80 + e / PER_WORD * 4));
            if (row0 + r < p.n_rows && m < p.n_models) {
              OT* to = (OT*)p.Z + (long long)(row0 + r) * p.ld_z + m;
              if constexpr (PER_WORD == 1) *(uint32_t*)to = w;
              else *(uint16_t*)to = (uint16_t)(w >> 16 * (e % 2));
            }
          }
        }
      }
    }
  }
  tmem_fence_before();
  __syncthreads();
  tmem_fence_after();
  if (warp == 3) tmem_free(tmem, Shape::tmem_cols);
}

}  // namespace wpsgd
