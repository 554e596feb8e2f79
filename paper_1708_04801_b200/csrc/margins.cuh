// Margins of many models on many rows, both 8-bit with a scale for each block of 128 columns:
//
//   Z[i, m] = sum_b s_i,b t_m,b D_b[i, m],   D_b[i, m] = sum_{c in block b} q_i,c p_m,c
//
// D_b is a product of 8-bit matrices, formed by the tensor cores (tcgen05.mma kind::f8f6f4, fp32 sums in tensor memory) for a tile of 128
// rows and BN models, one block of 128 columns at a time; the scales differ from block to block on both sides, so each D_b is read
// back and added to fp32 registers with its scales while the tensor cores form the next ones in other buffers.
//
// Few tiles with many blocks of columns: a cluster of CTAs per tile, each with a share of the blocks, whose sums meet in the first.
// 2 rows of 5918 columns on 15 models: 16.1 us with one CTA, 6.6 with eight, see margins_of for the rule.
//
// Bound by the rows where there are few models (262144 rows of 4096 columns on 16: 177 us, 6.3 TB/s), else by the way of D_b from the
// tensor cores to the sums (65536 rows of 4096 columns on 1024 models: 480 us, 1150 TFLOP/s). Of 1650 cycles per block of columns and SM the products take 520
// and the adding warps 900 (740 to read 128 KB of fragments from tensor memory, some 200 bytes a cycle); these wait 220 more for products and 80 for scales,
// storing takes 150, and 300 are not accounted for. A buffer is refilled when all adding warps have read it, and nothing is multiplied
// while a tile is stored.
//
// One persistent CTA per SM, a role per warp: warp 0 brings the tiles of Q and M into a ring of stages (TMA, 128-byte swizzle; what lies outside
// the matrices arrives as zeros), warp 1 issues the products, warp 2 brings the scales of a block's 128 rows and BN models (cp.async) into a
// ring of its own, warp 3 owns the tensor memory, the warps from 4 on add up. They read tensor memory in the order of a matrix fragment, four rows
// and 2 of 8 models per thread, and not a row per thread: a thread then needs COLS / 4 + 4 scales for COLS sums instead of COLS + 1,
// and it was the return of those from shared memory (128 bytes a cycle) that bounded the kernel.
// Every wait is bounded. When one runs out it is recorded in the status word, all roles leave, the copies and products in flight are waited
// for (bounded again), and the tensor memory is given back.
#pragma once

#include <cuda.h>

#include "async.cuh"
#include "common.cuh"
#include "quantize.cuh"
#include "tmem.cuh"

namespace wpsgd {

constexpr int MG_ROWS = 128;       // of a tile: the lanes of tensor memory
constexpr int MG_WINDOW = 4;       // blocks of columns whose scales are brought together
constexpr int MG_WINDOWS = 2;      // of them in shared memory

template <int BN>
struct MarginsShape {
  static constexpr int cols = BN == 256 ? 64 : BN == 128 ? 32 : 16;  // models of an adding warp
  static constexpr int groups = BN / cols;                           // of four such warps
  static constexpr int threads = 128 + 128 * groups;
  static constexpr int buffers = BN == 256 ? 2 : 4;   // of D_b in tensor memory
  static constexpr int tmem_cols = buffers * BN;      // a power of two, 64 .. 512
  static constexpr int stage_bytes = (MG_ROWS + BN) * Q_BLOCK;
  static constexpr int slot = MG_ROWS + BN + 8;       // scales of a block; + 8: 4 blocks of 8 rows lie in different banks
  static constexpr int fixed_bytes = 1024 + MG_WINDOWS * MG_WINDOW * slot * 4 + 512;  // 1024: alignment of the ring
  static constexpr int stages = (227 * 1024 - fixed_bytes) / stage_bytes < 10 ? (227 * 1024 - fixed_bytes) / stage_bytes : 10;
  static constexpr int smem = fixed_bytes + stages * stage_bytes;
  // the others' sums reach the first CTA of a cluster through its ring
  static constexpr int max_splits = 7 * BN * MG_ROWS * 4 <= stages * stage_bytes ? 8 : 3 * BN * MG_ROWS * 4 <= stages * stage_bytes ? 4 : 1;
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
  int splits;                     // CTAs of a cluster that share a tile's blocks of columns (1: none; more: one tile per cluster)
  bool pairs;                     // two neighbouring margins of a row share an aligned access
  long long spin_limit;
  long long drop_block;           // test hook: this block of columns is never requested (-1: none)
  DevStatus* status;
};

// ---- tcgen05 ---------------------------------------------------------------------------------------------------------------
// D fp32, A and B e4m3, both with contiguous k, M = 128
template <int BN>
__host__ __device__ constexpr uint32_t mma_shape() { return 1u << 4 | (uint32_t)(BN >> 3) << 17 | (uint32_t)(MG_ROWS >> 4) << 24; }
__device__ __forceinline__ void mma_e4m3(uint32_t d, uint64_t a, uint64_t b, uint32_t shape, bool add) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b),
               "r"(shape), "r"((uint32_t)add)
               : "memory");
}
// 8 columns of a warp's 32 lanes in the order of matrix fragments: thread t gets columns 2 (t % 4) and the next of lanes t / 4 (v[0], v[1]),
// t / 4 + 8 (v[2], v[3]), t / 4 + 16 and t / 4 + 24
__device__ __forceinline__ void tmem_load8(uint32_t addr, uint32_t (&v)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x1.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(addr));
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x1.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]) : "r"(addr + (16u << 16)));
}
__device__ __forceinline__ void tmem_wait_load(uint32_t (&v)[8]) {  // names the registers, so that no use of them moves before the wait
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7])::"memory");
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
__device__ __forceinline__ float lds_f32(uint32_t a) {
  float v;
  asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(a));
  return v;
}
__device__ __forceinline__ uint64_t lds_pair(uint32_t a) {
  uint64_t v;
  asm volatile("ld.shared.b64 %0, [%1];" : "=l"(v) : "r"(a));
  return v;
}

__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
// barrier of a cluster, for warps that need not be converged
__device__ __forceinline__ void cluster_sync_any() { asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory"); }

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

// Two margins of a row, of which `left` exist, in one access where they lie on its boundary (pairs)
__device__ __forceinline__ void store_pair(float* to, float2 z, int left, bool pairs) {
  if (pairs && left > 1) {
    *(float2*)to = z;
  } else {
    if (left > 0) to[0] = z.x;
    if (left > 1) to[1] = z.y;
  }
}
__device__ __forceinline__ void store_pair(__nv_bfloat16* to, float2 z, int left, bool pairs) {
  if (pairs && left > 1) {
    *(__nv_bfloat162*)to = __floats2bfloat162_rn(z.x, z.y);
  } else {
    if (left > 0) to[0] = __float2bfloat16_rn(z.x);
    if (left > 1) to[1] = __float2bfloat16_rn(z.y);
  }
}

template <typename OT, int BN, bool SPLIT>
__global__ void __launch_bounds__(MarginsShape<BN>::threads, 1)
margins_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_m, const __grid_constant__ MarginsParams p) {
  using Shape = MarginsShape<BN>;
  constexpr int S = Shape::stages, NB = Shape::buffers, SS = MG_WINDOWS, COLS = Shape::cols;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* ring = (unsigned char*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  float* scales = (float*)(ring + S * Shape::stage_bytes);
  unsigned long long* bars = (unsigned long long*)(scales + MG_WINDOWS * MG_WINDOW * Shape::slot);
  unsigned long long *full = bars, *empty = full + S, *acc_full = empty + S, *acc_empty = acc_full + NB, *sc_full = acc_empty + NB, *sc_empty = sc_full + SS,
                     *drained = sc_empty + SS;
  static_assert(8 * (2 * S + 2 * NB + 2 * SS + 1) + 12 <= 512, "barriers, tensor memory address, flag and count must fit");
  uint32_t& tmem_base = *(uint32_t*)(drained + 1);  // (no static shared memory: the dynamic part may be all of the SM's)
  volatile int* dead_flag = (volatile int*)(drained + 1) + 1;
  volatile uint32_t* issued = (volatile uint32_t*)(drained + 1) + 2;  // stages that the producer has gone through
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;  // (shfl: known to be the same in all lanes)
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
  const int rank = SPLIT ? blockIdx.x % p.splits : 0, first_tile = SPLIT ? blockIdx.x / p.splits : blockIdx.x, tile_step = SPLIT ? gridDim.x / p.splits : gridDim.x;
  const int k0 = SPLIT ? (int)((long long)p.blocks * rank / p.splits) : 0, k1 = SPLIT ? (int)((long long)p.blocks * (rank + 1) / p.splits) : p.blocks;

  if (warp == 0) {
    if (lane == 0) {
      uint32_t it = 0;
      bool ok = true;
      for (int t = first_tile; t < p.tiles && ok; t += tile_step) {
        const int row0 = t / p.tiles_m * MG_ROWS, m0 = t % p.tiles_m * BN;
        for (int k = k0; k < k1; ++k, ++it) {
          const uint32_t s = it % S;
          if (!(ok = wait(&empty[s], (it / S & 1) ^ 1, 41))) break;
          if (k == p.drop_block) continue;
          unsigned char* stage = ring + s * Shape::stage_bytes;
          mbar_arrive_expect_tx(&full[s], Shape::stage_bytes);
          tma_load_2d(stage, &map_q, k * Q_BLOCK, row0, &full[s]);
          tma_load_2d(stage + MG_ROWS * Q_BLOCK, &map_m, k * Q_BLOCK, m0, &full[s]);
        }
      }
      *issued = it;
    }
  } else if (warp == 1) {
    // the whole warp goes through the loop, so that addresses and descriptors stay in uniform registers; one elected thread issues
    const uint64_t first = mma_operand((uint32_t)__cvta_generic_to_shared(ring));
    uint32_t s = 0, s_parity = 0, b = 0, b_parity = 1;
    bool ok = true;
    for (int t = first_tile; t < p.tiles && ok; t += tile_step) {
      for (int k = k0; k < k1; ++k) {
        ok = wait(&full[s], s_parity, 43) && wait(&acc_empty[b], b_parity, 42);
        if (!(ok = __all_sync(0xffffffffu, ok))) break;
        tmem_fence_after();
        const uint64_t q = first + s * (Shape::stage_bytes >> 4), m = q + (MG_ROWS * Q_BLOCK >> 4);
        if (elect_one()) {
#pragma unroll
          for (int j = 0; j < Q_BLOCK / 32; ++j)  // 32 columns a product
            mma_e4m3(tmem + b * BN, q + 2 * j, m + 2 * j, mma_shape<BN>(), j > 0);
          mma_commit(&empty[s]);
          mma_commit(&acc_full[b]);
        }
        __syncwarp();
        if (++s == S) { s = 0; s_parity ^= 1; }
        if (++b == NB) { b = 0; b_parity ^= 1; }
      }
    }
  } else if (warp == 2) {
    // a lane brings one of 4 blocks of 8 rows: 16 bytes of a row in one instruction
    uint32_t win = 0;
    bool ok = true;
    const int ahead = lane % MG_WINDOW, sub = lane / MG_WINDOW;
    for (int t = first_tile; t < p.tiles && ok; t += tile_step) {
      const int row0 = t / p.tiles_m * MG_ROWS, m0 = t % p.tiles_m * BN;
      for (int kw = k0; kw < k1; kw += MG_WINDOW, ++win) {
        if (!(ok = wait(&sc_empty[win % SS], (win / SS & 1) ^ 1, 44))) break;
        const int k = kw + ahead;
        const uint32_t dst = (uint32_t)__cvta_generic_to_shared(scales + (win % SS * MG_WINDOW + ahead) * Shape::slot);
#pragma unroll
        for (int i = 0; i < MG_ROWS; i += 32 / MG_WINDOW) {
          const int r = row0 + i + sub;
          const bool in = r < p.n_rows && k < k1;
          cp_async4_or_zero(dst + (i + sub) * 4, p.q_scales + (in ? r * p.ld_qs + k : 0), in);
        }
#pragma unroll
        for (int i = 0; i < BN; i += 32 / MG_WINDOW) {
          const int m = m0 + i + sub;
          const bool in = m < p.n_models && k < k1;
          cp_async4_or_zero(dst + (MG_ROWS + i + sub) * 4, p.m_scales + (in ? m * p.ld_ms + k : 0), in);
        }
        cp_async_arrive(&sc_full[win % SS]);
      }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
  } else if (warp >= 4) {
    const int quarter = warp & 3, group = (warp - 4) >> 2;  // a warp reads the 32 lanes of tensor memory of its number modulo 4
    const uint32_t my_tmem = tmem + ((uint32_t)(32 * quarter) << 16) + group * COLS;
    const uint32_t my_row = 32 * quarter + lane / 4, my_col = group * COLS + 2 * (lane % 4);  // the first of this thread's rows and models
    const uint32_t scales_at = (uint32_t)__cvta_generic_to_shared(scales);
    uint32_t it = 0, win = 0;
    bool ok = true;
    for (int t = first_tile; t < p.tiles; t += tile_step) {
      uint64_t acc[4][COLS / 8];  // row my_row + 8 i, models my_col + 8 j and the next
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < COLS / 8; ++j) acc[i][j] = 0;
      for (int k = k0; k < k1; ++k, ++it) {
        const uint32_t b = it % NB, q = win % SS;
        ok = ((k - k0) % MG_WINDOW || wait(&sc_full[q], win / SS & 1, 45)) && wait(&acc_full[b], it / NB & 1, 46);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        tmem_fence_after();
        const uint32_t slot = scales_at + (q * MG_WINDOW + (k - k0) % MG_WINDOW) * Shape::slot * 4;
        uint64_t rs[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t r = __float_as_uint(lds_f32(slot + (my_row + 8 * i) * 4));
          rs[i] = pair_of(r, r);
        }
        uint32_t v[2][8];
        tmem_load8(my_tmem + b * BN, v[0]);
#pragma unroll
        for (int c = 0; c < COLS / 8; ++c) {  // the next 8 columns are on their way while these are added
          const uint64_t cs = lds_pair(slot + (MG_ROWS + my_col + 8 * c) * 4);
          tmem_wait_load(v[c % 2]);
          if (c + 1 < COLS / 8) {
            tmem_load8(my_tmem + b * BN + 8 * (c + 1), v[(c + 1) % 2]);
          } else {  // the last of this block: its buffer is free
            tmem_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_one(&acc_empty[b]);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[i][c] = fma2(pair_of(v[c % 2][2 * i], v[c % 2][2 * i + 1]), mul2(rs[i], cs), acc[i][c]);
        }
        if ((k - k0) % MG_WINDOW == MG_WINDOW - 1 || k == k1 - 1) {
          __syncwarp();
          if (lane == 0) mbar_arrive_one(&sc_empty[q]);
          ++win;
        }
      }
      if constexpr (SPLIT) {  // the cluster's sums meet in its first CTA, in the order of the blocks of columns
        constexpr int PT = 128 * Shape::groups;
        const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring) + (threadIdx.x - 128) * 8;
        cluster_sync_any();  // rings are done with
        if (rank > 0) {
          uint32_t to;
          asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(to) : "r"(ring_at));
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < COLS / 8; ++j)
              asm volatile("st.shared::cluster.b64 [%0], %1;" ::"r"(to + (((rank - 1) * 4 + i) * (COLS / 8) + j) * (PT * 8)), "l"(acc[i][j]) : "memory");
        }
        cluster_sync_any();
        if (rank > 0) break;
        for (int r = 1; r < p.splits; ++r)
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < COLS / 8; ++j) acc[i][j] = add2(acc[i][j], lds_pair(ring_at + (((r - 1) * 4 + i) * (COLS / 8) + j) * (PT * 8)));
      }
      if (!ok) break;
      const int row = t / p.tiles_m * MG_ROWS + my_row, model = t % p.tiles_m * BN + my_col;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (row + 8 * i >= p.n_rows) continue;
        OT* to = (OT*)p.Z + (long long)(row + 8 * i) * p.ld_z + model;
#pragma unroll
        for (int j = 0; j < COLS / 8; ++j) store_pair(to + 8 * j, halves(acc[i][j]), p.n_models - model - 8 * j, p.pairs);
      }
    }
  }
  if (SPLIT && warp < 4) {  // as often as the adding warps
    cluster_sync_any();
    cluster_sync_any();
  }
  tmem_fence_before();
  __syncthreads();
  tmem_fence_after();
  if (*dead_flag) {  // copies and products in flight end before the block does and tensor memory is given back
    if (warp == 0 && lane == 0) {
      const uint32_t n = *issued;
      for (uint32_t j = n > S ? n - S : 0; j < n; ++j)
        if (k0 + j % (uint32_t)(k1 - k0) != p.drop_block) mbar_wait_bounded(&full[j % S], j / S & 1, DRAIN_LIMIT);
    }
    if (warp == 1) {
      if (elect_one()) mma_commit(drained);  // by the thread that issued the products: a commit covers its own alone
      __syncwarp();
      if (lane == 0) mbar_wait_bounded(drained, 0, DRAIN_LIMIT);
    }
    __syncthreads();
  }
  if (warp == 3) tmem_free(tmem, Shape::tmem_cols);
}

}  // namespace wpsgd
