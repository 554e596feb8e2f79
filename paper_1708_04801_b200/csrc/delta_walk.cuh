// The walk over a chain's chunks by tcgen05: all labels of a head (up to 128) are the lanes of tensor memory (see delta_chunk.cuh for the mathematics).
//
// Everything that ties one product to the next has labels as rows: S^T [labels x features], R^T and U^T [labels x 64]. They are A operands in tensor memory, written there by
// eight warps that take the accumulators out (a thread has a label and half of the columns), so that K, Q, T and P, as they lie in shared memory, are B operands of all
// products: K and Q tiles of 128 bytes a row with the 128-byte swizzle (K once with features as k and once with rows as k), T and P columns of 16 x 16 blocks with the 32-byte swizzle. A
// chunk is a string of three products with the warps' work between them: R^T = S^T K^T (two parts of S), U^T = R^T T^T (three pairs of parts, columns from the block on), and
// dS^T = (r U)^T K (two parts); S^T Q^T and U^T P^T run beside it, and the answers leave while the next chunk's first product runs. S stays in registers in fp32.
//
// Roles: eight warps with S, as above; four that scale and bring out the answers; three that bring the chunks; one thread that issues the products.
//
// Bounds: the string. 56 products of 16 of k a chunk are 1900 cycles of the tensor cores at 128 x 128; a chunk takes 4700: S to two parts 900, its product 600, R 570, T R 700, r U 400, the
// step of S 600, and 450 of waiting for barriers that are complete (160 to 190 cycles each). 65536 rows in 16 chains of 8 heads of features and 16 of labels, 128 x 128: 370 us; by mma.sync
// 720; with the answers by the eight warps, between the other steps, 394; with them and the labels by threads that have a label each, 445 (a store of 2 bytes a lane for each row: 615).
// With models and steps kept for a gradient, half the rows: 227 (their stores, 48 KB a chunk, take 1800 cycles of the string). Tried and slower: one lane that polls for its warp (394 to
// 440), the next labels loaded before S (370 to 390), models kept while U is formed (227 to 231).
#pragma once

#include "delta_chunk.cuh"
#include "tmem.cuh"

namespace wpsgd {

constexpr int WALK_LABELS = 128, WALK_WARPS = 8, WALK_ANSWERS = 4, WALK_COPIERS = 3, WALK_FIRST_COPIER = WALK_WARPS + WALK_ANSWERS, WALK_ISSUER = WALK_FIRST_COPIER + WALK_COPIERS,
              WALK_THREADS = 32 * (WALK_ISSUER + 1);
// Registers of a thread: 128 as launched; the warps that hold S take from the others, 256 * 168 + 256 * 88 = 512 * 128
constexpr int WALK_REGS = 168, WALK_FEWER_REGS = 88;
constexpr uint32_t WALK_COLUMNS = 512;
// Columns of tensor memory. fp32: dS, R and then U, the answers. bf16: two parts each of S, of R and then r U, of U.
constexpr uint32_t TM_DS = 0, TM_R = 128, TM_O = 192, TM_S = 256, TM_S_LO = 320, TM_RH = 384, TM_RL = 416, TM_UH = 448, TM_UL = 480;

// A wait that gives up after its own limit, or when another role has. False: leave.
struct WalkWait {
  long long limit;
  volatile int* dead;
  __device__ __forceinline__ bool operator()(unsigned long long* bar, uint32_t parity) const {
    for (long long i = 0; i < limit; ++i) {
      if (mbar_try_wait(bar, parity)) return true;
      if (*dead) break;
    }
    return false;
  }
  __device__ __forceinline__ bool warp(unsigned long long* bar, uint32_t parity) const { return __all_sync(0xffffffffu, (*this)(bar, parity)); }
};

// What the roles tell each other: products done (one arrival each), operands written or accumulators read (one of each warp)
struct WalkBarriers {
  unsigned long long r_done, q_done, u_done, s_done, o_done, drained, s_there[2], r_there, u_there, o_read, p_there;
};

template <int DK, bool SAVE>
__global__ void __launch_bounds__(WALK_THREADS, 1) delta_walk_kernel(const __grid_constant__ DeltaChunkParams p, const __grid_constant__ DeltaMaps maps) {
  using Shape = ChainShape<DK, 8>;
  constexpr int STAGES = Shape::stages, HALF = DK / 2;  // features of a thread
  extern __shared__ unsigned char chain_smem[];
  __shared__ ChunkBarriers bars[STAGES];
  __shared__ WalkBarriers w;
  __shared__ uint32_t tmem_base;
  __shared__ int dead_flag;
  volatile int* dead = &dead_flag;
  const int tid = threadIdx.x, warp = warp_index(), lane = tid & 31;
  unsigned char* const ring = chain_smem + (-smem32(chain_smem) & 1023u);
  if (tid == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(&bars[s].rows, 32 * WALK_COPIERS);
      mbar_init(&bars[s].bulk, 1);
      mbar_init(&bars[s].empty, WALK_WARPS + WALK_ANSWERS + 1);
    }
    for (unsigned long long* b : {&w.r_done, &w.q_done, &w.u_done, &w.s_done, &w.o_done, &w.drained}) mbar_init(b, 1);
    for (unsigned long long* b : {&w.s_there[0], &w.s_there[1], &w.r_there, &w.u_there}) mbar_init(b, WALK_WARPS);
    mbar_init(&w.o_read, WALK_ANSWERS);
    mbar_init(&w.p_there, WALK_WARPS + WALK_ANSWERS);
    dead_flag = 0;
    mbar_fence_init();
  }
  if (warp == WALK_ISSUER) tmem_alloc(&tmem_base, WALK_COLUMNS);
  tmem_fence_before();
  __syncthreads();
  tmem_fence_after();
  const uint32_t tm = tmem_base;
  kernel_inputs_ready();
  const int h = blockIdx.x % p.hv, chain = p.order[blockIdx.x / p.hv], kh = h / (p.hv / p.hk);
  const int first = p.chunk_off[chain], n = p.chunk_off[chain + 1] - first;
  const DeltaSpan span = span_of(p, first, n);
  const WalkWait wait = {p.spin_limit, dead};
  auto give_up = [&](int i) {
    *dead = 1;
    set_status(p.status, DEV_TIMEOUT, 25, i);
  };

  const uint32_t lanes = tm + ((uint32_t)(warp & 3) << 21);  // of a warp that takes accumulators out: 32 lanes, or labels
  const int labels0 = (warp & 3) * 32, t = lane & 3;
  // 32 labels and rows, from t0 on, of an accumulator: acc[z][4 n + e], label 16 z + lane / 4 (e < 2) or 8 further, row t0 + 8 n + 2 t + e % 2
  uint32_t acc[2][16];
  auto take = [&](uint32_t at, int t0) {
    tmem_load_tiles(lanes + at + t0, acc[0]);
    tmem_load_tiles(lanes + at + t0 + (16u << 16), acc[1]);
    tmem_wait_load(acc[0], acc[1]);
  };
  auto tell = [&](unsigned long long* bar) {
    tmem_fence_before();
    __syncwarp();
    if (lane == 0) arrive(bar);
  };
  // 32 labels and rows (a word has two rows) by way of a tile in shared memory, of which `own` are the warp's, to rows in memory
  auto put_rows = [&](const uint32_t (&words)[2][8], unsigned char* own, auto vec, __nv_bfloat16* to, long long ld, int rows, int cols) {
    const uint32_t at = smem32(own) + lane_nk(lane, Shape::vrow);
    __syncwarp();
#pragma unroll
    for (int z = 0; z < 2; ++z)
#pragma unroll
      for (int y = 0; y < 2; ++y) stsm_t(at + z * 32 + y * 16 * Shape::vrow * 2, words[z][4 * y], words[z][4 * y + 1], words[z][4 * y + 2], words[z][4 * y + 3]);
    __syncwarp();
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int row = 8 * u + lane / 4, col = lane % 4 * 8;
      if (row >= rows || col >= cols) continue;
      const uint4 v = *(const uint4*)(own + (row * Shape::vrow + col) * 2);
      __nv_bfloat16* o = to + row * ld + col;
      if (decltype(vec)::value) {
        *(uint4*)o = v;
      } else {
        const uint32_t two[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (col + e < cols) ((unsigned short*)o)[e] = (unsigned short)(two[e / 2] >> (16 * (e % 2)));
      }
    }
  };

  if (warp >= WALK_FIRST_COPIER) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(WALK_FEWER_REGS));
    if (warp < WALK_ISSUER) {
      bring_chunks<DK, 8>(p, maps, p.v, smem32(ring), first, false, n, span, h, kh, 0, warp - WALK_FIRST_COPIER, WALK_COPIERS, lane, bars);
    } else {
      if (elect_one()) {
        int i = 0;
        for (; i < n; ++i) {
          const int s = i % STAGES;
          const uint32_t k_at = smem32(ring + s * Shape::stage), q_at = k_at + Shape::q_at, t_at = k_at + Shape::block_at;
          if (!wait(&bars[s].bulk, (i / STAGES) & 1) || !wait(&bars[s].rows, (i / STAGES) & 1)) break;
          if (!p.maps || span.len(i) < DC) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // features and queries that threads have copied
          bool there = true;
#pragma unroll
          for (int j = 0; j < HALF / 32; ++j) {  // 32 features of either half at a time, as they come
            there = there && wait(&w.s_there[j], i & 1);
            if (!there) break;
            tmem_fence_after();
#pragma unroll
            for (int part = 0; part < 2; ++part)
#pragma unroll
              for (int y = 0; y < 4; ++y) {
                const int x = y / 2 * (HALF / 16) + 2 * j + y % 2;
                mma_bf16(tm + TM_R, tm + (part ? TM_S_LO : TM_S) + 8 * x, mma_operand(k_at + x / 4 * WIDE_BYTES + x % 4 * 32), mma_shape16(DC, false), j || part || y);
              }
          }
          if (!there) break;
          mma_commit(&w.r_done);
          // a triangle's column of blocks x: rows of the result from 16 x on
          auto triangle = [&](uint32_t d, uint32_t hi, uint32_t lo, uint32_t at, bool add) {
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              mma_bf16(tm + d + 16 * x, tm + hi + 8 * x, mma_operand32(at + tri_at(x, x)), mma_shape16(DC - 16 * x, false), add || x);
              mma_bf16(tm + d + 16 * x, tm + lo + 8 * x, mma_operand32(at + tri_at(x, x)), mma_shape16(DC - 16 * x, false), true);
              mma_bf16(tm + d + 16 * x, tm + hi + 8 * x, mma_operand32(at + DC_T_LO + tri_at(x, x)), mma_shape16(DC - 16 * x, false), true);
            }
          };
          if (!wait(&w.r_there, i & 1)) break;
          tmem_fence_after();
          triangle(TM_R, TM_RH, TM_RL, t_at, false);
          mma_commit(&w.u_done);
          if (i > 0 && !wait(&w.o_read, (i - 1) & 1)) break;
          tmem_fence_after();
#pragma unroll
          for (int x = 0; x < DK / 16; ++x) mma_bf16(tm + TM_O, tm + TM_S + 8 * x, mma_operand(q_at + x / 4 * WIDE_BYTES + x % 4 * 32), mma_shape16(DC, false), x > 0);
          mma_commit(&w.q_done);
          if (!wait(&w.u_there, i & 1)) break;
          tmem_fence_after();
#pragma unroll
          for (int part = 0; part < 2; ++part)
#pragma unroll
            for (int x = 0; x < 4; ++x) mma_bf16(tm + TM_DS, tm + (part ? TM_RL : TM_RH) + 8 * x, mma_operand_outer(k_at + x * 2048, WIDE_BYTES), mma_shape16(DK, true), part || x);
          mma_commit(&w.s_done);
          if (!wait(&w.p_there, i & 1)) break;
          tmem_fence_after();
          triangle(TM_O, TM_UH, TM_UL, t_at + DC_P, true);
          mma_commit(&w.o_done);
          mma_commit(&bars[s].empty);
        }
        if (i < n) give_up(i);
        mma_commit(&w.drained);  // what was issued is done before tensor and shared memory go
        mbar_wait_bounded(&w.drained, 0, DRAIN_LIMIT);
      }
      __syncwarp();
    }
  } else if (warp >= WALK_WARPS) {  // answers
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(WALK_FEWER_REGS));
    bool ok = true;
    for (int i = 0; i < n; ++i) {
      const int s = i % STAGES;
      unsigned char* block = ring + s * Shape::stage + Shape::block_at;
      const DeltaFactors* f = (const DeltaFactors*)(block + DC_FACTORS);
      // scale c S^T Q^T, to which U^T P^T is added
      if (!(ok = wait.warp(&bars[s].bulk, (i / STAGES) & 1) && wait.warp(&w.q_done, i & 1))) break;
      tmem_fence_after();
#pragma unroll
      for (int t0 = 0; t0 < DC; t0 += 32) {
        take(TM_O, t0);
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          const float2 c = *(const float2*)(f->c + t0 + 8 * m + 2 * t);
          const float cx = p.scale * c.x, cy = p.scale * c.y;
#pragma unroll
          for (int z = 0; z < 2; ++z)
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
              acc[z][4 * m + e] = __float_as_uint(cx * __uint_as_float(acc[z][4 * m + e]));
              acc[z][4 * m + e + 1] = __float_as_uint(cy * __uint_as_float(acc[z][4 * m + e + 1]));
            }
        }
        tmem_store_tiles(lanes + TM_O + t0, acc[0]);
        tmem_store_tiles(lanes + TM_O + t0 + (16u << 16), acc[1]);
      }
      tmem_wait_store();
      tell(&w.p_there);
      if (!(ok = wait.warp(&w.o_done, i & 1))) break;
      tmem_fence_after();
      uint32_t words[2][2][8];
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        take(TM_O, 32 * y);
#pragma unroll
        for (int z = 0; z < 2; ++z)
#pragma unroll
          for (int e = 0; e < 8; ++e) words[y][z][e] = pack2(__uint_as_float(acc[z][2 * e]), __uint_as_float(acc[z][2 * e + 1]));
      }
      tell(&w.o_read);
      // by way of the place of T and P, which no product reads any more
      static_assert(DC * Shape::vrow * 2 <= DC_FACTORS, "answers must fit");
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        unsigned char* own = block + (32 * y * Shape::vrow + labels0) * 2;
        __nv_bfloat16* out = p.out + (span.row0 + (long long)i * DC + 32 * y) * p.ld_out + h * p.dv + labels0;
        if (p.vec_out) put_rows(words[y], own, std::true_type(), out, p.ld_out, span.len(i) - 32 * y, p.dv - labels0);
        else put_rows(words[y], own, std::false_type(), out, p.ld_out, span.len(i) - 32 * y, p.dv - labels0);
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // the next block comes there by a bulk copy
      __syncwarp();
      if (lane == 0) arrive(&bars[s].empty);
    }
    if (!ok && lane == 0) give_up(n);
    __syncwarp();
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(WALK_REGS));
    const int half = warp >> 2, label = labels0 + lane, t0 = half * 32, f0 = half * HALF;
    const bool there = label < p.dv;
    const long long model = (((long long)chain * p.hv + h) * p.dv + label) * p.dk;
    const bool vec = p.dk % 4 == 0 && (((uintptr_t)p.W0 | (uintptr_t)p.W) & 15) == 0;
    float S[HALF];
#pragma unroll
    for (int x = 0; x < HALF; x += 4) {
      float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      if (p.W0 && there) {
        const float* from = p.W0 + model + f0 + x;
        const int left = p.dk - f0 - x;
        if (vec) {
          if (left > 0) v = *(const float4*)from;
        } else {
          if (left > 0) v.x = from[0];
          if (left > 1) v.y = from[1];
          if (left > 2) v.z = from[2];
          if (left > 3) v.w = from[3];
        }
      }
      S[x] = v.x, S[x + 1] = v.y, S[x + 2] = v.z, S[x + 3] = v.w;
    }
    unsigned char* const own = ring + Shape::v_at + (t0 * Shape::vrow + labels0) * 2;  // where the warp's labels come in
    // two parts of x, four values to a tile of 8 columns, to operands
    auto put_parts = [&](const float (&x)[2][16], uint32_t hi_at, uint32_t lo_at, uint32_t (&hi)[2][8]) {
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        uint32_t lo[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) split2(x[z][2 * e], x[z][2 * e + 1], hi[z][e], lo[e]);
        tmem_store_words(lanes + hi_at + t0 / 2 + ((uint32_t)z << 20), hi[z]);
        tmem_store_words(lanes + lo_at + t0 / 2 + ((uint32_t)z << 20), lo);
      }
    };
    float last = 1.0f;
    bool ok = true;
    for (int i = 0; i <= n; ++i) {
      const int s = i % STAGES;
      const unsigned char* st = ring + s * Shape::stage;
      const DeltaFactors* f = (const DeltaFactors*)(st + Shape::block_at + DC_FACTORS);
      const long long which = (long long)(first + i) * p.hv + h;
      // S^T <- e^{b_C} S^T + dS^T, and its parts
      if (i > 0) {
        if (!(ok = wait.warp(&w.s_done, (i - 1) & 1))) break;
        tmem_fence_after();
      }
#pragma unroll
      for (int j = 0; j < HALF / 32; ++j) {
        if (i > 0) {
          uint32_t v[32];
          tmem_load32(lanes + TM_DS + f0 + 32 * j, v);
#pragma unroll
          for (int e = 0; e < 32; ++e) S[32 * j + e] = fmaf(last, S[32 * j + e], __uint_as_float(v[e]));
        }
        if (i == n) continue;
        uint32_t hi[16], lo[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) split2(S[32 * j + 2 * e], S[32 * j + 2 * e + 1], hi[e], lo[e]);
        tmem_store16(lanes + TM_S + f0 / 2 + 16 * j, hi);
        tmem_store16(lanes + TM_S_LO + f0 / 2 + 16 * j, lo);
        tmem_wait_store();
        tell(&w.s_there[j]);
      }
      if (i == n) break;
      if (SAVE && label < p.dvp) {  // models before the chunk, one bf16 part
        uint4* to = (uint4*)(p.starts + which * p.dvp * DK + model_unit(label, f0 / 8, p.dvp, DK));
#pragma unroll
        for (int e = 0; e < HALF / 8; ++e)
          to[e * model_labels(label, p.dvp)] = make_uint4(pack2(S[8 * e], S[8 * e + 1]), pack2(S[8 * e + 2], S[8 * e + 3]), pack2(S[8 * e + 4], S[8 * e + 5]), pack2(S[8 * e + 6], S[8 * e + 7]));
      }
      // R^T = beta (V^T - c S^T K^T)
      float x[2][16];
      uint32_t words[2][8];
      {
        uint32_t v[2][2][4];
        if (!(ok = wait.warp(&bars[s].bulk, (i / STAGES) & 1) && wait.warp(&bars[s].rows, (i / STAGES) & 1))) break;
#pragma unroll
        for (int z = 0; z < 2; ++z)
#pragma unroll
          for (int y = 0; y < 2; ++y) ldsm_t(v[z][y], smem32(own) + s * Shape::stage + lane_nk(lane, Shape::vrow) + z * 32 + y * 16 * Shape::vrow * 2);
        if (!(ok = wait.warp(&w.r_done, i & 1))) break;
        tmem_fence_after();
        take(TM_R, t0);
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          const float2 c = *(const float2*)(f->c + t0 + 8 * m + 2 * t), be = *(const float2*)(f->beta + t0 + 8 * m + 2 * t);
#pragma unroll
          for (int z = 0; z < 2; ++z)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const uint32_t two = v[z][m / 2][m % 2 * 2 + e];
              x[z][4 * m + 2 * e] = be.x * (__uint_as_float(two << 16) - c.x * __uint_as_float(acc[z][4 * m + 2 * e]));
              x[z][4 * m + 2 * e + 1] = be.y * (__uint_as_float(two & 0xffff0000u) - c.y * __uint_as_float(acc[z][4 * m + 2 * e + 1]));
            }
        }
      }
      put_parts(x, TM_RH, TM_RL, words);
      tmem_wait_store();
      tell(&w.r_there);
      // U and r U
      if (!(ok = wait.warp(&w.u_done, i & 1))) break;
      tmem_fence_after();
      take(TM_R, t0);
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        const float2 r = *(const float2*)(f->r + t0 + 8 * m + 2 * t);
#pragma unroll
        for (int z = 0; z < 2; ++z)
#pragma unroll
          for (int e = 0; e < 4; e += 2) {
            x[z][4 * m + e] = r.x * __uint_as_float(acc[z][4 * m + e]);
            x[z][4 * m + e + 1] = r.y * __uint_as_float(acc[z][4 * m + e + 1]);
          }
      }
      put_parts(x, TM_RH, TM_RL, words);
      tmem_wait_store();
      tell(&w.u_there);
      last = f->last;
#pragma unroll
      for (int z = 0; z < 2; ++z)
#pragma unroll
        for (int e = 0; e < 16; ++e) x[z][e] = __uint_as_float(acc[z][e]);
      put_parts(x, TM_UH, TM_UL, words);
      tmem_wait_store();
      tell(&w.p_there);
      if (SAVE) put_rows(words, own + s * Shape::stage, std::true_type(), p.steps + (which * DC + t0) * p.dvp + labels0, p.dvp, 32, p.dvp - labels0);
      __syncwarp();
      if (lane == 0) arrive(&bars[s].empty);
    }
    if (!ok) {
      if (lane == 0) give_up(n);
    } else if (p.W && there) {
      float* to = p.W + model + f0;
#pragma unroll
      for (int x = 0; x < HALF; x += 4) {
        const int left = p.dk - f0 - x;
        if (vec) {
          if (left > 0) *(float4*)(to + x) = make_float4(S[x], S[x + 1], S[x + 2], S[x + 3]);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (e < left) to[x + e] = S[x + e];
        }
      }
    }
    __syncwarp();
  }
  kernel_started();
  tmem_fence_before();
  __syncthreads();
  tmem_fence_after();
  if (warp == WALK_ISSUER) tmem_free(tm, WALK_COLUMNS);
}

}  // namespace wpsgd
