// Chains whose labels are vectors, 64 rows at a time on the tensor cores (gated delta rule, see include/wpsgd.h). bf16 rows, fp32 models.
//
// A chunk of C = 64 rows of a head from the models S (features x labels here, W^T): with b the sums of the log decays up to each row of the chunk,
// c_i = e^{b_i}, D_ij = e^{b_i - b_j} for i >= j, the steps U (rows x labels) that all rows take solve a unit triangular system:
//   (I + A) U = R,   A_ij = beta_i D_ij k_i.k_j (i > j),   R = beta (V - c K S)
//   answers          O = scale (c Q S) + P U,   P_ij = scale D_ij q_i.k_j (i >= j)
//   models after it  S' = e^{b_C} S + K^T (r U),  r_i = e^{b_C - b_i}.
// Only S ties the chunks of a chain together. So a first kernel forms T = (I + A)^{-1} and P for all chunks at once, and a second walks
// the chunks of each chain: three products a chunk with S, T and K, and two for the answers.
//
// Columns of S, U, R and O (labels) know nothing of each other, and every product that ties one chunk to the next has labels as rows of its A operand. Heads of more than 64 labels
// walk by tcgen05, with labels as the lanes of tensor memory (delta_walk.cuh). Here are those of fewer, which would leave most of its 128 rows empty: a warp has 16 labels for good:
// S^T, [16 x dk], is the fp32 accumulator of mma.sync m16n8k16, whose layout is that of the A operand of the next product, so S, R and U go from product to product
// in registers, K, Q, T and P come from shared memory as B operands (with ldmatrix, transposed where needed), and nothing is exchanged
// between warps: no barrier but those of the ring that brings the chunks.
//
// Bounds, 65536 rows in 16 chains of four speeds, 8 heads of features and 16 of labels, 128 x 128: the first kernel 205 us, latency of its steps between barriers
// (1.6 instructions a cycle, four blocks an SM); the second 370 us (by mma.sync 720, tensor pipe 55 % and shared memory 65 % of the time). Many chains and heads fill the
// GPU; a single one is bound by the latency of a chunk.
//
// Rounding: an fp32 factor x enters a product as two bf16 parts, x = hi + lo (2^-17 of x is left out): K S and K^T U
// two products, T R and P U three. The answers, which leave as bf16, take S as one bf16 part (1e-3 of them; one part of P would be 2.5e-3).
#pragma once

#include <cuda.h>

#include "async.cuh"
#include "common.cuh"
#include "delta_rows.cuh"

namespace wpsgd {

constexpr int DC = 64;             // rows of a chunk
constexpr int DC_TILE = DC + 8;    // elements from row to row of a 64 x 64 tile in shared memory: ldmatrix reads 8 rows from 8 different bank groups
constexpr int DC_TILE_BYTES = DC * DC_TILE * 2;
// Lower triangles are kept as their ten blocks of 16 x 16, 512 bytes each, column by column: the blocks of a column of blocks are 16 to 64 rows of one
// operand of tcgen05. A row of a block is two units of 16 bytes, swapped in rows 4 to 7 and 12 to 15 (the swizzle of 32 bytes), so that the 8 rows that ldmatrix reads at a time lie in
// different banks.
constexpr int DC_TRI = 10 * 512;
__host__ __device__ constexpr int tri_at(int i, int j) { return (i + j * (7 - j) / 2) * 512; }
__device__ __forceinline__ int tri_unit(int row, int half) { return row * 32 + ((half ^ (row >> 2 & 1)) << 4); }
// What the first kernel leaves for each chunk and head, brought by one copy: T and P in two parts each, the factors of the rows. b is held as b log2(e) = hi + lo
// (its sums are formed in 64 bits): D_ij = 2^{(hi_i - hi_j) + (lo_i - lo_j)} is then as good as its fp32 exponent.
struct DeltaFactors {
  float c[DC], r[DC], beta[DC], hi[DC], lo[DC], last, pad[3];
};
constexpr int DC_T_LO = DC_TRI, DC_P = 2 * DC_TRI, DC_P_LO = 3 * DC_TRI, DC_FACTORS = 4 * DC_TRI, DC_BLOCK = DC_FACTORS + (int)sizeof(DeltaFactors);
static_assert(DC_BLOCK % 16 == 0, "blocks are copied in units of 16 bytes");

struct DeltaChunk {
  long long row0;
  int len, chain;
};

// Rows of bf16 heads that start on 16 bytes; width a multiple of 8
struct DeltaHeads {
  const __nv_bfloat16* p;
  long long ld;
  int heads, width;
};

struct DeltaChunkParams {
  const long long* shard_off;
  long long n_rows;
  int n_chains, hk, hv, dk, dv;  // dk, dv as the caller has them
  int dvp;                       // dv rounded up to 16
  DeltaHeads q, k, v, dout;
  const __nv_bfloat16 *g, *beta;
  long long ld_g, ld_beta;
  float scale;
  int* chunk_off;      // [n_chains + 1]: first chunk of each chain
  int* order;          // [n_chains]: longest first
  DeltaChunk* chunks;  // [chunk_off[n_chains]]
  unsigned char* blocks;        // [chunks][hv][DC_BLOCK]
  __nv_bfloat16* starts;        // [chunks][hv][dvp x DK]: models before the chunk, for the gradient, see model_unit
  __nv_bfloat16* steps;         // [chunks][hv][DC][dvp]: U
  unsigned char* gram;          // [chunks][hv][DC_TRI]: D_ij k_i.k_j, for the gradient; NULL where it is not kept
  const float* W0;
  float* W;
  __nv_bfloat16* out;
  long long ld_out;
  int vec_out, slices;
  int new_out;  // answers of rows outside the chains are set to zeros
  int maps;  // whole chunks come by tensor maps
  int prep_heads;
  long long spin_limit, drop;
  DevStatus* status;
};

// Models of a chunk and head as they are kept for the gradients of the rows: 64 labels at a time (fewer at the end), of these 8 features at a time, so that a
// warp whose threads have a label each, or 8 labels and 8 features, writes whole lines. First element of a unit of 8 features.
constexpr int MODEL_SLICE = 64;
__device__ __forceinline__ int model_labels(int label, int dvp) { return min(MODEL_SLICE, dvp - label / MODEL_SLICE * MODEL_SLICE); }
__device__ __forceinline__ int model_unit(int label, int unit, int dvp, int DK) {
  return label / MODEL_SLICE * MODEL_SLICE * DK + (unit * model_labels(label, dvp) + label % MODEL_SLICE) * 8;
}

// ---- tensor-core helpers ------------------------------------------------------------------------------------------------------------
__device__ __forceinline__ void mma16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldsm(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldsm_t(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void stsm_t(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
// The warp's number as the compiler knows it to be one for all lanes: branches on it need no way back to convergence
__device__ __forceinline__ int warp_index() { return __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0); }
__device__ __forceinline__ uint32_t smem32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ uint32_t pack2(float x, float y) {  // x in the low half
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(y), "f"(x));
  return r;
}
// (x, y) = hi + lo
__device__ __forceinline__ void split2(float x, float y, uint32_t& hi, uint32_t& lo) {
  hi = pack2(x, y);
  lo = pack2(x - __uint_as_float(hi << 16), y - __uint_as_float(hi & 0xffff0000u));
}
// Two neighbouring accumulator tiles [16 x 8] as the A operand of a product over their 16 columns
__device__ __forceinline__ void a_parts(const float (&x)[4], const float (&y)[4], uint32_t (&hi)[4], uint32_t (&lo)[4]) {
  split2(x[0], x[1], hi[0], lo[0]);
  split2(x[2], x[3], hi[1], lo[1]);
  split2(y[0], y[1], hi[2], lo[2]);
  split2(y[2], y[3], hi[3], lo[3]);
}
// Features and queries of a chunk in shared memory: 64 columns to a tile, rows of 128 bytes whose 16-byte units are exchanged as a tensor map's 128-byte swizzle does, unit u of row r
// at u ^ (r & 7). wide_nk and wide_mk: a lane's offset for the 16 x 16 elements at (0, 0), as lane_nk and lane_mk; those at row 16 i and column 16 j are at wide(offset, i, j).
constexpr int WIDE_BYTES = DC * 128;
__device__ __forceinline__ uint32_t wide_unit(int row, int unit) { return row * 128 + ((unit ^ (row & 7)) << 4); }
__device__ __forceinline__ uint32_t wide_nk(int lane) { return wide_unit((lane & 7) + ((lane >> 4) & 1) * 8, (lane >> 3) & 1); }
__device__ __forceinline__ uint32_t wide_mk(int lane) { return wide_unit((lane & 7) + ((lane >> 3) & 1) * 8, (lane >> 4) & 1); }
__device__ __forceinline__ uint32_t wide(uint32_t offset, int i, int j) { return (offset ^ (j % 4 << 5)) + i * 2048 + j / 4 * WIDE_BYTES; }
// Byte offset of a lane's row for 16 x 16 elements at (0, 0) of a tile with `stride` elements a row. lane_nk: B operand of [n][k] (plain), A operand of [k][m]
// (transposed); lane_mk: A operand of [m][k] (plain), B operand of [k][n] (transposed).
__device__ __forceinline__ uint32_t lane_nk(int lane, int stride) { return (((lane & 7) + ((lane >> 4) & 1) * 8) * stride + ((lane >> 3) & 1) * 8) * 2; }
__device__ __forceinline__ uint32_t lane_mk(int lane, int stride) { return (((lane & 7) + ((lane >> 3) & 1) * 8) * stride + ((lane >> 4) & 1) * 8) * 2; }
// The same in a block of a triangle
__device__ __forceinline__ uint32_t tri_nk(int lane) { return tri_unit((lane & 7) + ((lane >> 4) & 1) * 8, (lane >> 3) & 1); }
__device__ __forceinline__ uint32_t tri_mk(int lane) { return tri_unit((lane & 7) + ((lane >> 3) & 1) * 8, (lane >> 4) & 1); }
__device__ __forceinline__ float exp2_fast(float x) {  // 2 ulp, zero below 2^-126
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// ---- chunks of the chains ---------------------------------------------------------------------------------------------------------------
// Offsets checked, chunks counted and listed, chains ordered by length. One block; offsets that are out of order leave no chunks at all.
constexpr int PLAN_THREADS = 1024, PLAN_ORDER = 1024;  // chains that are put in order

__global__ void __launch_bounds__(PLAN_THREADS) delta_plan_kernel(const __grid_constant__ DeltaChunkParams p) {
  __shared__ int warp_sums[32], lengths[PLAN_ORDER];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  kernel_started();
  kernel_inputs_ready();
  int bad = 0;
  for (int c = tid; c < p.n_chains; c += PLAN_THREADS) {
    const long long a = p.shard_off[c], b = p.shard_off[c + 1];
    if (a < 0 || b < a || b > p.n_rows) bad = 1;
  }
  bad = __syncthreads_or(bad);
  if (bad && tid == 0) set_status(p.status, DEV_BOUNDS, 24, 0);
  int carry = 0;
  for (int base = 0; base < p.n_chains; base += PLAN_THREADS) {
    const int c = base + tid;
    int n = 0;
    if (c < p.n_chains && !bad) n = (int)((p.shard_off[c + 1] - p.shard_off[c] + DC - 1) / DC);
    int sum = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += v;
    }
    if (lane == 31) warp_sums[warp] = sum;
    __syncthreads();
    int ws = warp_sums[lane];
    const int w = ws;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, ws, o);
      if (lane >= o) ws += v;
    }
    const int first = carry + __shfl_sync(0xffffffffu, ws - w, warp) + sum - n;
    carry += __shfl_sync(0xffffffffu, ws, 31);
    if (c < p.n_chains) {
      p.chunk_off[c] = first;
      if (c < PLAN_ORDER) lengths[c] = n;
    }
    __syncthreads();
  }
  if (tid == 0) p.chunk_off[p.n_chains] = carry;
  __syncthreads();
  for (int c = warp; c < p.n_chains; c += PLAN_THREADS / 32) {
    const int first = p.chunk_off[c], n = (c + 1 < p.n_chains ? p.chunk_off[c + 1] : carry) - first;
    const long long row0 = p.shard_off[c], rows = p.shard_off[c + 1] - row0;
    for (int i = lane; i < n; i += 32) p.chunks[first + i] = {row0 + (long long)i * DC, (int)min((long long)DC, rows - (long long)i * DC), c};
  }
  for (int c = tid; c < p.n_chains; c += PLAN_THREADS) {
    int rank = c;
    if (p.n_chains <= PLAN_ORDER) {
      rank = 0;
      for (int o = 0; o < p.n_chains; ++o) rank += lengths[o] > lengths[c] || (lengths[o] == lengths[c] && o < c);
    }
    p.order[rank] = c;
  }
}

// Heads of a width that is no multiple of 8, or that do not start on 16 bytes, laid out anew: [n_rows][heads][width rounded up], zeros behind. Up to three tensors in one launch,
// one for each blockIdx.y. Rows outside the chains are left out.
struct DeltaPack {
  struct {
    const __nv_bfloat16* from;
    long long ld;
    __nv_bfloat16* to;
    int heads, width;
  } t[3];
  const int* chunk_off;  // of the plan
  const DeltaChunk* chunks;
  int n_chains;
};
__global__ void __launch_bounds__(256) delta_pack_kernel(const __grid_constant__ DeltaPack p) {
  kernel_started();
  kernel_inputs_ready();
  const auto& t = p.t[blockIdx.y];
  const int per = (t.width + 7) / 8, chunks = p.chunk_off[p.n_chains];
  if (chunks == 0) return;
  const long long units = (long long)t.heads * per, begin = p.chunks[0].row0 * units, end = (p.chunks[chunks - 1].row0 + p.chunks[chunks - 1].len) * units;
  for (long long u = begin + (long long)blockIdx.x * 256 + threadIdx.x; u < end; u += (long long)gridDim.x * 256) {
    const long long head = row_of(u, per), row = row_of(head, t.heads);
    const int col = (int)(u - head * per) * 8, h = (int)(head - row * t.heads);
    const unsigned short* src = (const unsigned short*)t.from + row * t.ld + (long long)h * t.width;
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t a = col + 2 * i < t.width ? src[col + 2 * i] : 0, b = col + 2 * i + 1 < t.width ? src[col + 2 * i + 1] : 0;
      w[i] = a | b << 16;
    }
    *(uint4*)(t.to + head * per * 8 + col) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// 16 bytes to shared memory, zeros where `yes` is false
__device__ __forceinline__ void copy16(uint32_t to, const void* from, bool yes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(yes ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.commit_group;\n\tcp.async.wait_group 0;" ::: "memory"); }

// ---- T, P and the factors of a chunk ----------------------------------------------------------------------------------------------------------
// One block of four warps for each chunk and head of labels, or the heads of labels that share features (`prep_heads` of them) where there are many. K K^T and Q K^T on the tensor cores, a warp with 16 rows and the columns up to them; then T by blocks: the four
// diagonal blocks of 16 by substitution in fp32, a column to a lane, and what is below them by T_10 = -T_11 A_10 T_00, first for blocks of 16, then for
// those of 32. These products are taken transposed, T_10^T = -(T_00^T A_10^T) T_11^T: the accumulator of the first is the A operand of the second, and
// every factor is in two bf16 parts, three products each.
constexpr int PREP_THREADS = 128, PREP_HEADS = PREP_THREADS / 32;  // heads of labels of a block at most: a warp has the gates of each

template <int DK>
struct PrepShape {
  static constexpr int row = DK + 8;
  static constexpr int rows = 2 * DC * row * 2, tris = 6 * DC_TRI, diag = 4 * 16 * 17 * 4;  // K and Q; T, P and A in two parts; diagonal blocks of A
  static constexpr int smem = (rows > tris ? rows : tris) + diag;
};

// acc += a b for a = ah + al, b = bh + bl, 16 x 16 in two tiles
__device__ __forceinline__ void mma_split(float (&c0)[4], float (&c1)[4], const uint32_t (&ah)[4], const uint32_t (&al)[4], const uint32_t (&bh)[4], const uint32_t (&bl)[4]) {
  mma16(c0, ah, bh[0], bh[1]);
  mma16(c1, ah, bh[2], bh[3]);
  mma16(c0, al, bh[0], bh[1]);
  mma16(c1, al, bh[2], bh[3]);
  mma16(c0, ah, bl[0], bl[1]);
  mma16(c1, ah, bl[2], bl[3]);
}
// Two parts of a 16 x 16 accumulator, negated and transposed, to a block of T
__device__ __forceinline__ void put_negative_t(uint32_t at, const float (&c0)[4], const float (&c1)[4]) {
  uint32_t hi[4], lo[4];
  split2(-c0[0], -c0[1], hi[0], lo[0]);
  split2(-c0[2], -c0[3], hi[1], lo[1]);
  split2(-c1[0], -c1[1], hi[2], lo[2]);
  split2(-c1[2], -c1[3], hi[3], lo[3]);
  stsm_t(at, hi[0], hi[1], hi[2], hi[3]);
  stsm_t(at + DC_T_LO, lo[0], lo[1], lo[2], lo[3]);
}

// Answers of rows outside the chains set to zeros: every `blocks`th such row from the `block`th on
__device__ __noinline__ void clear_answers(const DeltaChunkParams& p, int chunks, long long block, long long blocks) {
  const long long lo = chunks > 0 ? p.chunks[0].row0 : 0, hi = chunks > 0 ? p.chunks[chunks - 1].row0 + p.chunks[chunks - 1].len : 0;
  const int width = p.hv * p.dv;
  for (long long i = block; i < lo + p.n_rows - hi; i += blocks) {
    __nv_bfloat16* row = p.out + (i < lo ? i : hi + i - lo) * p.ld_out;
    if (p.vec_out) {
      for (int c = threadIdx.x * 8; c < width; c += PREP_THREADS * 8) *(uint4*)(row + c) = make_uint4(0u, 0u, 0u, 0u);
    } else {
      for (int c = threadIdx.x; c < width; c += PREP_THREADS) ((unsigned short*)row)[c] = 0;
    }
  }
}

template <int DK>
__global__ void __launch_bounds__(PREP_THREADS) delta_prepare_kernel(const __grid_constant__ DeltaChunkParams p) {
  constexpr int ROW = PrepShape<DK>::row;
  constexpr int T_AT = 0, P_AT = DC_P, A_AT = 4 * DC_TRI;  // T and P as they are kept, then A
  extern __shared__ __align__(16) unsigned char prep_smem[];
  __nv_bfloat16* Ks = (__nv_bfloat16*)prep_smem;
  __nv_bfloat16* Qs = Ks + DC * ROW;
  unsigned char* tris = prep_smem;  // over K and Q, once their products are done
  float* diag = (float*)(prep_smem + PrepShape<DK>::smem - PrepShape<DK>::diag);
  __shared__ float bhis[PREP_HEADS][DC], blos[PREP_HEADS][DC], steps[PREP_HEADS][DC];
  const int tid = threadIdx.x, warp = warp_index(), lane = tid & 31, g = lane >> 2, t = lane & 3;
  kernel_started();
  kernel_inputs_ready();
  const int groups = p.hv / p.prep_heads, chunk = blockIdx.x / groups, h0 = blockIdx.x % groups * p.prep_heads, kh = h0 / (p.hv / p.hk);
  const int chunks = p.chunk_off[p.n_chains];
  if (chunk >= chunks) {
    if (p.new_out) clear_answers(p, chunks, (long long)blockIdx.x - (long long)chunks * groups, (long long)gridDim.x - (long long)chunks * groups);
    return;
  }
  const DeltaChunk at = p.chunks[chunk];

  for (int u = tid; u < DC * (DK / 8); u += PREP_THREADS) {
    const int row = u / (DK / 8), col = u % (DK / 8) * 8;
    const bool there = row < at.len && col < p.k.width;
    const long long i = there ? at.row0 + row : 0;
    const int c = there ? kh * p.k.width + col : 0;
    copy16(smem32(Ks + row * ROW + col), p.k.p + i * p.k.ld + c, there);
    copy16(smem32(Qs + row * ROW + col), p.q.p + i * p.q.ld + c, there);
  }
  if (warp < p.prep_heads) {  // b of a head by a scan over a warp's lanes, two rows a lane, in 64 bits
    const int h = h0 + warp;
    double d[2];
    float beta[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int row = 2 * lane + i;
      const float gg = row < at.len ? __bfloat162float(p.g[(at.row0 + row) * p.ld_g + h]) : 0.0f;
      d[i] = gg < DELTA_MIN_G ? DELTA_MIN_G : gg;
      beta[i] = row < at.len ? __bfloat162float(p.beta[(at.row0 + row) * p.ld_beta + h]) : 0.0f;
    }
    double sum = d[0] + d[1];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const double v = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += v;
    }
    const double last = __shfl_sync(0xffffffffu, sum, 31);
    DeltaFactors* f = (DeltaFactors*)(p.blocks + ((long long)chunk * p.hv + h) * DC_BLOCK + DC_FACTORS);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int row = 2 * lane + i;
      const double b = i ? sum : sum - d[1], b2 = b * 1.4426950408889634;
      const float hi = (float)b2, lo = (float)(b2 - (double)hi);
      bhis[warp][row] = hi;
      blos[warp][row] = lo;
      steps[warp][row] = beta[i];
      f->c[row] = expf((float)b);
      f->r[row] = expf((float)(last - b));
      f->beta[row] = beta[i];
      f->hi[row] = hi;
      f->lo[row] = lo;
    }
    if (lane == 0) f->last = expf((float)last);
  }
  copies_done();
  __syncthreads();

  float kk[4][2][4], qk[4][2][4];
#pragma unroll
  for (int n = 0; n < 4; ++n)
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) kk[n][i][e] = qk[n][i][e] = 0.0f;
  const uint32_t ka = smem32(Ks) + lane_mk(lane, ROW) + warp * 16 * ROW * 2, qa = smem32(Qs) + lane_mk(lane, ROW) + warp * 16 * ROW * 2, kb = smem32(Ks) + lane_nk(lane, ROW);
#pragma unroll
  for (int x = 0; x < DK / 16; ++x) {
    uint32_t ak[4], aq[4], b[4];
    ldsm(ak, ka + x * 32);
    ldsm(aq, qa + x * 32);
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      if (n > warp) break;
      ldsm(b, kb + n * 16 * ROW * 2 + x * 32);
      mma16(kk[n][0], ak, b[0], b[1]);
      mma16(kk[n][1], ak, b[2], b[3]);
      mma16(qk[n][0], aq, b[0], b[1]);
      mma16(qk[n][1], aq, b[2], b[3]);
    }
  }
  for (int h = h0; h < h0 + p.prep_heads; ++h) {
    unsigned char* block = p.blocks + ((long long)chunk * p.hv + h) * DC_BLOCK;
    const float *bhi = bhis[h - h0], *blo = blos[h - h0], *betas = steps[h - h0];
    __syncthreads();  // also: K and Q, or the triangles of the head before, have been read
    const float hi0 = bhi[warp * 16 + g], lo0 = blo[warp * 16 + g], hi1 = bhi[warp * 16 + g + 8], lo1 = blo[warp * 16 + g + 8], be0 = betas[warp * 16 + g], be1 = betas[warp * 16 + g + 8];
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      if (n > warp) break;
      unsigned char* to = tris + tri_at(warp, n);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int col = n * 16 + i * 8 + 2 * t;
        const float2 ch = *(const float2*)(bhi + col), cl = *(const float2*)(blo + col);
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
          const int row = warp * 16 + g + 4 * e;
          const float hi = e ? hi1 : hi0, lo = e ? lo1 : lo0, be = e ? be1 : be0;
          float d0 = exp2_fast((hi - ch.x) + (lo - cl.x)), d1 = exp2_fast((hi - ch.y) + (lo - cl.y));
          if (n == warp) {  // selected, not multiplied: above the diagonal the exponent is of the other sign
            d0 = col <= row ? d0 : 0.0f;
            d1 = col + 1 <= row ? d1 : 0.0f;
          }
          const int unit = tri_unit(g + 4 * e, i) + 4 * t;
          uint32_t h2, l2;
          split2(p.scale * d0 * qk[n][i][e], p.scale * d1 * qk[n][i][e + 1], h2, l2);
          *(uint32_t*)(to + P_AT + unit) = h2;
          *(uint32_t*)(to + P_AT + DC_TRI + unit) = l2;
          const float k0 = d0 * kk[n][i][e], k1 = d1 * kk[n][i][e + 1], a0 = be * k0, a1 = be * k1;
          if (p.gram) *(uint32_t*)(p.gram + ((long long)chunk * p.hv + h) * DC_TRI + tri_at(warp, n) + unit) = pack2(k0, k1);
          if (n == warp) {
            float* a = diag + (warp * 16 + g + 4 * e) * 17 + i * 8 + 2 * t;
            a[0] = a0;  // the substitution reads below the diagonal only
            a[1] = a1;
          } else {
            split2(a0, a1, h2, l2);
            *(uint32_t*)(to + A_AT + unit) = h2;
            *(uint32_t*)(to + A_AT + DC_TRI + unit) = l2;
          }
        }
      }
    }
    __syncwarp();
    if (lane < 16) {  // column `lane` of the warp's diagonal block
      const float* a = diag + warp * 16 * 17;
      unsigned char* to = tris + T_AT + tri_at(warp, warp);
      float x[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        float s = i == lane ? 1.0f : 0.0f;
#pragma unroll
        for (int m = 0; m < i; ++m) s = fmaf(-a[i * 17 + m], x[m], s);
        x[i] = s;
        const __nv_bfloat16 hi = __float2bfloat16_rn(s);
        const int unit = tri_unit(i, lane >> 3) + (lane & 7) * 2;
        *(__nv_bfloat16*)(to + unit) = hi;
        *(__nv_bfloat16*)(to + DC_T_LO + unit) = __float2bfloat16_rn(s - __bfloat162float(hi));
      }
    }
    __syncthreads();
    const uint32_t nk = smem32(tris) + tri_nk(lane);
    if (warp & 1) {  // blocks (1, 0) and (3, 2)
      const int o = warp - 1, d0 = tri_at(o, o), d1 = tri_at(warp, warp), od = tri_at(warp, o);
      float x[2][4] = {}, y[2][4] = {};
      uint32_t ah[4], al[4], bh[4], bl[4];
      ldsm_t(ah, nk + T_AT + d0);
      ldsm_t(al, nk + T_AT + DC_T_LO + d0);
      ldsm(bh, nk + A_AT + od);
      ldsm(bl, nk + A_AT + DC_TRI + od);
      mma_split(x[0], x[1], ah, al, bh, bl);
      a_parts(x[0], x[1], ah, al);
      ldsm(bh, nk + T_AT + d1);
      ldsm(bl, nk + T_AT + DC_T_LO + d1);
      mma_split(y[0], y[1], ah, al, bh, bl);
      put_negative_t(nk + T_AT + od, y[0], y[1]);
    }
    __syncthreads();
    {  // the block of 32: columns 16 j of it, rows 32 + 16 i
      const int j = warp & 1, i = warp >> 1;
      float x[4][4] = {}, y[2][4] = {};
      uint32_t ah[4], al[4], bh[4], bl[4];
#pragma unroll
      for (int m = 0; m < 2; ++m) {  // X^T = T_00^T A_10^T over rows of T_00 from its diagonal on
        if (m < j) continue;
        const int tt = tri_at(m, j);
        ldsm_t(ah, nk + T_AT + tt);
        ldsm_t(al, nk + T_AT + DC_T_LO + tt);
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          const int aa = tri_at(2 + n, m);
          ldsm(bh, nk + A_AT + aa);
          ldsm(bl, nk + A_AT + DC_TRI + aa);
          mma_split(x[2 * n], x[2 * n + 1], ah, al, bh, bl);
        }
      }
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        if (m > i) continue;
        const int tt = tri_at(2 + i, 2 + m);
        a_parts(x[2 * m], x[2 * m + 1], ah, al);
        ldsm(bh, nk + T_AT + tt);
        ldsm(bl, nk + T_AT + DC_T_LO + tt);
        mma_split(y[0], y[1], ah, al, bh, bl);
      }
      put_negative_t(nk + T_AT + tri_at(2 + i, j), y[0], y[1]);
    }
    __syncthreads();
    for (int u = tid; u < 4 * DC_TRI / 16; u += PREP_THREADS) *(uint4*)(block + u * 16) = *(const uint4*)(tris + u * 16);
  }
}

// ---- the walk over a chain's chunks ---------------------------------------------------------------------------------------------------------------
// A block has a chain, a head and 16 NW labels of it: NW warps as described above, beside four that only copy. (Backward there may be eight, and each brings its share of the next
// chunk while it works on this one, so that a scheduler's registers go to the two warps that multiply: a ninth warp that only copies would leave them 168 each.) Three stages where they fit: a warp may be a chunk ahead of the slowest.
template <int DK, int NW>
struct ChainShape {
  static constexpr int vrow = 16 * NW + 8;  // elements
  static constexpr int q_at = DK / 64 * WIDE_BYTES, v_at = 2 * q_at, block_at = v_at + DC * vrow * 2, stage = (block_at + DC_BLOCK + 1023) / 1024 * 1024;
  static constexpr int stages = 3 * stage <= 225 * 1024 ? 3 : 2;
  static constexpr int smem = stages * stage + 1024;  // tiles start on 1024 bytes
  static constexpr int copiers = NW < 8 ? 4 : 0, threads = 32 * (NW + copiers);
};

// A warp's share of 64 rows of a tile, `UNITS` units of 16 bytes a row, unit u of row r at place(r, u); zeros behind the chunk's end and from column `width` on. (A bulk copy for each row
// takes 64 cycles to issue, whatever its size: 0.8 ms for 16384 chunks of 128 features and labels.)
template <int UNITS, typename Place>
__device__ __forceinline__ void copy_rows(Place place, const __nv_bfloat16* from, long long ld, int len, int width, int warp, int warps, int lane) {
  constexpr int per = 32 / UNITS;  // rows at a time
  static_assert(UNITS <= 32 && 32 % UNITS == 0, "a warp has whole rows");
  const int unit = lane % UNITS;
#pragma unroll 4
  for (int r = warp * per + lane / UNITS; r < DC; r += warps * per) {
    const bool there = unit * 8 < width && r < len;
    copy16(place(r, unit), from + (there ? r * ld + unit * 8 : 0), there);
  }
}
// 64 rows and 64 columns from (x, y) of the rows that a tensor map describes
__device__ __forceinline__ void tma_tile(uint32_t to, const CUtensorMap* map, int x, int y, unsigned long long* bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(to), "l"(map), "r"(x), "r"(y), "r"(smem32(bar)) : "memory");
}
__device__ __forceinline__ void bulk_block(uint32_t to, const void* from, uint32_t bytes, unsigned long long* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(to), "l"(from), "r"(bytes), "r"(smem32(bar)) : "memory");
}

// Rows of a chain, and of its chunk i. (Looked up in the list of chunks by each warp, they would be waited for twice a chunk: 1400 of 12000 cycles.)
struct DeltaSpan {
  long long row0, rows;
  __device__ __forceinline__ int len(int i) const { return (int)min((long long)DC, rows - (long long)i * DC); }
};
// From the list of chunks, which was checked: the offsets may have changed since a run that a gradient follows
__device__ __forceinline__ DeltaSpan span_of(const DeltaChunkParams& p, int first, int n) {
  if (n == 0) return {0, 0};
  return {p.chunks[first].row0, (long long)(n - 1) * DC + p.chunks[first + n - 1].len};
}
// Tensor maps of the rows of all heads of features and queries: whole chunks come by them where a head has all the features of its tiles. (All of a chunk by 16-byte copies of the warps
// cost 200 of 850 us for 65536 rows of 16 heads: they share the way to shared memory with the operands.)
struct DeltaMaps {
  CUtensorMap k, q;
};
// The barriers of a stage: `rows` takes an arrival of every thread that brings, `bulk` one and the bytes of what one thread asks for
struct ChunkBarriers {
  unsigned long long rows, bulk, empty;
};
// A warp's share of a chunk: features, queries, labels (or their gradients) and the block of the first kernel.
template <int DK, int NW>
__device__ __forceinline__ void bring_chunk(const DeltaChunkParams& p, const DeltaMaps& maps, const DeltaHeads& labels, uint32_t st, int chunk, const DeltaSpan& span, int i, int h, int kh, int col0,
                                            int warp, int warps, int lane, ChunkBarriers* bars) {
  using Shape = ChainShape<DK, NW>;
  const long long row0 = span.row0 + (long long)i * DC;
  const int len = span.len(i);
  const bool whole = p.maps && len == DC;
  if (warp == 0 && elect_one()) {
    mbar_arrive_expect_tx(&bars->bulk, DC_BLOCK + (whole ? 2 * Shape::q_at : 0));
    if (whole)
#pragma unroll
      for (int j = 0; j < DK / 64; ++j) {
        tma_tile(st + j * WIDE_BYTES, &maps.k, kh * DK + j * 64, (int)row0, &bars->bulk);
        tma_tile(st + Shape::q_at + j * WIDE_BYTES, &maps.q, kh * DK + j * 64, (int)row0, &bars->bulk);
      }
    bulk_block(st + Shape::block_at, p.blocks + ((long long)chunk * p.hv + h) * DC_BLOCK, DC_BLOCK, &bars->bulk);
  }
  if (!whole) {
    auto place = [&](int r, int u) { return st + wide_unit(r, u & 7) + u / 8 * WIDE_BYTES; };
    copy_rows<DK / 8>(place, p.k.p + row0 * p.k.ld + kh * p.k.width, p.k.ld, len, p.k.width, warp, warps, lane);
    copy_rows<DK / 8>([&](int r, int u) { return place(r, u) + Shape::q_at; }, p.q.p + row0 * p.q.ld + kh * p.q.width, p.q.ld, len, p.q.width, warp, warps, lane);
  }
  copy_rows<2 * NW>([&](int r, int u) { return st + Shape::v_at + (r * Shape::vrow + u * 8) * 2; }, labels.p + row0 * labels.ld + h * labels.width + col0, labels.ld, len, labels.width - col0, warp,
                    warps, lane);
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem32(&bars->rows)) : "memory");
}
// What the warp that asks for bulk copies does when it gives up: chunks `from` to `to` - 1 are in flight
template <int STAGES>
__device__ __forceinline__ void bulk_done(ChunkBarriers* bars, int from, int to) {
  for (int i = from; i < to; ++i) mbar_wait_bounded(&bars[i % STAGES].bulk, (i / STAGES) & 1, DRAIN_LIMIT);
}
// A copying warp's work: its share of all n chunks, the last first where `back`
template <int DK, int NW>
__device__ __forceinline__ void bring_chunks(const DeltaChunkParams& p, const DeltaMaps& maps, const DeltaHeads& labels, uint32_t smem, int first, bool back, int n, const DeltaSpan& span, int h,
                                             int kh, int col0, int warp, int warps, int lane, ChunkBarriers* bars) {
  using Shape = ChainShape<DK, NW>;
  int brought = 0;
  for (int i = 0; i < n; ++i) {
    const int s = i % Shape::stages;
    if (i >= Shape::stages && !__all_sync(0xffffffffu, mbar_wait_bounded(&bars[s].empty, (i / Shape::stages - 1) & 1, p.spin_limit))) {
      if (lane == 0) set_status(p.status, DEV_TIMEOUT, 27, i);
      break;
    }
    if (i == p.drop) break;  // a test hook: this chunk and those behind it are never brought
    const int j = back ? n - 1 - i : i;
    bring_chunk<DK, NW>(p, maps, labels, smem + s * Shape::stage, first + j, span, j, h, kh, col0, warp, warps, lane, &bars[s]);
    brought = i + 1;
  }
  copies_done();
  if (warp == 0) bulk_done<Shape::stages>(bars, max(0, brought - Shape::stages), brought);  // nothing is in flight when the block ends
}
__device__ __forceinline__ void arrive(unsigned long long* bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem32(bar)) : "memory"); }

// 16 labels of 64 rows from registers (labels x rows, two rows in a word) to memory, by way of the warp's own columns of the tile that its labels came in
template <bool VEC>
__device__ __forceinline__ void put_labels(const float (&x)[8][4], unsigned char* tile, int stride, int lane, __nv_bfloat16* to, long long ld, int rows, int cols) {
  __syncwarp();
  const uint32_t at = smem32(tile) + lane_nk(lane, stride / 2);
#pragma unroll
  for (int n = 0; n < 4; ++n) stsm_t(at + n * 16 * stride, pack2(x[2 * n][0], x[2 * n][1]), pack2(x[2 * n][2], x[2 * n][3]), pack2(x[2 * n + 1][0], x[2 * n + 1][1]), pack2(x[2 * n + 1][2], x[2 * n + 1][3]));
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int u = i * 32 + lane, row = u / 2, col = u % 2 * 8;
    if (row >= rows || col >= cols) continue;
    const uint4 v = *(const uint4*)(tile + row * stride + col * 2);
    __nv_bfloat16* o = to + row * ld + col;
    if (VEC) {
      *(uint4*)o = v;
    } else {
      const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (col + e < cols) ((unsigned short*)o)[e] = (unsigned short)(w[e / 2] >> (16 * (e % 2)));
    }
  }
}

template <int DK, int NW, bool SAVE>
__global__ void __launch_bounds__(ChainShape<DK, NW>::threads) delta_chain_kernel(const __grid_constant__ DeltaChunkParams p, const __grid_constant__ DeltaMaps maps) {
  using Shape = ChainShape<DK, NW>;
  constexpr int VROW = Shape::vrow * 2, STAGES = Shape::stages;  // bytes
  static_assert(Shape::copiers > 0, "chunks are brought by warps of their own");
  extern __shared__ unsigned char chain_smem[];
  __shared__ ChunkBarriers bars[STAGES];
  const int tid = threadIdx.x, warp = warp_index(), lane = tid & 31, g = lane >> 2, t = lane & 3;
  unsigned char* const ring = chain_smem + (-smem32(chain_smem) & 1023u);
  kernel_inputs_ready();
  const int slice = blockIdx.x % p.slices, h = blockIdx.x / p.slices % p.hv, chain = p.order[blockIdx.x / p.slices / p.hv], kh = h / (p.hv / p.hk);
  const int col0 = slice * 16 * NW, warps = min(NW, (p.dvp - col0) / 16);  // warps with labels
  const int first = p.chunk_off[chain], n = p.chunk_off[chain + 1] - first;
  const DeltaSpan span = span_of(p, first, n);
  if (tid == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(&bars[s].rows, 32 * Shape::copiers);
      mbar_init(&bars[s].bulk, 1);
      mbar_init(&bars[s].empty, warps);
    }
    mbar_fence_init();
  }
  __syncthreads();
  if (warp >= NW) {
    bring_chunks<DK, NW>(p, maps, p.v, smem32(ring), first, false, n, span, h, kh, col0, warp - NW, Shape::copiers, lane, bars);
    return;
  }
  if (warp >= warps) return;
  // S^T: labels g and g + 8 of the warp's 16, features 8 n + 2 t and the next
  float S[DK / 8][4];
  const int label = col0 + warp * 16 + g;
  const long long model = ((long long)chain * p.hv + h) * p.dv;
#pragma unroll
  for (int x = 0; x < DK / 8; ++x)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int f = 8 * x + 2 * t + (e & 1), l = label + (e >> 1) * 8;
      S[x][e] = p.W0 && f < p.dk && l < p.dv ? p.W0[(model + l) * p.dk + f] : 0.0f;
    }

  for (int i = 0; i < n; ++i) {
    const int s = i % STAGES;
    const bool there = __all_sync(0xffffffffu, mbar_wait_bounded(&bars[s].bulk, (i / STAGES) & 1, p.spin_limit));
    if (!there || !__all_sync(0xffffffffu, mbar_wait_bounded(&bars[s].rows, (i / STAGES) & 1, p.spin_limit))) {
      if (lane == 0) set_status(p.status, DEV_TIMEOUT, 25, i);
      return;
    }
    unsigned char* st = ring + s * Shape::stage;
    const unsigned char* block = st + Shape::block_at;
    const DeltaFactors* f = (const DeltaFactors*)(block + DC_FACTORS);
    const long long which = (long long)(first + i) * p.hv + h;
    const uint32_t k_at = smem32(st), q_at = k_at + Shape::q_at, nk = wide_nk(lane), mk = wide_mk(lane);
    const uint32_t t_nk = smem32(block) + tri_nk(lane), v_nk = smem32(st + Shape::v_at) + warp * 32 + lane_nk(lane, Shape::vrow);

    // S^T K^T
    float R[8][4];
#pragma unroll
    for (int x = 0; x < 8; ++x)
#pragma unroll
      for (int e = 0; e < 4; ++e) R[x][e] = 0.0f;
#pragma unroll
    for (int x = 0; x < DK / 16; ++x) {
      uint32_t hi[4], lo[4], b[4][4];
      a_parts(S[2 * x], S[2 * x + 1], hi, lo);
      if (SAVE) {  // models before the chunk, one bf16 part
        uint32_t* to = (uint32_t*)(p.starts + which * p.dvp * DK + model_unit(label, 2 * x, p.dvp, DK) + 2 * t);
        to[0] = hi[0];
        to[32] = hi[1];
        to[4 * model_labels(label, p.dvp)] = hi[2];
        to[4 * model_labels(label, p.dvp) + 32] = hi[3];
      }
#pragma unroll
      for (int y = 0; y < 4; ++y) ldsm(b[y], k_at + wide(nk, y, x));
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        mma16(R[2 * y], hi, b[y][0], b[y][1]);
        mma16(R[2 * y + 1], hi, b[y][2], b[y][3]);
      }
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        mma16(R[2 * y], lo, b[y][0], b[y][1]);
        mma16(R[2 * y + 1], lo, b[y][2], b[y][3]);
      }
    }
    // R^T = beta (V^T - c S^T K^T)
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      uint32_t v[4];
      ldsm_t(v, v_nk + y * 16 * VROW);
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        const int x = 2 * y + z, at = 8 * x + 2 * t;
        const float2 c = *(const float2*)(f->c + at), be = *(const float2*)(f->beta + at);
        const uint32_t v0 = v[2 * z], v1 = v[2 * z + 1];
        R[x][0] = be.x * (__uint_as_float(v0 << 16) - c.x * R[x][0]);
        R[x][1] = be.y * (__uint_as_float(v0 & 0xffff0000u) - c.y * R[x][1]);
        R[x][2] = be.x * (__uint_as_float(v1 << 16) - c.x * R[x][2]);
        R[x][3] = be.y * (__uint_as_float(v1 & 0xffff0000u) - c.y * R[x][3]);
      }
    }
    // U^T = R^T T^T, rows of T from the block of 16 columns on: chains of dependent products, between them S^T Q^T, which waits for nothing
    float U[8][4], O[8][4];
#pragma unroll
    for (int x = 0; x < 8; ++x)
#pragma unroll
      for (int e = 0; e < 4; ++e) U[x][e] = O[x][e] = 0.0f;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      uint32_t hi[4], lo[4], bh[4], bl[4];
      a_parts(R[2 * x], R[2 * x + 1], hi, lo);
#pragma unroll
      for (int y = x; y < 4; ++y) {
        ldsm(bh, t_nk + tri_at(y, x));
        ldsm(bl, t_nk + DC_T_LO + tri_at(y, x));
        mma_split(U[2 * y], U[2 * y + 1], hi, lo, bh, bl);
      }
#pragma unroll
      for (int z = x * DK / 64; z < (x + 1) * DK / 64; ++z) {
        const uint32_t a[4] = {pack2(S[2 * z][0], S[2 * z][1]), pack2(S[2 * z][2], S[2 * z][3]), pack2(S[2 * z + 1][0], S[2 * z + 1][1]), pack2(S[2 * z + 1][2], S[2 * z + 1][3])};
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          ldsm(bh, q_at + wide(nk, y, z));
          mma16(O[2 * y], a, bh[0], bh[1]);
          mma16(O[2 * y + 1], a, bh[2], bh[3]);
        }
      }
    }
    if (SAVE) put_labels<true>(U, st + Shape::v_at + warp * 32, VROW, lane, p.steps + which * DC * p.dvp + col0 + warp * 16, p.dvp, DC, 16);
    // O^T = scale c S^T Q^T + U^T P^T, and S^T <- e^{b_C} S^T + (r U)^T K
    const uint64_t last = pair_of(__float_as_uint(f->last), __float_as_uint(f->last));
#pragma unroll
    for (int x = 0; x < DK / 8; ++x)
#pragma unroll
      for (int e = 0; e < 4; e += 2) {
        const float2 v = halves(mul2(last, pair_of(__float_as_uint(S[x][e]), __float_as_uint(S[x][e + 1]))));
        S[x][e] = v.x, S[x][e + 1] = v.y;
      }
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      const float2 c = *(const float2*)(f->c + 8 * x + 2 * t);
      const float cx = p.scale * c.x, cy = p.scale * c.y;
      O[x][0] *= cx, O[x][1] *= cy, O[x][2] *= cx, O[x][3] *= cy;
    }
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      uint32_t hi[4], lo[4], bh[4], bl[4];
      a_parts(U[2 * x], U[2 * x + 1], hi, lo);
#pragma unroll
      for (int y = x; y < 4; ++y) {
        ldsm(bh, t_nk + DC_P + tri_at(y, x));
        ldsm(bl, t_nk + DC_P_LO + tri_at(y, x));
        mma_split(O[2 * y], O[2 * y + 1], hi, lo, bh, bl);
      }
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        const float2 r = *(const float2*)(f->r + 16 * x + 8 * z + 2 * t);
        U[2 * x + z][0] *= r.x, U[2 * x + z][1] *= r.y, U[2 * x + z][2] *= r.x, U[2 * x + z][3] *= r.y;
      }
      a_parts(U[2 * x], U[2 * x + 1], hi, lo);
#pragma unroll
      for (int y = 0; y < DK / 16; ++y) {
        ldsm_t(bh, k_at + wide(mk, x, y));
        mma16(S[2 * y], hi, bh[0], bh[1]);
        mma16(S[2 * y + 1], hi, bh[2], bh[3]);
        mma16(S[2 * y], lo, bh[0], bh[1]);
        mma16(S[2 * y + 1], lo, bh[2], bh[3]);
      }
    }
    __nv_bfloat16* out = p.out + (span.row0 + (long long)i * DC) * p.ld_out + h * p.dv + col0 + warp * 16;
    const int cols = min(16, p.dv - col0 - warp * 16);
    if (p.vec_out) put_labels<true>(O, st + Shape::v_at + warp * 32, VROW, lane, out, p.ld_out, span.len(i), cols);
    else put_labels<false>(O, st + Shape::v_at + warp * 32, VROW, lane, out, p.ld_out, span.len(i), cols);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // a stage's rows may have come by copies of threads, and come by the tensor map next
    __syncwarp();
    if (lane == 0) arrive(&bars[s].empty);
  }
  kernel_started();
  if (p.W)
#pragma unroll
    for (int x = 0; x < DK / 8; ++x)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int f = 8 * x + 2 * t + (e & 1), l = label + (e >> 1) * 8;
        if (f < p.dk && l < p.dv) p.W[(model + l) * p.dk + f] = S[x][e];
      }
}

}  // namespace wpsgd
