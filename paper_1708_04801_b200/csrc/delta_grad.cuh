// Gradients of the chains whose labels are vectors (see delta_chunk.cuh for the forward form and its symbols, include/wpsgd.h for the calls).
//
// With O' = dL/dO, G = dL/dS' and everything per chunk and head:
//   dU = P^T O' + r K G,   dR = T^T dU,   dV = beta dR,
//   G before the chunk = e^{b_C} G + Q^T (scale c O') - K^T (beta c dR).
// That is a walk like the forward one, from a chain's last chunk to its first: G^T [16 labels x dk] in a warp's registers, dU and dR
// from product to product. It leaves dR and G of every chunk, and a third kernel takes all chunks at once:
//   F = scale D o tril(O' U^T),  E = -D o stril(dR U^T),
//   dQ = scale c O' S^T + F K,   x = E K - c dR S^T,   back = F^T Q + (beta E)^T K + r U G^T,   dK = beta x + back,
//   dbeta_i = dR_i.v_i + x_i.k_i.
// dg_i is what passes the decay of row i: with H_ab = (O' U^T)_ab P_ab - (dR U^T)_ab A_ab, what the step of row b gives the answer and the step of row a,
//   dg_i = sum_{a >= i > b} H_ab + sum_{a >= i} (scale c_a O'_a S^T q_a - beta_a c_a dR_a S^T k_a) + sum_{b < i} r_b U_b G^T k_b + e^{b_C} S.G,
// the first sum from the end of the chunk on by the row sums of H less its column sums: the same numbers on both sides, so that what does not pass row i cancels.
//
// Rounding: G, P, dU, scale c O' and beta c dR in two bf16 parts in the walk's products; S, U, G, dR, F, E and beta E are rounded to bf16 once where the third kernel multiplies them, and
// D o K K^T (which dg and dbeta take, by A) as it is kept: second parts would cost the third kernel, whose time goes with what it brings, a fifth more memory and twice the products. Gradients
// leave as bf16: those of the labels are off by that rounding alone (1.7e-3 of their norm), the others by 2.4e-3 to 3e-3.
//
// Bounds, 32768 rows in 16 chains, 8 heads of features and 16 of labels, 128 x 128: the walk 436 us, by mma.sync as the forward one of few labels; the third kernel
// 620 us, of which its copies alone would take 220 and the tensor pipe is active for 200: the steps between the products (F and E, sums, the way out) wait for each
// other at barriers, and 128 registers hold no second piece of work. Tried and slower, 3216 chunks and heads of 128 x 128 (241 us): two blocks of 8 warps an SM with half of
// the columns each, F and E formed twice (321); 8 warps with 255 registers (275, when 16 took 268); the sums over heads that share features in shared memory instead of
// a ring of whole slices (267).
#pragma once

#include "delta_chunk.cuh"

namespace wpsgd {

struct DeltaGradParams {
  DeltaChunkParams f;
  __nv_bfloat16* ends;   // [chunks][hv][dvp x DK]: G behind the chunk, as starts
  __nv_bfloat16* drs;    // [chunks][hv][DC][dvp]: dR
  float* totals;         // [blocks][2][DC][DK]: sums over the heads of labels that share features
  const float* dW;
  float* dW0;
  __nv_bfloat16 *dq, *dk, *dv, *dg, *dbeta;
  int vec_dv, vec_dk;  // rows of dv take 16 bytes at a time, rows of dq and dk 4
};

template <int DK, int NW>
__global__ void __launch_bounds__(ChainShape<DK, NW>::threads) delta_back_kernel(const __grid_constant__ DeltaGradParams gp, const __grid_constant__ DeltaMaps maps) {
  const DeltaChunkParams& p = gp.f;
  using Shape = ChainShape<DK, NW>;
  constexpr int VROW = Shape::vrow * 2, STAGES = Shape::stages;  // bytes
  constexpr bool COPIERS = Shape::copiers > 0;
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
      mbar_init(&bars[s].rows, 32 * (COPIERS ? Shape::copiers : warps));
      mbar_init(&bars[s].bulk, 1);
      mbar_init(&bars[s].empty, warps);
    }
    mbar_fence_init();
  }
  __syncthreads();
  if (COPIERS && warp >= NW) {
    bring_chunks<DK, NW>(p, maps, p.dout, smem32(ring), first, true, n, span, h, kh, col0, warp - NW, Shape::copiers, lane, bars);
    return;
  }
  if (warp >= warps) return;
  int brought = 0;
  if (!COPIERS && n > 0 && p.drop != 0) {
    bring_chunk<DK, NW>(p, maps, p.dout, smem32(ring), first + n - 1, span, n - 1, h, kh, col0, warp, warps, lane, &bars[0]);
    brought = 1;
  }

  float G[DK / 8][4];  // G^T, as S^T in the forward walk
  const int label = col0 + warp * 16 + g;
  const long long model = ((long long)chain * p.hv + h) * p.dv;
#pragma unroll
  for (int x = 0; x < DK / 8; ++x)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int f = 8 * x + 2 * t + (e & 1), l = label + (e >> 1) * 8;
      G[x][e] = gp.dW && f < p.dk && l < p.dv ? gp.dW[(model + l) * p.dk + f] : 0.0f;
    }

  for (int i = 0; i < n; ++i) {
    const int s = i % STAGES, s1 = (i + 1) % STAGES;
    bool ok = true;
    if (!COPIERS && i + 1 < n) {  // the next chunk, once all have left the one that was there; p.drop (a test hook): from which on none is brought
      if (i + 1 >= STAGES) ok = __all_sync(0xffffffffu, mbar_wait_bounded(&bars[s1].empty, ((i + 1) / STAGES - 1) & 1, p.spin_limit));
      if (ok && (p.drop < 0 || i + 1 < p.drop)) {
        bring_chunk<DK, NW>(p, maps, p.dout, smem32(ring) + s1 * Shape::stage, first + n - 2 - i, span, n - 2 - i, h, kh, col0, warp, warps, lane, &bars[s1]);
        brought = i + 2;
      }
    }
    ok = ok && __all_sync(0xffffffffu, mbar_wait_bounded(&bars[s].bulk, (i / STAGES) & 1, p.spin_limit));
    if (!ok || !__all_sync(0xffffffffu, mbar_wait_bounded(&bars[s].rows, (i / STAGES) & 1, p.spin_limit))) {
      if (lane == 0) set_status(p.status, DEV_TIMEOUT, 26, i);
      copies_done();  // nothing of this warp's is in flight when it leaves
      if (!COPIERS && warp == 0) bulk_done<STAGES>(bars, max(0, brought - STAGES), brought);
      return;
    }
    unsigned char* st = ring + s * Shape::stage;
    const unsigned char* block = st + Shape::block_at;
    const DeltaFactors* f = (const DeltaFactors*)(block + DC_FACTORS);
    const int chunk = first + n - 1 - i;
    const long long which = (long long)chunk * p.hv + h;
    const uint32_t k_at = smem32(st), q_at = k_at + Shape::q_at, nk = wide_nk(lane), mk = wide_mk(lane);
    const uint32_t t_mk = smem32(block) + tri_mk(lane), v_nk = smem32(st + Shape::v_at) + warp * 32 + lane_nk(lane, Shape::vrow);

    // dU^T = r G^T K^T + O'^T P
    float M[8][4];
#pragma unroll
    for (int x = 0; x < 8; ++x)
#pragma unroll
      for (int e = 0; e < 4; ++e) M[x][e] = 0.0f;
#pragma unroll
    for (int x = 0; x < DK / 16; ++x) {
      uint32_t hi[4], lo[4], b[4][4];
      a_parts(G[2 * x], G[2 * x + 1], hi, lo);
      uint32_t* to = (uint32_t*)(gp.ends + which * p.dvp * DK + model_unit(label, 2 * x, p.dvp, DK) + 2 * t);
      to[0] = hi[0];
      to[32] = hi[1];
      to[4 * model_labels(label, p.dvp)] = hi[2];
      to[4 * model_labels(label, p.dvp) + 32] = hi[3];
      if (NW == 8 && i == 0 && !gp.dW) continue;  // a gradient of zeros: nothing to multiply
#pragma unroll
      for (int y = 0; y < 4; ++y) ldsm(b[y], k_at + wide(nk, y, x));
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        mma16(M[2 * y], hi, b[y][0], b[y][1]);
        mma16(M[2 * y + 1], hi, b[y][2], b[y][3]);
      }
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        mma16(M[2 * y], lo, b[y][0], b[y][1]);
        mma16(M[2 * y + 1], lo, b[y][2], b[y][3]);
      }
    }
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      const float2 r = *(const float2*)(f->r + 8 * x + 2 * t);
      M[x][0] *= r.x, M[x][1] *= r.y, M[x][2] *= r.x, M[x][3] *= r.y;
    }
    const uint64_t last = pair_of(__float_as_uint(f->last), __float_as_uint(f->last));
#pragma unroll
    for (int x = 0; x < DK / 8; ++x)
#pragma unroll
      for (int e = 0; e < 4; e += 2) {
        const float2 v = halves(mul2(last, pair_of(__float_as_uint(G[x][e]), __float_as_uint(G[x][e + 1]))));
        G[x][e] = v.x, G[x][e + 1] = v.y;
      }
    uint32_t o[4][4];
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      uint32_t b[4];
      ldsm_t(o[x], v_nk + x * 16 * VROW);
#pragma unroll
      for (int y = 0; y <= x; ++y) {
        ldsm_t(b, t_mk + DC_P + tri_at(x, y));
        mma16(M[2 * y], o[x], b[0], b[1]);
        mma16(M[2 * y + 1], o[x], b[2], b[3]);
        ldsm_t(b, t_mk + DC_P_LO + tri_at(x, y));
        mma16(M[2 * y], o[x], b[0], b[1]);
        mma16(M[2 * y + 1], o[x], b[2], b[3]);
      }
    }
    // dR^T = dU^T T, columns of T up to the block of 16 rows: chains of dependent products, between them G^T + (scale c O')^T Q
    float R[8][4];
#pragma unroll
    for (int x = 0; x < 8; ++x)
#pragma unroll
      for (int e = 0; e < 4; ++e) R[x][e] = 0.0f;
#pragma unroll
    for (int x = 3; x >= 0; --x) {
      uint32_t hi[4], lo[4], bh[4], bl[4];
      a_parts(M[2 * x], M[2 * x + 1], hi, lo);
#pragma unroll
      for (int y = 0; y <= x; ++y) {
        ldsm_t(bh, t_mk + tri_at(x, y));
        ldsm_t(bl, t_mk + DC_T_LO + tri_at(x, y));
        mma_split(R[2 * y], R[2 * y + 1], hi, lo, bh, bl);
      }
#pragma unroll
      for (int z = 0; z < 4; ++z) {
        const float2 c = *(const float2*)(f->c + 16 * x + 8 * (z >> 1) + 2 * t);
        split2(p.scale * c.x * __uint_as_float(o[x][z] << 16), p.scale * c.y * __uint_as_float(o[x][z] & 0xffff0000u), hi[z], lo[z]);
      }
#pragma unroll
      for (int y = 0; y < DK / 16; ++y) {
        ldsm_t(bh, q_at + wide(mk, x, y));
        mma16(G[2 * y], hi, bh[0], bh[1]);
        mma16(G[2 * y + 1], hi, bh[2], bh[3]);
        mma16(G[2 * y], lo, bh[0], bh[1]);
        mma16(G[2 * y + 1], lo, bh[2], bh[3]);
      }
    }
    put_labels<true>(R, st + Shape::v_at + warp * 32, VROW, lane, gp.drs + which * DC * p.dvp + col0 + warp * 16, p.dvp, DC, 16);
    // G^T -= (beta c dR)^T K
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      uint32_t hi[4], lo[4], b[4];
      float y0[4], y1[4];
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        const float2 be = *(const float2*)(f->beta + 16 * x + 8 * z + 2 * t), c = *(const float2*)(f->c + 16 * x + 8 * z + 2 * t);
        float* r = R[2 * x + z];
        r[0] *= be.x, r[1] *= be.y, r[2] *= be.x, r[3] *= be.y;  // dV
        float* y = z ? y1 : y0;
        y[0] = -c.x * r[0], y[1] = -c.y * r[1], y[2] = -c.x * r[2], y[3] = -c.y * r[3];
      }
      a_parts(y0, y1, hi, lo);
#pragma unroll
      for (int y = 0; y < DK / 16; ++y) {
        ldsm_t(b, k_at + wide(mk, x, y));
        mma16(G[2 * y], hi, b[0], b[1]);
        mma16(G[2 * y + 1], hi, b[2], b[3]);
        mma16(G[2 * y], lo, b[0], b[1]);
        mma16(G[2 * y + 1], lo, b[2], b[3]);
      }
    }
    __nv_bfloat16* out = gp.dv + ((span.row0 + (long long)(n - 1 - i) * DC) * p.hv + h) * p.dv + col0 + warp * 16;
    const int cols = min(16, p.dv - col0 - warp * 16);
    if (gp.vec_dv) put_labels<true>(R, st + Shape::v_at + warp * 32, VROW, lane, out, (long long)p.hv * p.dv, span.len(n - 1 - i), cols);
    else put_labels<false>(R, st + Shape::v_at + warp * 32, VROW, lane, out, (long long)p.hv * p.dv, span.len(n - 1 - i), cols);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (lane == 0) arrive(&bars[s].empty);
  }
  kernel_started();
  if (gp.dW0)
#pragma unroll
    for (int x = 0; x < DK / 8; ++x)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int f = 8 * x + 2 * t + (e & 1), l = label + (e >> 1) * 8;
        if (f < p.dk && l < p.dv) gp.dW0[(model + l) * p.dk + f] = G[x][e];
      }
}

// ---- gradients of the rows ---------------------------------------------------------------------------------------------------------------
// One block of 16 warps per SM goes through pieces of work, each a chunk and a head of labels; the heads that share features follow each other. A warp has 16
// rows and a quarter of the columns. Labels come in slices of 64 by cp.async through a ring that runs on from one piece into the next; the sums over labels (O' S^T,
// dR S^T, U G^T, O' U^T, dR U^T) stay in registers, and F and E go through shared memory to the products with K and Q. Sums over the diagonal of a product (dR.v of a
// row, S.G) are taken from fragments that are there for others. One block's sums
// fill half of an SM's registers.
constexpr int ROWS_PARTS = 4, ROWS_THREADS = 128 * ROWS_PARTS, ROWS_SLICE = 64;  // parts of the columns, four warps each

template <int DK>
struct RowsShape {
  static constexpr int row = DK + 8, vrow = ROWS_SLICE + 8;
  static constexpr int models = ROWS_SLICE * DK * 2, labels = DC * vrow * 2, stage = 2 * models + 4 * labels;
  static constexpr int qk = 2 * DC * row * 2, tiles = 3 * DC_TRI, kept = DC_BLOCK - DC_P + DC_TRI, sums = (ROWS_PARTS * 3 + 4) * DC * 4;
  static constexpr int stages = 2, smem = qk + tiles + kept + sums + stages * stage, totals = 2 * DC * DK;
};
static_assert(RowsShape<128>::smem <= 226 * 1024, "must fit an SM");

// Zeros in elements from `begin` to `end` - 1, by the threads of the whole grid
__device__ __forceinline__ void clear_span(__nv_bfloat16* p, long long begin, long long end) {
  unsigned short* const first = (unsigned short*)p + begin;
  const long long n = end - begin, ahead = min((long long)((-(uintptr_t)first & 15) / 2), n), units = (n - ahead) / 8;  // elements before the first whole 16 bytes, and those
  const long long at = (long long)blockIdx.x * blockDim.x + threadIdx.x, step = (long long)gridDim.x * blockDim.x;
  for (long long u = at; u < units; u += step) *(uint4*)(first + ahead + u * 8) = make_uint4(0u, 0u, 0u, 0u);
  if (at < n - units * 8) first[at < ahead ? at : at + units * 8] = 0;  // fewer than 16 at the ends
}
// Rows outside every chain have no part in the answers: their gradients are zeros
__device__ __forceinline__ void clear_outside(const DeltaGradParams& gp, int chunks) {
  const DeltaChunkParams& p = gp.f;
  const long long lo = chunks > 0 ? p.chunks[0].row0 : 0, hi = chunks > 0 ? p.chunks[chunks - 1].row0 + p.chunks[chunks - 1].len : 0;
  const long long wk = (long long)p.hk * p.dk, wv = (long long)p.hv * p.dv;
  for (int side = 0; side < 2; ++side) {
    const long long begin = side ? hi : 0, end = side ? p.n_rows : lo;
    if (begin >= end) continue;
    clear_span(gp.dq, begin * wk, end * wk);
    clear_span(gp.dk, begin * wk, end * wk);
    clear_span(gp.dv, begin * wv, end * wv);
    clear_span(gp.dg, begin * p.hv, end * p.hv);
    clear_span(gp.dbeta, begin * p.hv, end * p.hv);
  }
}

template <int DK>
__global__ void __launch_bounds__(ROWS_THREADS) delta_rowgrad_kernel(const __grid_constant__ DeltaGradParams gp) {
  using Shape = RowsShape<DK>;
  constexpr int ROW = Shape::row, VROW = Shape::vrow, NT = DK / 8 / ROWS_PARTS, PAIRS = 4 / ROWS_PARTS;  // tiles of 8 columns of a warp; blocks of 16 columns of F and E
  const DeltaChunkParams& p = gp.f;
  constexpr int STAGES = Shape::stages;
  const int more = p.hv / p.hk;
  extern __shared__ __align__(16) unsigned char rows_smem[];
  __nv_bfloat16* Qs = (__nv_bfloat16*)rows_smem;
  __nv_bfloat16* Ks = Qs + DC * ROW;
  unsigned char* Fs = rows_smem + Shape::qk;
  unsigned char *Es = Fs + DC_TRI, *Bs = Es + DC_TRI;                         // E, and beta E
  unsigned char *Ps = Bs + DC_TRI, *Gs = Ps + DC_BLOCK - DC_P;                     // P in two parts and the factors; D o K K^T
  const DeltaFactors* f = (const DeltaFactors*)(Ps + DC_FACTORS - DC_P);
  float* sums = (float*)(Gs + DC_TRI);  // [ROWS_PARTS][DC][3]
  float* cols = sums + ROWS_PARTS * DC * 3;      // [4 blocks of rows][DC]
  unsigned char* stages = (unsigned char*)(cols + 4 * DC);
  float* totals = gp.totals + (size_t)blockIdx.x * Shape::totals;  // where several heads share features
  __shared__ float model_dots[ROWS_THREADS / 32];
  const int tid = threadIdx.x, warp = warp_index(), lane = tid & 31, g = lane >> 2, t = lane & 3;
  // block of 16 rows and quarter of the columns. The ten warps with a block of F and E come first, so that no scheduler has more than three of them
  const int up = warp - 10, wr = warp < 10 ? (warp >= 1) + (warp >= 3) + (warp >= 6) : (up >= 3) + (up >= 5), wc = warp < 10 ? warp - wr * (wr + 1) / 2 : up < 3 ? up + 1 : up < 5 ? up - 1 : 3;
  kernel_inputs_ready();
  const int slices = (p.dvp + ROWS_SLICE - 1) / ROWS_SLICE;
  // Pieces: all heads of labels of a (chunk, head of features), then the next of this block's. What a copy needs is kept beside them: a piece changes once in
  // several slices, and the divisions would cost more instructions than the products.
  const int chunks = p.chunk_off[p.n_chains], chunk_step = gridDim.x / p.hk, head_step = gridDim.x % p.hk;
  struct Piece {
    int chunk, kh, hh, slice, len;
    long long row0;
  };
  auto find = [&](Piece& w) {
    if (w.chunk >= chunks) return;
    const DeltaChunk at = p.chunks[w.chunk];
    w.len = at.len;
    w.row0 = at.row0;
  };
  // true: another piece
  auto advance = [&](Piece& w) {
    if (++w.slice < slices) return false;
    w.slice = 0;
    if (++w.hh < more) return true;
    w.hh = 0;
    w.chunk += chunk_step;
    w.kh += head_step;
    if (w.kh >= p.hk) {
      w.kh -= p.hk;
      ++w.chunk;
    }
    find(w);
    return true;
  };
  const int row_l = tid / (ROWS_SLICE / 8), col_l = tid % (ROWS_SLICE / 8) * 8;  // of labels
  static_assert(ROWS_THREADS == DC * ROWS_SLICE / 8, "a thread has a unit of each tile of labels");
  const __nv_bfloat16 *from_s, *from_g, *from_u, *from_r, *from_o, *from_v;  // this thread's part of the next slice
  auto aim = [&](const Piece& w) {
    if (w.chunk >= chunks) return;
    const int h = w.kh * more + w.hh;
    const long long which = (long long)w.chunk * p.hv + h, kept = (which * DC + row_l) * p.dvp + col_l, i = w.row0 + (row_l < w.len ? row_l : 0);
    from_s = p.starts + which * p.dvp * DK;
    from_g = gp.ends + which * p.dvp * DK;
    from_u = p.steps + kept;
    from_r = gp.drs + kept;
    from_o = p.dout.p + i * p.dout.ld + h * p.dout.width + col_l;
    from_v = p.v.p + i * p.v.ld + h * p.v.width + col_l;
  };
  auto bring = [&](const Piece& w, int ring) {  // a slice of the labels of S, G, U, dR, O' and V
    if (w.chunk >= chunks) return;
    const int l0 = w.slice * ROWS_SLICE, l = l0 + col_l;
    const uint32_t st = smem32(stages) + ring * Shape::stage;
#pragma unroll
    for (int u = tid; u < ROWS_SLICE * (DK / 8); u += ROWS_THREADS) {
      const int at_l = u % ROWS_SLICE, unit = u / ROWS_SLICE, from = (unit * model_labels(l0, p.dvp) + at_l) * 8;
      const bool there = l0 + at_l < p.dvp;
      copy16(st + unit * ROWS_SLICE * 16 + at_l * 16, there ? from_s + from : p.starts, there);
      copy16(st + Shape::models + unit * ROWS_SLICE * 16 + at_l * 16, there ? from_g + from : gp.ends, there);
    }
    const uint32_t to = st + 2 * Shape::models + (row_l * VROW + col_l) * 2;
    const bool there = l < p.dvp, given = row_l < w.len && l < p.v.width;  // labels and their gradients are of one width, rounded up to 8
    copy16(to, there ? from_u : p.steps, there);
    copy16(to + Shape::labels, there ? from_r : gp.drs, there);
    copy16(to + 2 * Shape::labels, given ? from_o : p.dout.p, given);
    copy16(to + 3 * Shape::labels, given ? from_v : p.v.p, given);
    from_s += ROWS_SLICE * DK, from_g += ROWS_SLICE * DK, from_u += ROWS_SLICE, from_r += ROWS_SLICE, from_o += ROWS_SLICE, from_v += ROWS_SLICE;
  };
  auto commit = [] { asm volatile("cp.async.commit_group;" ::: "memory"); };

  Piece now = {(int)(blockIdx.x / p.hk), (int)(blockIdx.x % p.hk), 0, 0, 0, 0};
  find(now);
  Piece next = now;
  aim(next);
  int at_ring = 0, next_ring = 0;
  for (int i = 0; i + 1 < STAGES; ++i) {
    bring(next, next_ring++);
    commit();
    if (advance(next)) aim(next);
  }
  const int row0 = 16 * wr, colw = wc * (DK / ROWS_PARTS), i0 = row0 + g, i1 = i0 + 8;
  while (now.chunk < chunks) {
    const int chunk = now.chunk, kh = now.kh, hh = now.hh, h = kh * more + hh;
    const DeltaChunk at = {now.row0, now.len, 0};
    float dP[2 * PAIRS][4], dA[2 * PAIRS][4], aQ[NT][4], aX[NT][4], aH[NT][4], rv[2][4], sg[2][4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
#pragma unroll
      for (int x = 0; x < 2 * PAIRS; ++x) dP[x][e] = dA[x][e] = 0.0f;
#pragma unroll
      for (int x = 0; x < NT; ++x) aQ[x][e] = aX[x][e] = aH[x][e] = 0.0f;
      rv[0][e] = rv[1][e] = sg[0][e] = sg[1][e] = 0.0f;
    }
    for (int sl = 0; sl < slices; ++sl) {
      asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 2) : "memory");
      __syncthreads();  // this slice is there for all, and all have left the slice before
      bring(next, next_ring);
      if (advance(next)) aim(next);
      if (++next_ring == STAGES) next_ring = 0;
      if (sl == 0) {  // and what the piece needs after its slices: all have left that of the piece before
        if (hh == 0) {
          for (int u = tid; u < DC * (DK / 8); u += ROWS_THREADS) {
            const int row = u / (DK / 8), col = u % (DK / 8) * 8;
            const bool there = row < at.len && col < p.k.width;
            const long long i = there ? at.row0 + row : 0;
            const int c = there ? kh * p.k.width + col : 0;
            copy16(smem32(Ks + row * ROW + col), p.k.p + i * p.k.ld + c, there);
            copy16(smem32(Qs + row * ROW + col), p.q.p + i * p.q.ld + c, there);
          }
        }
        const long long which = (long long)chunk * p.hv + h;
        for (int i = tid * 16; i < DC_BLOCK - DC_P; i += ROWS_THREADS * 16) copy16(smem32(Ps) + i, p.blocks + which * DC_BLOCK + DC_P + i, true);
        for (int i = tid * 16; i < DC_TRI; i += ROWS_THREADS * 16) copy16(smem32(Gs) + i, p.gram + which * DC_TRI + i, true);
      }
      commit();
      const uint32_t st = smem32(stages) + at_ring * Shape::stage;
      if (++at_ring == STAGES) at_ring = 0;
      const uint32_t s_mk = st + (lane & 15) * 16 + ((lane >> 4) + colw / 8) * ROWS_SLICE * 16, g_mk = s_mk + Shape::models, u_at = st + 2 * Shape::models;
      const uint32_t a_mk = u_at + lane_mk(lane, VROW) + row0 * VROW * 2, u_nk = u_at + lane_nk(lane, VROW) + wc * 16 * PAIRS * VROW * 2, v_nk = u_at + 3 * Shape::labels + lane_nk(lane, VROW) + row0 * VROW * 2;
#pragma unroll
      for (int x = 0; x < ROWS_SLICE / 16; ++x) {
        uint32_t aU[4], aR[4], aO[4], b[4];
        ldsm(aU, a_mk + x * 32);
        ldsm(aR, a_mk + Shape::labels + x * 32);
        ldsm(aO, a_mk + 2 * Shape::labels + x * 32);
#pragma unroll
        for (int y = 0; y < PAIRS; ++y) {
          if (PAIRS * wc + y > wr) break;
          ldsm(b, u_nk + y * 16 * VROW * 2 + x * 32);
          mma16(dP[2 * y], aO, b[0], b[1]);
          mma16(dP[2 * y + 1], aO, b[2], b[3]);
          mma16(dA[2 * y], aR, b[0], b[1]);
          mma16(dA[2 * y + 1], aR, b[2], b[3]);
        }
        if (wc == x % ROWS_PARTS) {  // dR.v of the warp's rows: the diagonal of dR V^T
          ldsm(b, v_nk + x * 32);
          mma16(rv[0], aR, b[0], b[1]);
          mma16(rv[1], aR, b[2], b[3]);
        }
#pragma unroll
        for (int y = 0; y < NT / 2; ++y) {
          uint32_t bg[4];
          ldsm_t(b, s_mk + x * 256 + y * 2 * ROWS_SLICE * 16);
          ldsm_t(bg, g_mk + x * 256 + y * 2 * ROWS_SLICE * 16);
          mma16(aQ[2 * y], aO, b[0], b[1]);
          mma16(aQ[2 * y + 1], aO, b[2], b[3]);
          mma16(aX[2 * y], aR, b[0], b[1]);
          mma16(aX[2 * y + 1], aR, b[2], b[3]);
          mma16(aH[2 * y], aU, bg[0], bg[1]);
          mma16(aH[2 * y + 1], aU, bg[2], bg[3]);
          if ((y & 3) == wr) {  // S.G: the diagonal of S^T G, the same 16 labels and features as both operands
            const uint32_t as[4] = {b[0], b[2], b[1], b[3]};
            mma16(sg[0], as, bg[0], bg[1]);
            mma16(sg[1], as, bg[2], bg[3]);
          }
        }
      }
      advance(now);
    }
    if (slices < STAGES) {  // what the piece needs next came with a slice that has not been waited for
      asm volatile("cp.async.wait_group 0;" ::: "memory");
      __syncthreads();
    }

    // F, E and beta E of the warp's 16 x 32 elements, and the sums of H over its rows and columns
    float row_p[2] = {}, row_a[2] = {};
    const float be0 = f->beta[i0], be1 = f->beta[i1], hi0 = f->hi[i0], hi1 = f->hi[i1], lo0 = f->lo[i0], lo1 = f->lo[i1];
#pragma unroll
    for (int y = 0; y < PAIRS; ++y) {
      if (PAIRS * wc + y > wr) break;
      const int at_tri = tri_at(wr, PAIRS * wc + y);
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int j = (PAIRS * wc + y) * 16 + 8 * x + 2 * t;
        const float2 ch = *(const float2*)(f->hi + j), cl = *(const float2*)(f->lo + j);
        float col_h[2] = {};
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
          const int i = i0 + 4 * e, unit = at_tri + tri_unit(g + 4 * e, x) + 4 * t;
          const float be = e ? be1 : be0, hi = e ? hi1 : hi0, lo = e ? lo1 : lo0;
          const uint32_t p2 = *(const uint32_t*)(Ps + unit), l2 = *(const uint32_t*)(Ps + DC_TRI + unit), k2 = *(const uint32_t*)(Gs + unit);
          const float d[2] = {exp2_fast((hi - ch.x) + (lo - cl.x)), exp2_fast((hi - ch.y) + (lo - cl.y))};
          const float pp[2] = {__uint_as_float(p2 << 16) + __uint_as_float(l2 << 16), __uint_as_float(p2 & 0xffff0000u) + __uint_as_float(l2 & 0xffff0000u)};
          const float kk[2] = {__uint_as_float(k2 << 16), __uint_as_float(k2 & 0xffff0000u)};
          float F[2], E[2];
#pragma unroll
          for (int z = 0; z < 2; ++z) {
            const bool below = j + z < i;
            const float dp = dP[2 * y + x][e + z], da = -dA[2 * y + x][e + z];
            F[z] = j + z <= i ? p.scale * d[z] * dp : 0.0f;
            E[z] = below ? d[z] * da : 0.0f;
            const float hp = below ? dp * pp[z] : 0.0f, ha = below ? da * kk[z] : 0.0f;
            row_p[e / 2] += hp;
            row_a[e / 2] += ha;
            col_h[z] += fmaf(be, ha, hp);
          }
          *(uint32_t*)(Fs + unit) = pack2(F[0], F[1]);
          *(uint32_t*)(Es + unit) = pack2(E[0], E[1]);
          *(uint32_t*)(Bs + unit) = pack2(be * E[0], be * E[1]);
        }
#pragma unroll
        for (int z = 0; z < 2; ++z) {
          float v = col_h[z];
          v += __shfl_xor_sync(0xffffffffu, v, 4);
          v += __shfl_xor_sync(0xffffffffu, v, 8);
          v += __shfl_xor_sync(0xffffffffu, v, 16);
          if (g == 0) cols[wr * DC + j + z] = v;
        }
      }
    }
    const bool diagonal = t == g >> 1;  // this lane has elements (g, g) and (g + 8, g + 8) of the diagonal products
    {
      const float v = warp_sum(diagonal ? (g & 1 ? sg[0][1] + sg[1][3] : sg[0][0] + sg[1][2]) : 0.0f);
      if (lane == 0) model_dots[warp] = v;
    }
    __syncthreads();

    // of rows i0 and i1: what passes from S and from H's rows, dbeta, k.(r U G^T)
    const float c0 = f->c[i0], c1 = f->c[i1], r0 = f->r[i0], r1 = f->r[i1], last = f->last;
    float dots[3][2] = {{fmaf(be0, row_a[0], row_p[0]), fmaf(be1, row_a[1], row_p[1])},
                        {row_a[0] + (diagonal ? (g & 1 ? rv[0][1] : rv[0][0]) : 0.0f), row_a[1] + (diagonal ? (g & 1 ? rv[1][3] : rv[1][2]) : 0.0f)},
                        {0.0f, 0.0f}};
    auto pair_at = [&](const __nv_bfloat16* tile, int row, int x) {  // two elements of a row in the warp's columns
      const uint32_t v = *(const uint32_t*)(tile + row * ROW + colw + 8 * x + 2 * t);
      return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
    };
#pragma unroll
    for (int x = 0; x < NT; ++x) {
      aQ[x][0] *= p.scale * c0, aQ[x][1] *= p.scale * c0, aQ[x][2] *= p.scale * c1, aQ[x][3] *= p.scale * c1;
      aX[x][0] *= -c0, aX[x][1] *= -c0, aX[x][2] *= -c1, aX[x][3] *= -c1;
      aH[x][0] *= r0, aH[x][1] *= r0, aH[x][2] *= r1, aH[x][3] *= r1;
      const float2 k0 = pair_at(Ks, i0, x), k1 = pair_at(Ks, i1, x), q0 = pair_at(Qs, i0, x), q1 = pair_at(Qs, i1, x);
      const float x0 = k0.x * aX[x][0] + k0.y * aX[x][1], x1 = k1.x * aX[x][2] + k1.y * aX[x][3];
      dots[0][0] += fmaf(be0, x0, q0.x * aQ[x][0] + q0.y * aQ[x][1]);
      dots[0][1] += fmaf(be1, x1, q1.x * aQ[x][2] + q1.y * aQ[x][3]);
      dots[1][0] += x0;
      dots[1][1] += x1;
      dots[2][0] += k0.x * aH[x][0] + k0.y * aH[x][1];
      dots[2][1] += k1.x * aH[x][2] + k1.y * aH[x][3];
    }
#pragma unroll
    for (int d = 0; d < 3; ++d)
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        float v = dots[d][z];
        v += __shfl_xor_sync(0xffffffffu, v, 1);
        v += __shfl_xor_sync(0xffffffffu, v, 2);
        if (t == 0) sums[(wc * DC + i0 + 8 * z) * 3 + d] = v;
      }
    const uint32_t k_mk = smem32(Ks) + lane_mk(lane, ROW) + colw * 2, q_mk = smem32(Qs) + lane_mk(lane, ROW) + colw * 2;
    const uint32_t f_mk = smem32(Fs) + tri_mk(lane) + tri_at(wr, 0), f_nk = smem32(Fs) + tri_nk(lane) + tri_at(0, wr);
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      uint32_t a[4], e[4], b[4];
      if (x <= wr) {  // rows of F and E: dQ and x
        ldsm(a, f_mk + tri_at(0, x));
        ldsm(e, f_mk + DC_TRI + tri_at(0, x));
#pragma unroll
        for (int y = 0; y < NT / 2; ++y) {
          ldsm_t(b, k_mk + x * 16 * ROW * 2 + y * 32);
          mma16(aQ[2 * y], a, b[0], b[1]);
          mma16(aQ[2 * y + 1], a, b[2], b[3]);
          mma16(aX[2 * y], e, b[0], b[1]);
          mma16(aX[2 * y + 1], e, b[2], b[3]);
        }
      }
      if (x >= wr) {  // columns of F and beta E: back
        ldsm_t(a, f_nk + tri_at(x, 0));
        ldsm_t(e, f_nk + 2 * DC_TRI + tri_at(x, 0));
#pragma unroll
        for (int y = 0; y < NT / 2; ++y) {
          ldsm_t(b, q_mk + x * 16 * ROW * 2 + y * 32);
          mma16(aH[2 * y], a, b[0], b[1]);
          mma16(aH[2 * y + 1], a, b[2], b[3]);
          ldsm_t(b, k_mk + x * 16 * ROW * 2 + y * 32);
          mma16(aH[2 * y], e, b[0], b[1]);
          mma16(aH[2 * y + 1], e, b[2], b[3]);
        }
      }
    }
    __syncthreads();  // sums are there; Q, K, F, E and the factors are free
    // dQ (in aQ) and dK (in aX), added up over the heads of labels that share these features by the thread that has the elements
    float4* mine = (float4*)totals + tid;
#pragma unroll
    for (int x = 0; x < NT; ++x) {
      aX[x][0] = fmaf(be0, aX[x][0], aH[x][0]), aX[x][1] = fmaf(be0, aX[x][1], aH[x][1]);
      aX[x][2] = fmaf(be1, aX[x][2], aH[x][2]), aX[x][3] = fmaf(be1, aX[x][3], aH[x][3]);
      if (hh > 0) {
        const float4 q = mine[2 * x * ROWS_THREADS], k = mine[(2 * x + 1) * ROWS_THREADS];
        aQ[x][0] += q.x, aQ[x][1] += q.y, aQ[x][2] += q.z, aQ[x][3] += q.w;
        aX[x][0] += k.x, aX[x][1] += k.y, aX[x][2] += k.z, aX[x][3] += k.w;
      }
    }
    if (hh + 1 < more) {
#pragma unroll
      for (int x = 0; x < NT; ++x) {
        mine[2 * x * ROWS_THREADS] = make_float4(aQ[x][0], aQ[x][1], aQ[x][2], aQ[x][3]);
        mine[(2 * x + 1) * ROWS_THREADS] = make_float4(aX[x][0], aX[x][1], aX[x][2], aX[x][3]);
      }
    } else {
      const long long to0 = ((at.row0 + i0) * p.hk + kh) * p.dk + colw + 2 * t, to1 = to0 + 8ll * p.hk * p.dk;
#pragma unroll
      for (int x = 0; x < NT; ++x)
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
          const int col = colw + 8 * x + 2 * t;
          if ((e ? i1 : i0) >= at.len) continue;
          const long long to = (e ? to1 : to0) + 8 * x;
          if (gp.vec_dk) {
            if (col < p.dk) {
              *(uint32_t*)(gp.dq + to) = pack2(aQ[x][e], aQ[x][e + 1]);
              *(uint32_t*)(gp.dk + to) = pack2(aX[x][e], aX[x][e + 1]);
            }
          } else {
#pragma unroll
            for (int z = 0; z < 2; ++z)
              if (col + z < p.dk) {
                gp.dq[to + z] = __float2bfloat16_rn(aQ[x][e + z]);
                gp.dk[to + z] = __float2bfloat16_rn(aX[x][e + z]);
              }
          }
        }
    }
    if (warp == 0) {  // two rows a lane: dbeta, and dg by a scan from the chunk's end
      float db[2], ahead = 0.0f;
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        const int i = 2 * lane + z;
        float v[3];
#pragma unroll
        for (int d = 0; d < 3; ++d) {
          v[d] = 0.0f;
          for (int w = 0; w < ROWS_PARTS; ++w) v[d] += sums[(w * DC + i) * 3 + d];
        }
        for (int w = i / 16; w < 4; ++w) v[0] -= cols[w * DC + i];
        db[z] = v[0] - v[2];
        ahead += v[2];
        if (i < at.len) gp.dbeta[(at.row0 + i) * p.hv + h] = __float2bfloat16_rn(v[1]);
      }
      const float decay = last * warp_sum(lane < ROWS_THREADS / 32 ? model_dots[lane] : 0.0f) + warp_sum(ahead);
      float sum = db[0] + db[1];  // of this lane's rows and all behind them
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const float v = __shfl_down_sync(0xffffffffu, sum, o);
        if (lane + o < 32) sum += v;
      }
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        const int i = 2 * lane + z;
        if (i < at.len) gp.dg[(at.row0 + i) * p.hv + h] = __float2bfloat16_rn(decay + sum - (z ? db[0] : 0.0f));
      }
    }
  }
  kernel_started();
  copies_done();
  clear_outside(gp, chunks);
}

}  // namespace wpsgd
