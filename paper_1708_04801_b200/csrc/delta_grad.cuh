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
// Rounding: G, P, dU, scale c O' and beta c dR in two bf16 parts in the walk's products; S, U, G, dR, F and E are rounded to bf16
// once where the third kernel multiplies them. Gradients leave as bf16.
#pragma once

#include "delta_chunk.cuh"

namespace wpsgd {

struct DeltaGradParams {
  DeltaChunkParams f;
  __nv_bfloat16* ends;   // [chunks][hv][dvp][DK]: G behind the chunk
  __nv_bfloat16* drs;    // [chunks][hv][DC][dvp]: dR
  const float* dW;
  float* dW0;
  __nv_bfloat16 *dq, *dk, *dv, *dg, *dbeta;
  int vec_dv, vec_dk;  // rows of dv take 16 bytes at a time, rows of dq and dk 4
};

template <int DK, int NW>
__global__ void __launch_bounds__(ChainShape<DK, NW>::threads) delta_back_kernel(const __grid_constant__ DeltaGradParams gp) {
  const DeltaChunkParams& p = gp.f;
  using Shape = ChainShape<DK, NW>;
  constexpr int ROW = Shape::row * 2, VROW = Shape::vrow * 2, STAGES = Shape::stages, Q_AT = Shape::q_at, V_AT = Shape::v_at;  // bytes
  extern __shared__ __align__(16) unsigned char chain_smem[];
  __shared__ unsigned long long full[STAGES], empty[STAGES];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  kernel_started();
  kernel_inputs_ready();
  const int slice = blockIdx.x % p.slices, h = blockIdx.x / p.slices % p.hv, chain = p.order[blockIdx.x / p.slices / p.hv], kh = h / (p.hv / p.hk);
  const int col0 = slice * 16 * NW, warps = min(NW, (p.dvp - col0) / 16);  // warps with labels
  const int first = p.chunk_off[chain], n = p.chunk_off[chain + 1] - first;
  constexpr bool COPIERS = Shape::copiers > 0;
  const int bringers = COPIERS ? Shape::copiers : warps;
  if (tid == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(&full[s], 32 * bringers);
      mbar_init(&empty[s], warps);
    }
    mbar_fence_init();
  }
  __syncthreads();
  if (COPIERS && warp >= NW) {
    bring_chunks<DK, NW>(p, p.dout, smem32(chain_smem), first + n - 1, -1, n, h, kh, col0, warp - NW, lane, full, empty);
    return;
  }
  if (warp >= warps) return;
  if (!COPIERS && n > 0 && p.drop != 0) bring_chunk<DK, NW>(p, p.dout, smem32(chain_smem), first + n - 1, h, kh, col0, warp, warps, lane, &full[0]);

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
    if (!COPIERS && i + 1 < n) {  // the next chunk, once all have left the one that was there; p.drop (a test hook): one that is never brought
      if (i + 1 >= STAGES) ok = __all_sync(0xffffffffu, mbar_wait_bounded(&empty[s1], ((i + 1) / STAGES - 1) & 1, p.spin_limit));
      if (ok && i + 1 != p.drop) bring_chunk<DK, NW>(p, p.dout, smem32(chain_smem) + s1 * Shape::stage, first + n - 2 - i, h, kh, col0, warp, warps, lane, &full[s1]);
    }
    if (!ok || !__all_sync(0xffffffffu, mbar_wait_bounded(&full[s], (i / STAGES) & 1, p.spin_limit))) {
      if (lane == 0) set_status(p.status, DEV_TIMEOUT, 26, i);
      copies_done();  // none of this warp's is in flight when it leaves
      return;
    }
    unsigned char* st = chain_smem + s * Shape::stage;
    const unsigned char* block = st + Shape::block_at;
    const DeltaFactors* f = (const DeltaFactors*)(block + DC_FACTORS);
    const int chunk = first + n - 1 - i;
    const long long which = (long long)chunk * p.hv + h;
    const uint32_t k_nk = smem32(st) + lane_nk(lane, Shape::row), k_mk = smem32(st) + lane_mk(lane, Shape::row), q_mk = k_mk + Q_AT;
    const uint32_t t_mk = smem32(block) + tri_mk(lane), v_nk = smem32(st + V_AT) + warp * 32 + lane_nk(lane, Shape::vrow);

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
      uint32_t* to = (uint32_t*)(gp.ends + (which * p.dvp + label) * DK + 16 * x + 2 * t);
      to[0] = hi[0];
      to[4 * DK] = hi[1];
      to[4] = hi[2];
      to[4 * DK + 4] = hi[3];
#pragma unroll
      for (int y = 0; y < 4; ++y) ldsm(b[y], k_nk + y * 16 * ROW + x * 32);
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
    const float last = f->last;
#pragma unroll
    for (int x = 0; x < DK / 8; ++x)
#pragma unroll
      for (int e = 0; e < 4; ++e) G[x][e] *= last;
    // ... and G^T + (scale c O')^T Q
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      uint32_t a[4], b[4], hi[4], lo[4];
      ldsm_t(a, v_nk + x * 16 * VROW);
#pragma unroll
      for (int y = 0; y <= x; ++y) {
        ldsm_t(b, t_mk + DC_P + tri_at(x, y));
        mma16(M[2 * y], a, b[0], b[1]);
        mma16(M[2 * y + 1], a, b[2], b[3]);
        ldsm_t(b, t_mk + DC_P_LO + tri_at(x, y));
        mma16(M[2 * y], a, b[0], b[1]);
        mma16(M[2 * y + 1], a, b[2], b[3]);
      }
#pragma unroll
      for (int z = 0; z < 4; ++z) {
        const float2 c = *(const float2*)(f->c + 16 * x + 8 * (z >> 1) + 2 * t);
        split2(p.scale * c.x * __uint_as_float(a[z] << 16), p.scale * c.y * __uint_as_float(a[z] & 0xffff0000u), hi[z], lo[z]);
      }
#pragma unroll
      for (int y = 0; y < DK / 16; ++y) {
        ldsm_t(b, q_mk + x * 16 * ROW + y * 32);
        mma16(G[2 * y], hi, b[0], b[1]);
        mma16(G[2 * y + 1], hi, b[2], b[3]);
        mma16(G[2 * y], lo, b[0], b[1]);
        mma16(G[2 * y + 1], lo, b[2], b[3]);
      }
    }
    // dR^T = dU^T T: columns of T up to the block of 16 rows
    float R[8][4];
#pragma unroll
    for (int x = 0; x < 8; ++x)
#pragma unroll
      for (int e = 0; e < 4; ++e) R[x][e] = 0.0f;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      uint32_t hi[4], lo[4], bh[4], bl[4];
      a_parts(M[2 * x], M[2 * x + 1], hi, lo);
#pragma unroll
      for (int y = 0; y <= x; ++y) {
        ldsm_t(bh, t_mk + tri_at(x, y));
        ldsm_t(bl, t_mk + DC_T_LO + tri_at(x, y));
        mma_split(R[2 * y], R[2 * y + 1], hi, lo, bh, bl);
      }
    }
    put_labels<true>(R, st + V_AT + warp * 32, VROW, lane, gp.drs + which * DC * p.dvp + col0 + warp * 16, p.dvp, DC, 16);
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
        ldsm_t(b, k_mk + x * 16 * ROW + y * 32);
        mma16(G[2 * y], hi, b[0], b[1]);
        mma16(G[2 * y + 1], hi, b[2], b[3]);
        mma16(G[2 * y], lo, b[0], b[1]);
        mma16(G[2 * y + 1], lo, b[2], b[3]);
      }
    }
    const DeltaChunk at = p.chunks[chunk];
    __nv_bfloat16* out = gp.dv + (at.row0 * p.hv + h) * p.dv + col0 + warp * 16;
    const int cols = min(16, p.dv - col0 - warp * 16);
    if (gp.vec_dv) put_labels<true>(R, st + V_AT + warp * 32, VROW, lane, out, (long long)p.hv * p.dv, at.len, cols);
    else put_labels<false>(R, st + V_AT + warp * 32, VROW, lane, out, (long long)p.hv * p.dv, at.len, cols);
    __syncwarp();
    if (lane == 0) arrive(&empty[s]);
  }
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
// One block of 16 warps for each chunk and head of features, which goes through the heads of labels that share them. A warp has 16 rows
// and a quarter of the columns. Labels come in slices of 32 by cp.async, two slices under way; the sums over labels (O' S^T, dR S^T, U G^T, O' U^T, dR U^T) stay
// in registers, and F and E go through shared memory to the products with K and Q.
constexpr int ROWS_THREADS = 512, ROWS_SLICE = 32;

template <int DK>
struct RowsShape {
  static constexpr int row = DK + 8, vrow = ROWS_SLICE + 8;
  static constexpr int models = ROWS_SLICE * row * 2, labels = DC * vrow * 2, stage = 2 * models + 4 * labels;
  static constexpr int qk = 2 * DC * row * 2, tiles = 3 * DC_TILE_BYTES, sums = 4 * DC * 5 * 4, totals = 2 * DC * DK * 4;
  static constexpr int smem(bool grouped) { return qk + 2 * stage + tiles + (int)sizeof(DeltaFactors) + sums + (grouped ? totals : 0); }
};

template <int DK>
__global__ void __launch_bounds__(ROWS_THREADS) delta_rowgrad_kernel(const __grid_constant__ DeltaGradParams gp) {
  using Shape = RowsShape<DK>;
  constexpr int ROW = Shape::row, VROW = Shape::vrow, NT = DK / 32;  // tiles of 8 columns of a warp
  const DeltaChunkParams& p = gp.f;
  extern __shared__ __align__(16) unsigned char rows_smem[];
  __nv_bfloat16* Qs = (__nv_bfloat16*)rows_smem;
  __nv_bfloat16* Ks = Qs + DC * ROW;
  unsigned char* stages = rows_smem + Shape::qk;
  unsigned char* Fs = stages + 2 * Shape::stage;
  unsigned char *Es = Fs + DC_TILE_BYTES, *Bs = Es + DC_TILE_BYTES;  // E, and beta E
  DeltaFactors* f = (DeltaFactors*)(Bs + DC_TILE_BYTES);
  float* sums = (float*)(f + 1);  // [4 quarters][DC][4]
  float* cols = sums + 4 * DC * 4;  // [4 blocks of rows][DC]
  float* totals = cols + 4 * DC;
  __shared__ float label_dots[DC], model_dots[ROWS_THREADS / 32];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3, wr = warp & 3, wc = warp >> 2;
  kernel_started();
  kernel_inputs_ready();
  const int chunk = blockIdx.x / p.hk, kh = blockIdx.x % p.hk, more = p.hv / p.hk;
  if (chunk >= p.chunk_off[p.n_chains]) return;
  const DeltaChunk at = p.chunks[chunk];
  const int slices = (p.dvp + ROWS_SLICE - 1) / ROWS_SLICE;

  for (int u = tid; u < DC * (DK / 8); u += ROWS_THREADS) {
    const int row = u / (DK / 8), col = u % (DK / 8) * 8;
    const bool there = row < at.len && col < p.k.width;
    const long long i = there ? at.row0 + row : 0;
    const int c = there ? kh * p.k.width + col : 0;
    copy16(smem32(Ks + row * ROW + col), p.k.p + i * p.k.ld + c, there);
    copy16(smem32(Qs + row * ROW + col), p.q.p + i * p.q.ld + c, there);
  }
  auto bring = [&](int h, int slice) {  // labels slice * 32 to + 31 of S, G, U, dR, O' and V
    unsigned char* st = stages + (slice & 1) * Shape::stage;
    const long long which = (long long)chunk * p.hv + h;
    const int l0 = slice * ROWS_SLICE;
    for (int u = tid; u < ROWS_SLICE * (DK / 8); u += ROWS_THREADS) {
      const int l = u / (DK / 8), col = u % (DK / 8) * 8;
      const bool there = l0 + l < p.dvp;
      const long long from = there ? (which * p.dvp + l0 + l) * DK + col : 0;
      copy16(smem32(st + (l * ROW + col) * 2), p.starts + from, there);
      copy16(smem32(st + Shape::models + (l * ROW + col) * 2), gp.ends + from, there);
    }
    for (int u = tid; u < DC * (ROWS_SLICE / 8); u += ROWS_THREADS) {
      const int row = u / (ROWS_SLICE / 8), col = u % (ROWS_SLICE / 8) * 8, l = l0 + col;
      unsigned char* to = st + 2 * Shape::models + (row * VROW + col) * 2;
      const bool there = l < p.dvp, o_there = row < at.len && l < p.dout.width, v_there = row < at.len && l < p.v.width;
      const long long from = there ? (which * DC + row) * p.dvp + l : 0, i = row < at.len ? at.row0 + row : 0;
      copy16(smem32(to), p.steps + from, there);
      copy16(smem32(to + Shape::labels), gp.drs + from, there);
      copy16(smem32(to + 2 * Shape::labels), p.dout.p + (o_there ? i * p.dout.ld + h * p.dout.width + l : 0), o_there);
      copy16(smem32(to + 3 * Shape::labels), p.v.p + (v_there ? i * p.v.ld + h * p.v.width + l : 0), v_there);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };

  const int row0 = 16 * wr, colw = wc * (DK / 4);
  for (int hh = 0; hh < more; ++hh) {
    const int h = kh * more + hh;
    const unsigned char* block = p.blocks + ((long long)chunk * p.hv + h) * DC_BLOCK + DC_FACTORS;
    for (int i = tid; i < (int)sizeof(DeltaFactors) / 16; i += ROWS_THREADS) copy16(smem32((unsigned char*)f + i * 16), block + i * 16, true);
    bring(h, 0);
    uint32_t P2[2][2], L2[2][2], K2[2][2];  // two elements each of P (in two parts) and D o K K^T, laid out as dP and dA
    if (wc <= wr) {
      const long long which = (long long)chunk * p.hv + h;
      const unsigned char *from = p.blocks + which * DC_BLOCK + DC_P, *gram = p.gram + which * DC_TRI;
      const int at_tri = (wr * (wr + 1) / 2 + wc) * 512;
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int unit = at_tri + tri_unit(g + 8 * e, x) + 4 * t;
          P2[x][e] = __ldg((const uint32_t*)(from + unit));
          L2[x][e] = __ldg((const uint32_t*)(from + DC_TRI + unit));
          K2[x][e] = __ldg((const uint32_t*)(gram + unit));
        }
    }
    float dP[2][4], dA[2][4], aQ[NT][4], aX[NT][4], aH[NT][4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      dP[0][e] = dP[1][e] = dA[0][e] = dA[1][e] = 0.0f;
#pragma unroll
      for (int x = 0; x < NT; ++x) aQ[x][e] = aX[x][e] = aH[x][e] = 0.0f;
    }
    float label_dot = 0.0f, model_dot = 0.0f;  // of row tid / 8; of this thread's part of S and G
    for (int sl = 0; sl < slices; ++sl) {
      if (sl + 1 < slices) {
        bring(h, sl + 1);
        asm volatile("cp.async.wait_group 1;" ::: "memory");
      } else {
        asm volatile("cp.async.wait_group 0;" ::: "memory");
      }
      __syncthreads();
      const unsigned char* st = stages + (sl & 1) * Shape::stage;
      const uint32_t s_mk = smem32(st) + lane_mk(lane, ROW) + colw * 2, g_mk = s_mk + Shape::models;
      const uint32_t u_at = smem32(st + 2 * Shape::models), a_mk = u_at + lane_mk(lane, VROW) + row0 * VROW * 2, u_nk = u_at + lane_nk(lane, VROW) + wc * 16 * VROW * 2;
#pragma unroll
      for (int x = 0; x < ROWS_SLICE / 16; ++x) {
        uint32_t aU[4], aR[4], aO[4], b[4];
        ldsm(aU, a_mk + x * 32);
        ldsm(aR, a_mk + Shape::labels + x * 32);
        ldsm(aO, a_mk + 2 * Shape::labels + x * 32);
        if (wc <= wr) {
          ldsm(b, u_nk + x * 32);
          mma16(dP[0], aO, b[0], b[1]);
          mma16(dP[1], aO, b[2], b[3]);
          mma16(dA[0], aR, b[0], b[1]);
          mma16(dA[1], aR, b[2], b[3]);
        }
#pragma unroll
        for (int y = 0; y < NT / 2; ++y) {
          ldsm_t(b, s_mk + x * 16 * ROW * 2 + y * 32);
          mma16(aQ[2 * y], aO, b[0], b[1]);
          mma16(aQ[2 * y + 1], aO, b[2], b[3]);
          mma16(aX[2 * y], aR, b[0], b[1]);
          mma16(aX[2 * y + 1], aR, b[2], b[3]);
          ldsm_t(b, g_mk + x * 16 * ROW * 2 + y * 32);
          mma16(aH[2 * y], aU, b[0], b[1]);
          mma16(aH[2 * y + 1], aU, b[2], b[3]);
        }
      }
      {  // dR.v of a row by eight threads, four labels each; S.G by all
        const unsigned char* lab = st + 2 * Shape::models + (tid / 8 * VROW + tid % 8 * 4) * 2;
        const uint2 r = *(const uint2*)(lab + Shape::labels), v = *(const uint2*)(lab + 3 * Shape::labels);
        label_dot = fmaf(__uint_as_float(r.x << 16), __uint_as_float(v.x << 16), label_dot);
        label_dot = fmaf(__uint_as_float(r.x & 0xffff0000u), __uint_as_float(v.x & 0xffff0000u), label_dot);
        label_dot = fmaf(__uint_as_float(r.y << 16), __uint_as_float(v.y << 16), label_dot);
        label_dot = fmaf(__uint_as_float(r.y & 0xffff0000u), __uint_as_float(v.y & 0xffff0000u), label_dot);
        for (int u = tid; u < ROWS_SLICE * (DK / 8); u += ROWS_THREADS) {
          const unsigned char* m = st + (u / (DK / 8) * ROW + u % (DK / 8) * 8) * 2;
          float x[8], y[8];
          XVec<__nv_bfloat16>::widen(*(const uint4*)m, x);
          XVec<__nv_bfloat16>::widen(*(const uint4*)(m + Shape::models), y);
#pragma unroll
          for (int e = 0; e < 8; ++e) model_dot = fmaf(x[e], y[e], model_dot);
        }
      }
      __syncthreads();
    }

    // F, E and beta E of the warp's 16 x 16 elements, and the sums of H over its rows and columns
    float row_p[2] = {}, row_a[2] = {}, col_h[2][2] = {};
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int e = 0; e < 4; e += 2) {
        const int i = row0 + g + 4 * e, j = wc * 16 + 8 * x + 2 * t;
        float F[2] = {}, E[2] = {};
        if (wc <= wr) {
          const float be = f->beta[i];
          const uint32_t p2 = P2[x][e / 2], l2 = L2[x][e / 2], k2 = K2[x][e / 2];
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const float d = exp2_fast((f->hi[i] - f->hi[j + y]) + (f->lo[i] - f->lo[j + y]));
            const float pp = y ? __uint_as_float(p2 & 0xffff0000u) + __uint_as_float(l2 & 0xffff0000u) : __uint_as_float(p2 << 16) + __uint_as_float(l2 << 16);
            const float kk = y ? __uint_as_float(k2 & 0xffff0000u) : __uint_as_float(k2 << 16);
            const bool below = j + y < i;
            F[y] = j + y <= i ? p.scale * d * dP[x][e + y] : 0.0f;
            E[y] = below ? -d * dA[x][e + y] : 0.0f;
            const float hp = below ? dP[x][e + y] * pp : 0.0f, ha = below ? -dA[x][e + y] * kk : 0.0f;
            row_p[e / 2] += hp;
            row_a[e / 2] += ha;
            col_h[x][y] += fmaf(be, ha, hp);
          }
        }
        const int to = (i * DC_TILE + j) * 2;
        *(uint32_t*)(Fs + to) = pack2(F[0], F[1]);
        *(uint32_t*)(Es + to) = pack2(E[0], E[1]);
        *(uint32_t*)(Bs + to) = pack2(f->beta[i] * E[0], f->beta[i] * E[1]);
      }
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        float v = col_h[x][y];
        v += __shfl_xor_sync(0xffffffffu, v, 4);
        v += __shfl_xor_sync(0xffffffffu, v, 8);
        v += __shfl_xor_sync(0xffffffffu, v, 16);
        if (g == 0) cols[wr * DC + wc * 16 + 8 * x + 2 * t + y] = v;
      }
    label_dot += __shfl_xor_sync(0xffffffffu, label_dot, 1);
    label_dot += __shfl_xor_sync(0xffffffffu, label_dot, 2);
    label_dot += __shfl_xor_sync(0xffffffffu, label_dot, 4);
    if (tid % 8 == 0) label_dots[tid / 8] = label_dot;
    model_dot = warp_sum(model_dot);
    if (lane == 0) model_dots[warp] = model_dot;
    __syncthreads();

    const int i0 = row0 + g, i1 = i0 + 8;
    const float c0 = f->c[i0], c1 = f->c[i1], r0 = f->r[i0], r1 = f->r[i1], be0 = f->beta[i0], be1 = f->beta[i1];
    // of rows i0 and i1: what passes from S and from H's rows, x.k, k.(r U G^T)
    float dots[3][2] = {{fmaf(be0, row_a[0], row_p[0]), fmaf(be1, row_a[1], row_p[1])}, {row_a[0], row_a[1]}, {0.0f, 0.0f}};
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
    const uint32_t k_mk = smem32(Ks) + lane_mk(lane, ROW) + colw * 2, q_mk = smem32(Qs) + lane_mk(lane, ROW) + colw * 2;
    const uint32_t f_mk = smem32(Fs) + lane_mk(lane, DC_TILE) + row0 * DC_TILE * 2, f_nk = smem32(Fs) + lane_nk(lane, DC_TILE) + row0 * 2;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      uint32_t a[4], e[4], b[4];
      if (x <= wr) {  // rows of F and E: dQ and x
        ldsm(a, f_mk + x * 32);
        ldsm(e, f_mk + DC_TILE_BYTES + x * 32);
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
        ldsm_t(a, f_nk + x * 16 * DC_TILE * 2);
        ldsm_t(e, f_nk + 2 * DC_TILE_BYTES + x * 16 * DC_TILE * 2);
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
#pragma unroll
    for (int x = 0; x < NT; ++x) {
      aX[x][0] = fmaf(be0, aX[x][0], aH[x][0]), aX[x][1] = fmaf(be0, aX[x][1], aH[x][1]);  // dK
      aX[x][2] = fmaf(be1, aX[x][2], aH[x][2]), aX[x][3] = fmaf(be1, aX[x][3], aH[x][3]);
    }
#pragma unroll
    for (int d = 0; d < 3; ++d)
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        float v = dots[d][z];
        v += __shfl_xor_sync(0xffffffffu, v, 1);
        v += __shfl_xor_sync(0xffffffffu, v, 2);
        if (t == 0) sums[(wc * DC + i0 + 8 * z) * 4 + d] = v;
      }
    // the heads of labels that share these features, added up by the thread that has the elements
    if (more > 1) {
#pragma unroll
      for (int x = 0; x < NT; ++x)
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
          float2* tq = (float2*)(totals + (i0 + 4 * e) * DK + colw + 8 * x + 2 * t);
          float2* tk = tq + DC * DK / 2;
          if (hh > 0) {
            const float2 q = *tq, k = *tk;
            aQ[x][e] += q.x, aQ[x][e + 1] += q.y, aX[x][e] += k.x, aX[x][e + 1] += k.y;
          }
          if (hh + 1 < more) {
            *tq = make_float2(aQ[x][e], aQ[x][e + 1]);
            *tk = make_float2(aX[x][e], aX[x][e + 1]);
          }
        }
    }
    if (hh + 1 == more) {
#pragma unroll
      for (int x = 0; x < NT; ++x)
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
          const int i = i0 + 4 * e, col = colw + 8 * x + 2 * t;
          if (i >= at.len) continue;
          const long long to = ((at.row0 + i) * p.hk + kh) * p.dk + col;
          if (gp.vec_dk) {
            if (col < p.dk) {
              *(uint32_t*)(gp.dq + to) = pack2(aQ[x][e], aQ[x][e + 1]);
              *(uint32_t*)(gp.dk + to) = pack2(aX[x][e], aX[x][e + 1]);
            }
          } else {
#pragma unroll
            for (int y = 0; y < 2; ++y)
              if (col + y < p.dk) {
                gp.dq[to + y] = __float2bfloat16_rn(aQ[x][e + y]);
                gp.dk[to + y] = __float2bfloat16_rn(aX[x][e + y]);
              }
          }
        }
    }
    __syncthreads();
    if (warp == 0) {  // two rows a lane: dbeta, and dg by a scan from the chunk's end
      float db[2], ahead = 0.0f;
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        const int i = 2 * lane + z;
        float v[3] = {0, 0, 0};
        for (int w = 0; w < 4; ++w)
#pragma unroll
          for (int d = 0; d < 3; ++d) v[d] += sums[(w * DC + i) * 4 + d];
        for (int w = i / 16; w < 4; ++w) v[0] -= cols[w * DC + i];
        db[z] = v[0] - v[2];
        ahead += v[2];
        if (i < at.len) gp.dbeta[(at.row0 + i) * p.hv + h] = __float2bfloat16_rn(label_dots[i] + v[1]);
      }
      const float decay = f->last * warp_sum(lane < ROWS_THREADS / 32 ? model_dots[lane] : 0.0f) + warp_sum(ahead);
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
    __syncthreads();
  }
}

}  // namespace wpsgd
