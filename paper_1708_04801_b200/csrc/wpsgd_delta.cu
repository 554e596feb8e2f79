// C ABI of the chains whose labels are vectors (see include/wpsgd.h). Argument checks, workspaces, choice of kernels, launches.
#include <algorithm>
#include <cmath>

#include "delta_chunk.cuh"
#include "delta_grad.cuh"
#include "delta_rows.cuh"
#include "delta_walk.cuh"
#include "rows_host.cuh"

using namespace wpsgd;

namespace {

// The sizes, strides and types that every call takes; pointers are checked where they are followed
const char* check_shape(const wpsgd_delta_rows* r) {
  if (!r) return "rows are NULL";
  if (!known(r->type)) return "unknown type";
  if (r->n_rows < 0 || r->n_chains < 0 || r->heads_k < 1 || r->heads_v < 1 || r->dk < 1 || r->dv < 1) return "negative count, or no heads, features or labels";
  if (r->heads_v % r->heads_k) return "heads_v is not a multiple of heads_k";
  return nullptr;
}
const char* check_limits(const wpsgd_delta_rows* r) {
  if (r->dk > DELTA_MAX_D || r->dv > DELTA_MAX_D) return "more than 128 features or labels a head";
  if (r->heads_v > 65536 || r->n_rows > INT32_MAX || (r->n_rows / 64 + r->n_chains + 1) * r->heads_v > INT32_MAX / 16 || (long long)r->n_chains * r->heads_v * r->dv > INT32_MAX)
    return "too many rows, chains or heads";
  return nullptr;
}
const char* check_delta_rows(const wpsgd_delta_rows* r, bool chains) {
  if (!std::isfinite(r->scale)) return "scale is not finite";
  const long long wk = (long long)r->heads_k * r->dk, wv = (long long)r->heads_v * r->dv;
  if (r->ld_q < wk || r->ld_k < wk || r->ld_v < wv || r->ld_g < r->heads_v || r->ld_beta < r->heads_v) return "a stride is below the width of a row";
  for (const int64_t ld : {r->ld_q, r->ld_k, r->ld_v, r->ld_g, r->ld_beta})
    if (ld > INT64_MAX / 8 / std::max<int64_t>(r->n_rows, 1)) return "rows that pass 63 bits";
  if (r->n_rows > 0 && (!r->q || !r->k || !r->v || !r->g || !r->beta)) return "rows are NULL";
  const size_t es = element_size(r->type);
  if (((uintptr_t)r->q | (uintptr_t)r->k | (uintptr_t)r->v | (uintptr_t)r->g | (uintptr_t)r->beta) % es) return "rows are not aligned to their elements";
  if (chains && (!r->shard_off || (uintptr_t)r->shard_off % 8)) return "shard_off is NULL or not aligned to its elements";
  return nullptr;
}
// Whether `out` shares memory with any input of the rows
bool meets_rows(const Region& out, const wpsgd_delta_rows* r, bool chains) {
  const long long es = (long long)element_size(r->type), wk = r->heads_k * r->dk * es, wv = r->heads_v * r->dv * es, wh = r->heads_v * es, n = r->n_rows;
  return meet(out, {r->q, wk, r->ld_q * es, n}) || meet(out, {r->k, wk, r->ld_k * es, n}) || meet(out, {r->v, wv, r->ld_v * es, n}) || meet(out, {r->g, wh, r->ld_g * es, n}) ||
         meet(out, {r->beta, wh, r->ld_beta * es, n}) || (chains && meet(out, {r->shard_off, (r->n_chains + 1ll) * 8, (r->n_chains + 1ll) * 8, 1}));
}
Region block_of(const void* p, long long bytes) { return {p, bytes, bytes, p ? 1 : 0}; }
long long model_bytes(const wpsgd_delta_rows* r, long long n) { return n * r->heads_v * r->dv * r->dk * 4; }

wpsgd_status refuse(wpsgd_ctx* c, const char* call, const char* why, wpsgd_status s = WPSGD_ERR_INVALID_ARG) { return fail(c, s, std::string(call) + ": " + why); }

DeltaRowsParams rows_params(const wpsgd_ctx* c, const wpsgd_delta_rows* r, void* out, long long ld_out, const float* W0, float* W) {
  const size_t es = element_size(r->type), unit = 4 * es;
  const bool vec = r->dk % 4 == 0 && ((uintptr_t)r->q | (uintptr_t)r->k) % unit == 0 && (r->ld_q | r->ld_k) % 4 == 0 && aligned16(W0) && aligned16(W);
  return {r->q, r->k, r->v, r->g, r->beta, r->ld_q, r->ld_k, r->ld_v, r->ld_g, r->ld_beta, ld_out, out, W0, W, r->n_rows, (const long long*)r->shard_off, r->n_chains, nullptr, 0,
          r->heads_k, r->heads_v, r->dk, r->dv, r->scale, vec, 0, c->status};
}

wpsgd_status run_rows(wpsgd_ctx* c, const DeltaRowsParams& p) {
  const unsigned grid = (unsigned)(p.n_chains * ((p.hv * p.dv + ROWS_MODELS - 1) / ROWS_MODELS));
  auto go = [&](auto nj) {
    constexpr int NJ = decltype(nj)::value;
    const int row_bytes = rows_floats<NJ>(rows_heads(p.hk, p.hv, p.dv)) * 4, batch = std::max(1, std::min(ROWS_BATCH, 48 * 1024 / row_bytes));
    CU_TRY(c, (allow_smem<delta_rows_kernel<NJ>>(c)));
    CU_TRY(c, launch(delta_rows_kernel<NJ>, grid, 32 * DELTA_WARPS, (size_t)2 * batch * row_bytes, c->stream, p, batch));
    c->launches++;
    return WPSGD_OK;
  };
  return p.dk <= 32 ? go(std::integral_constant<int, 1>()) : p.dk <= 64 ? go(std::integral_constant<int, 2>()) : go(std::integral_constant<int, 4>());
}

// Rows by slots: from how many on a block has a run of them, so that the slots before it are looked through once and not in each block, and how many such blocks. By a block for each
// row and by runs, us (bf16, 16 x 16; fp32, 4 heads of 32 x 32; bf16, 128 x 128): 8192 rows 37 and 43, 136 and 115, 211 and 186; 16384 85 and 80, 331 and 221, 469 and 367; 131072 2725 and
// 529, 10640 and 1700. (Without slots 131072 rows take 313 and 1452; runs for 2, 4 or 8 blocks an SM: 760, 680 and 738 for 16 x 16.) Their time still has a part that grows with the square
// of the rows, n^2 / 4096 slots of 4 bytes where runs are of 2048: the most rows keep it at a few ms.
constexpr long long STEP_RUNS_FROM = 4096, STEP_BLOCKS = 148 * 6, STEP_MAX_ROWS = 1 << 22;
template <typename XT>
wpsgd_status run_step(wpsgd_ctx* c, const DeltaRowsParams& p) {
  const long long models = (long long)p.hv * p.dv, grid = p.n_rows * ((models + 31) / 32);
  if (grid > INT32_MAX) return fail(c, WPSGD_ERR_UNSUPPORTED, "delta_step: too many models");
  const int step_runs = p.slots && p.n_rows > STEP_RUNS_FROM;
  auto go = [&](auto nj) {
    constexpr int NJ = decltype(nj)::value;
    if (!step_runs) return launch(delta_step_kernel<XT, NJ>, (unsigned)grid, STEP_THREADS, 0, c->stream, p);
    const int run = (int)std::min<long long>(STEP_RUN, (p.n_rows + STEP_BLOCKS - 1) / STEP_BLOCKS);
    int lg = 6;
    while (1 << lg < 2 * run) ++lg;
    return launch(delta_step_runs_kernel<XT, NJ>, (unsigned)((p.n_rows + run - 1) / run), STEP_THREADS, ((size_t)(2 << lg) + run) * 4, c->stream, p, run, lg);
  };
  CU_TRY(c, p.dk <= 32 ? go(std::integral_constant<int, 1>()) : p.dk <= 64 ? go(std::integral_constant<int, 2>()) : go(std::integral_constant<int, 4>()));
  c->launches++;
  return WPSGD_OK;
}

// ---- chunks ------------------------------------------------------------------------------------------------------------------
// Where a workspace has what. Heads are laid out anew where the tensor-core kernels cannot take them as they are.
struct DeltaLayout {
  long long chunks;  // at most: the offsets are known on the device only
  int DK, dvp, dk8, dv8;
  bool pack_k, pack_v, kept;
  size_t chunk_off, order, table, q, k, v, blocks, starts, steps, gram, total;
  DeltaLayout(const wpsgd_delta_rows* r, bool save) {
    auto fits = [](const void* p, int64_t ld, int width) { return width % 8 == 0 && aligned16(p) && ld % 8 == 0; };
    chunks = r->n_rows / DC + r->n_chains;
    DK = r->dk <= 64 ? 64 : 128;
    dvp = (r->dv + 15) / 16 * 16;
    dk8 = (r->dk + 7) / 8 * 8;
    dv8 = (r->dv + 7) / 8 * 8;
    pack_k = !fits(r->q, r->ld_q, r->dk) || !fits(r->k, r->ld_k, r->dk);
    pack_v = !fits(r->v, r->ld_v, r->dv);
    size_t at = 0;
    auto take = [&](size_t bytes) {
      const size_t here = at;
      at = (at + bytes + 255) / 256 * 256;
      return here;
    };
    chunk_off = take(((size_t)r->n_chains + 1) * 4);
    order = take((size_t)r->n_chains * 4);
    table = take((size_t)chunks * sizeof(DeltaChunk));
    q = take(pack_k ? (size_t)r->n_rows * r->heads_k * dk8 * 2 : 0);
    k = take(pack_k ? (size_t)r->n_rows * r->heads_k * dk8 * 2 : 0);
    v = take(pack_v ? (size_t)r->n_rows * r->heads_v * dv8 * 2 : 0);
    blocks = take((size_t)chunks * r->heads_v * DC_BLOCK);
    starts = take(save ? (size_t)chunks * r->heads_v * dvp * DK * 2 : 0);
    steps = take(save ? (size_t)chunks * r->heads_v * DC * dvp * 2 : 0);
    gram = take(save ? (size_t)chunks * r->heads_v * DC_TRI : 0);
    total = at;
    kept = save;
  }
};

DeltaChunkParams chunk_params(const wpsgd_ctx* c, const wpsgd_delta_rows* r, const DeltaLayout& lay, unsigned char* ws) {
  using bf16 = const __nv_bfloat16;
  DeltaChunkParams p = {};
  p.shard_off = (const long long*)r->shard_off;
  p.n_rows = r->n_rows;
  p.n_chains = r->n_chains, p.hk = r->heads_k, p.hv = r->heads_v, p.dk = r->dk, p.dv = r->dv, p.dvp = lay.dvp;
  p.q = lay.pack_k ? DeltaHeads{(bf16*)(ws + lay.q), (long long)r->heads_k * lay.dk8, r->heads_k, lay.dk8} : DeltaHeads{(bf16*)r->q, r->ld_q, r->heads_k, r->dk};
  p.k = lay.pack_k ? DeltaHeads{(bf16*)(ws + lay.k), (long long)r->heads_k * lay.dk8, r->heads_k, lay.dk8} : DeltaHeads{(bf16*)r->k, r->ld_k, r->heads_k, r->dk};
  p.v = lay.pack_v ? DeltaHeads{(bf16*)(ws + lay.v), (long long)r->heads_v * lay.dv8, r->heads_v, lay.dv8} : DeltaHeads{(bf16*)r->v, r->ld_v, r->heads_v, r->dv};
  p.g = (bf16*)r->g, p.beta = (bf16*)r->beta, p.ld_g = r->ld_g, p.ld_beta = r->ld_beta;
  p.scale = r->scale;
  p.chunk_off = (int*)(ws + lay.chunk_off);
  p.order = (int*)(ws + lay.order);
  p.chunks = (DeltaChunk*)(ws + lay.table);
  p.blocks = ws + lay.blocks;
  p.starts = (__nv_bfloat16*)(ws + lay.starts);
  p.steps = (__nv_bfloat16*)(ws + lay.steps);
  p.gram = lay.kept ? ws + lay.gram : nullptr;
  p.spin_limit = c->opt_spin_limit, p.drop = c->opt_drop_block;
  p.status = c->status;
  return p;
}

struct Packs {
  DeltaPack p = {};
  int n = 0;
  long long most = 0;  // units of the largest
  void add(const void* from, long long ld, int heads, int width, const __nv_bfloat16* to) {
    p.t[n++] = {(const __nv_bfloat16*)from, ld, (__nv_bfloat16*)to, heads, width};
    most = std::max(most, (long long)heads * ((width + 7) / 8));
  }
  wpsgd_status launch_for(wpsgd_ctx* c, const DeltaChunkParams& plan) {  // behind the plan's kernel
    if (n == 0 || plan.n_rows == 0) return WPSGD_OK;
    p.chunk_off = plan.chunk_off, p.chunks = plan.chunks, p.n_chains = plan.n_chains;
    CU_TRY(c, launch(delta_pack_kernel, dim3(grid_for(plan.n_rows * most, 256), n), 256, 0, c->stream, p));
    c->launches++;
    return WPSGD_OK;
  }
};

// Tensor maps of features and queries for the walks, 64 rows by 64 columns at a time; false: whole heads do not fill such tiles, or sizes that a map cannot describe
bool encode_maps(DeltaMaps* maps, const DeltaChunkParams& p) {
  if ((p.k.width != 64 && p.k.width != 128) || p.n_rows < DC || !tensor_map_encoder()) return false;
  auto encode = [&](CUtensorMap* map, const DeltaHeads& h) {
    const cuuint64_t dims[2] = {(cuuint64_t)h.heads * h.width, (cuuint64_t)p.n_rows}, strides[1] = {(cuuint64_t)h.ld * 2};
    const cuuint32_t box[2] = {64, DC}, steps[2] = {1, 1};
    return tensor_map_encoder()(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, (void*)h.p, dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                                CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
  };
  return encode(&maps->k, p.k) && encode(&maps->q, p.q);
}

// Warps (of 16 labels) of a block that walks a chain: as many as leave every SM a block, so that few blocks bring the same rows
int chain_warps(long long heads, int dvp) {
  int w = 8;
  while (w > 1 && (w / 2 >= dvp / 16 || heads * ((dvp / 16 + w - 1) / w) < 148)) w /= 2;
  return w;
}

template <int DK, int NW>
wpsgd_status walk(wpsgd_ctx* c, const DeltaChunkParams& p, const DeltaMaps& maps, bool save) {
  using Shape = ChainShape<DK, NW>;
  const unsigned grid = (unsigned)((long long)p.n_chains * p.hv * p.slices);
  if (save) {
    CU_TRY(c, (allow_smem<delta_chain_kernel<DK, NW, true>>(c)));
    CU_TRY(c, launch(delta_chain_kernel<DK, NW, true>, grid, Shape::threads, Shape::smem, c->stream, p, maps));
  } else {
    CU_TRY(c, (allow_smem<delta_chain_kernel<DK, NW, false>>(c)));
    CU_TRY(c, launch(delta_chain_kernel<DK, NW, false>, grid, Shape::threads, Shape::smem, c->stream, p, maps));
  }
  c->launches++;
  return WPSGD_OK;
}

// Labels from which on a head walks by tcgen05, whose products have 128 of them whatever there are; fewer are at most four warps of mma.sync. By mma.sync and by tcgen05, us: 16384 rows,
// 32 chains, 16 heads of 64 features and 32 labels 81 and 88, 64 x 64 87 and 91, 128 x 64 110 and 109, 64 x 128 144 and 97, 128 x 96 197 and 116, 128 x 128 205 and 127; one chain of 8192
// rows, 2 heads of 128 x 128 358 and 334. (Not by the number of chains: what a chain gives does not depend on the others. 4 chunks of 15 chains and heads of 128 x 128: 20 and 25.)
constexpr int WALK_MIN = 65;
template <int DK>
wpsgd_status walk_tmem(wpsgd_ctx* c, const DeltaChunkParams& p, const DeltaMaps& maps, bool save) {
  constexpr int smem = ChainShape<DK, 8>::smem;
  const unsigned grid = (unsigned)((long long)p.n_chains * p.hv);
  if (save) {
    CU_TRY(c, (allow_smem<delta_walk_kernel<DK, true>>(c)));
    CU_TRY(c, launch(delta_walk_kernel<DK, true>, grid, WALK_THREADS, smem, c->stream, p, maps));
  } else {
    CU_TRY(c, (allow_smem<delta_walk_kernel<DK, false>>(c)));
    CU_TRY(c, launch(delta_walk_kernel<DK, false>, grid, WALK_THREADS, smem, c->stream, p, maps));
  }
  c->launches++;
  return WPSGD_OK;
}

template <int DK>
wpsgd_status run_chunks(wpsgd_ctx* c, DeltaChunkParams p, const DeltaLayout& lay, bool save, Packs& packs) {
  CU_TRY(c, launch(delta_plan_kernel, 1, PLAN_THREADS, 0, c->stream, p));
  c->launches++;
  if (const wpsgd_status s = packs.launch_for(c, p)) return s;
  if (lay.chunks > 0) {
    CU_TRY(c, (allow_smem<delta_prepare_kernel<DK>>(c)));
    // heads that share features by one block where that leaves every SM eight: their products of features are formed once
    p.prep_heads = 1;
    for (int n = 2; n <= PREP_HEADS && lay.chunks * p.hv / n >= 148 * 8; ++n)
      if (p.hv / p.hk % n == 0) p.prep_heads = n;
    const long long blocks = lay.chunks + p.new_out;  // those of no chunk clear what is outside the chains; one at least
    CU_TRY(c, launch(delta_prepare_kernel<DK>, (unsigned)(blocks * (p.hv / p.prep_heads)), PREP_THREADS, PrepShape<DK>::smem, c->stream, p));
    c->launches++;
  }
  DeltaMaps maps = {};
  p.maps = encode_maps(&maps, p);
  if (p.dvp >= WALK_MIN) return walk_tmem<DK>(c, p, maps, save);
  const int w = chain_warps((long long)p.n_chains * p.hv, p.dvp);
  p.slices = (p.dvp / 16 + w - 1) / w;
  return w == 4 ? walk<DK, 4>(c, p, maps, save) : w == 2 ? walk<DK, 2>(c, p, maps, save) : walk<DK, 1>(c, p, maps, save);
}

// Blocks that go through the chunks' rows: one per SM
int rows_blocks(const wpsgd_delta_rows* r, const DeltaLayout& lay) { return (int)std::min<long long>(lay.chunks * r->heads_k, 148); }

// The gradient's own workspace
struct DeltaGradLayout {
  bool pack_o;
  size_t dout, ends, drs, totals, total;
  DeltaGradLayout(const wpsgd_delta_rows* r, const DeltaLayout& lay, const void* p, int64_t ld) {
    pack_o = r->dv % 8 != 0 || !aligned16(p) || ld % 8 != 0;
    auto up = [](size_t n) { return (n + 255) / 256 * 256; };
    dout = 0;
    ends = up((size_t)r->n_rows * r->heads_v * lay.dv8 * 2);  // kept free also where the rows of dout are taken as they are: the size goes by `rows` alone
    drs = ends + up((size_t)lay.chunks * r->heads_v * lay.dvp * lay.DK * 2);
    totals = drs + up((size_t)lay.chunks * r->heads_v * DC * lay.dvp * 2);
    total = totals + (r->heads_v > r->heads_k ? (size_t)rows_blocks(r, lay) * 2 * DC * lay.DK * 4 : 0);
  }
};

template <int DK, int NW>
wpsgd_status walk_back(wpsgd_ctx* c, const DeltaGradParams& p, const DeltaMaps& maps) {
  using Shape = ChainShape<DK, NW>;
  CU_TRY(c, (allow_smem<delta_back_kernel<DK, NW>>(c)));
  CU_TRY(c, launch(delta_back_kernel<DK, NW>, (unsigned)((long long)p.f.n_chains * p.f.hv * p.f.slices), Shape::threads, Shape::smem, c->stream, p, maps));
  c->launches++;
  return WPSGD_OK;
}

template <int DK>
wpsgd_status grad_chunks(wpsgd_ctx* c, DeltaGradParams p, const DeltaLayout& lay, int blocks) {
  const int w = chain_warps((long long)p.f.n_chains * p.f.hv, p.f.dvp);
  p.f.slices = (p.f.dvp / 16 + w - 1) / w;
  DeltaMaps maps = {};
  p.f.maps = encode_maps(&maps, p.f);
  const wpsgd_status s = w == 8 ? walk_back<DK, 8>(c, p, maps) : w == 4 ? walk_back<DK, 4>(c, p, maps) : w == 2 ? walk_back<DK, 2>(c, p, maps) : walk_back<DK, 1>(c, p, maps);
  if (s != WPSGD_OK || lay.chunks == 0) return s;
  CU_TRY(c, (allow_smem<delta_rowgrad_kernel<DK>>(c)));
  CU_TRY(c, launch(delta_rowgrad_kernel<DK>, (unsigned)blocks, ROWS_THREADS, RowsShape<DK>::smem, c->stream, p));
  c->launches++;
  return WPSGD_OK;
}

}  // namespace

extern "C" {

wpsgd_status wpsgd_delta_workspace(const wpsgd_delta_rows* rows, wpsgd_delta_use use, int64_t* bytes) {
  if (!bytes) return refuse(nullptr, "delta_workspace", "bytes is NULL");
  *bytes = 0;
  if (const char* why = check_shape(rows)) return refuse(nullptr, "delta_workspace", why);
  if (const char* why = check_limits(rows)) return refuse(nullptr, "delta_workspace", why, WPSGD_ERR_UNSUPPORTED);
  if ((int)use < 0 || (int)use > 2) return refuse(nullptr, "delta_workspace", "unknown use");
  if (use != WPSGD_DELTA_RUN && rows->type != WPSGD_X_BF16) return refuse(nullptr, "delta_workspace", "gradients are of bf16 rows", WPSGD_ERR_UNSUPPORTED);
  if (rows->type != WPSGD_X_BF16) return WPSGD_OK;
  const DeltaLayout lay(rows, use != WPSGD_DELTA_RUN);
  *bytes = (int64_t)(use == WPSGD_DELTA_GRAD ? DeltaGradLayout(rows, lay, nullptr, 0).total : lay.total);
  return WPSGD_OK;
}

wpsgd_status wpsgd_delta_run(wpsgd_ctx* c, const wpsgd_delta_rows* rows, const float* W0, float* W_out, void* out, int64_t ld_out, wpsgd_delta_use use, void* workspace,
                             int64_t workspace_bytes) {
  if (!c) return fail(nullptr, WPSGD_ERR_INVALID_ARG, "ctx is NULL");
  if (const char* why = check_shape(rows)) return refuse(c, "delta_run", why);
  if (const char* why = check_limits(rows)) return refuse(c, "delta_run", why, WPSGD_ERR_UNSUPPORTED);
  if (const char* why = check_delta_rows(rows, true)) return refuse(c, "delta_run", why);
  const long long es = (long long)element_size(rows->type), wv = (long long)rows->heads_v * rows->dv;
  if (ld_out < wv || ld_out > INT64_MAX / 8 / std::max<int64_t>(rows->n_rows, 1) || (rows->n_rows > 0 && !out) || (uintptr_t)out % es) return refuse(c, "delta_run", "out is NULL, not aligned to its elements, or its stride is below the width of a row");
  if (((uintptr_t)W0 | (uintptr_t)W_out) % 4) return refuse(c, "delta_run", "models are not aligned to their elements");
  const Region to = {out, wv * es, ld_out * es, rows->n_rows}, from = block_of(W0, model_bytes(rows, rows->n_chains)), models = block_of(W_out, model_bytes(rows, rows->n_chains));
  if (meets_rows(to, rows, true) || meets_rows(models, rows, true) || meet(to, from) || meet(to, models) || (W0 != W_out && meet(from, models))) return refuse(c, "delta_run", "an output overlaps an input or another output");
  if ((int)use & ~(WPSGD_DELTA_RUN_SAVE | WPSGD_DELTA_NEW_OUT)) return refuse(c, "delta_run", "unknown use");
  const bool save = (int)use & WPSGD_DELTA_RUN_SAVE, new_out = (int)use & WPSGD_DELTA_NEW_OUT;
  if (save && rows->type != WPSGD_X_BF16) return refuse(c, "delta_run", "gradients are of bf16 rows", WPSGD_ERR_UNSUPPORTED);
  DeviceGuard guard(c->device);
  if (rows->n_chains == 0) {  // all rows are outside
    const bool whole = ld_out * es <= INT32_MAX;  // rows further apart than a copy of rows can be are cleared one by one
    if (new_out && rows->n_rows > 0 && whole) CU_TRY(c, cudaMemset2DAsync(out, ld_out * es, 0, wv * es, rows->n_rows, c->stream));
    for (int64_t i = 0; new_out && !whole && i < rows->n_rows; ++i) CU_TRY(c, cudaMemsetAsync((char*)out + i * ld_out * es, 0, wv * es, c->stream));
    return WPSGD_OK;
  }
  if (rows->type == WPSGD_X_F32) {
    DeltaRowsParams p = rows_params(c, rows, out, ld_out, W0, W_out);
    p.new_out = new_out;
    return run_rows(c, p);
  }
  const DeltaLayout lay(rows, save);
  if (!workspace || !aligned16(workspace) || workspace_bytes < (long long)lay.total) return refuse(c, "delta_run", "the workspace is NULL, not aligned to 16 bytes or too small");
  const Region ws = block_of(workspace, (long long)lay.total);
  if (meets_rows(ws, rows, true) || meet(ws, to) || meet(ws, from) || meet(ws, models)) return refuse(c, "delta_run", "the workspace overlaps an argument");
  DeltaChunkParams p = chunk_params(c, rows, lay, (unsigned char*)workspace);
  p.W0 = W0, p.W = W_out, p.out = (__nv_bfloat16*)out, p.ld_out = ld_out;
  p.vec_out = rows->dv % 8 == 0 && ld_out % 8 == 0 && aligned16(out);
  p.new_out = new_out;
  Packs packs;
  if (lay.pack_k) packs.add(rows->q, rows->ld_q, rows->heads_k, rows->dk, p.q.p);
  if (lay.pack_k) packs.add(rows->k, rows->ld_k, rows->heads_k, rows->dk, p.k.p);
  if (lay.pack_v) packs.add(rows->v, rows->ld_v, rows->heads_v, rows->dv, p.v.p);
  return lay.DK == 64 ? run_chunks<64>(c, p, lay, save, packs) : run_chunks<128>(c, p, lay, save, packs);
}

wpsgd_status wpsgd_delta_grad(wpsgd_ctx* c, const wpsgd_delta_rows* rows, const void* saved, int64_t saved_bytes, const void* dout, int64_t ld_dout, const float* dW, void* dq, void* dk,
                              void* dv, void* dg, void* dbeta, float* dW0, void* workspace, int64_t workspace_bytes) {
  if (!c) return fail(nullptr, WPSGD_ERR_INVALID_ARG, "ctx is NULL");
  if (const char* why = check_shape(rows)) return refuse(c, "delta_grad", why);
  if (const char* why = check_limits(rows)) return refuse(c, "delta_grad", why, WPSGD_ERR_UNSUPPORTED);
  if (rows->type != WPSGD_X_BF16) return refuse(c, "delta_grad", "gradients are of bf16 rows", WPSGD_ERR_UNSUPPORTED);
  if (const char* why = check_delta_rows(rows, true)) return refuse(c, "delta_grad", why);
  const long long n = rows->n_rows, wk = (long long)rows->heads_k * rows->dk * 2, wv = (long long)rows->heads_v * rows->dv * 2, wh = rows->heads_v * 2ll, models = model_bytes(rows, rows->n_chains);
  if (ld_dout < wv / 2 || ld_dout > INT64_MAX / 8 / std::max<long long>(n, 1) || (n > 0 && (!dout || !dq || !dk || !dv || !dg || !dbeta))) return refuse(c, "delta_grad", "NULL argument, or the stride of dout is below the width of a row");
  if (((uintptr_t)dout | (uintptr_t)dq | (uintptr_t)dk | (uintptr_t)dv | (uintptr_t)dg | (uintptr_t)dbeta) % 2 || ((uintptr_t)dW | (uintptr_t)dW0) % 4) return refuse(c, "delta_grad", "an argument is not aligned to its elements");
  if (rows->n_chains == 0) {  // all rows are outside
    DeviceGuard guard(c->device);
    if (n > 0)
      for (const auto& [p, bytes] : {std::pair<void*, long long>{dq, n * wk}, {dk, n * wk}, {dv, n * wv}, {dg, n * wh}, {dbeta, n * wh}}) CU_TRY(c, cudaMemsetAsync(p, 0, bytes, c->stream));
    return WPSGD_OK;
  }
  const DeltaLayout lay(rows, true);
  const DeltaGradLayout own(rows, lay, dout, ld_dout);
  if (!saved || !aligned16(saved) || saved_bytes < (long long)lay.total) return refuse(c, "delta_grad", "what the run saved is NULL, not aligned to 16 bytes or too small");
  if (!workspace || !aligned16(workspace) || workspace_bytes < (long long)own.total) return refuse(c, "delta_grad", "the workspace is NULL, not aligned to 16 bytes or too small");
  const Region from = {dout, wv, ld_dout * 2, n}, kept = block_of(saved, (long long)lay.total), before = block_of(dW, models);
  const Region to[7] = {block_of(dq, n * wk), block_of(dk, n * wk), block_of(dv, n * wv), block_of(dg, n * wh), block_of(dbeta, n * wh), block_of(dW0, models), block_of(workspace, (long long)own.total)};
  for (int i = 0; i < 7; ++i) {
    bool meets = meets_rows(to[i], rows, true) || meet(to[i], from) || meet(to[i], kept) || (!(i == 5 && dW0 == dW) && meet(to[i], before));
    for (int j = 0; j < i; ++j) meets = meets || meet(to[i], to[j]);
    if (meets) return refuse(c, "delta_grad", "an output or the workspace overlaps an input or another output");
  }
  DeviceGuard guard(c->device);
  unsigned char* ws = (unsigned char*)workspace;
  DeltaGradParams p = {chunk_params(c, rows, lay, (unsigned char*)saved), (__nv_bfloat16*)(ws + own.ends), (__nv_bfloat16*)(ws + own.drs), (float*)(ws + own.totals), dW, dW0, (__nv_bfloat16*)dq, (__nv_bfloat16*)dk,
                       (__nv_bfloat16*)dv, (__nv_bfloat16*)dg, (__nv_bfloat16*)dbeta, rows->dv % 8 == 0 && aligned16(dv), rows->dk % 2 == 0 && ((uintptr_t)dq | (uintptr_t)dk) % 4 == 0};
  p.f.dout = own.pack_o ? DeltaHeads{(const __nv_bfloat16*)(ws + own.dout), (long long)rows->heads_v * lay.dv8, rows->heads_v, lay.dv8}
                        : DeltaHeads{(const __nv_bfloat16*)dout, ld_dout, rows->heads_v, rows->dv};
  Packs packs;
  if (own.pack_o) packs.add(dout, ld_dout, rows->heads_v, rows->dv, p.f.dout.p);
  if (const wpsgd_status s = packs.launch_for(c, p.f)) return s;
  return lay.DK == 64 ? grad_chunks<64>(c, p, lay, rows_blocks(rows, lay)) : grad_chunks<128>(c, p, lay, rows_blocks(rows, lay));
}

wpsgd_status wpsgd_delta_step(wpsgd_ctx* c, const wpsgd_delta_rows* rows, float* W, const int32_t* slots, int64_t n_slots, void* out, int64_t ld_out) {
  if (!c) return fail(nullptr, WPSGD_ERR_INVALID_ARG, "ctx is NULL");
  wpsgd_delta_rows single;
  if (rows) {  // chains are not looked at: whatever stands there is not a reason to refuse
    single = *rows;
    single.n_chains = 0;
    single.shard_off = nullptr;
    rows = &single;
  }
  if (const char* why = check_shape(rows)) return refuse(c, "delta_step", why);
  if (const char* why = check_limits(rows)) return refuse(c, "delta_step", why, WPSGD_ERR_UNSUPPORTED);
  if (const char* why = check_delta_rows(rows, false)) return refuse(c, "delta_step", why);
  const long long es = (long long)element_size(rows->type), wv = (long long)rows->heads_v * rows->dv, per_slot = model_bytes(rows, 1);
  if (ld_out < wv || ld_out > INT64_MAX / 8 / std::max<int64_t>(rows->n_rows, 1) || (rows->n_rows > 0 && (!out || !W)) || (uintptr_t)out % es || (uintptr_t)W % 4 || (uintptr_t)slots % 4)
    return refuse(c, "delta_step", "NULL or misaligned argument, or a stride below the width of a row");
  if (n_slots < 0 || n_slots > INT64_MAX / 8 / per_slot) return refuse(c, "delta_step", "negative number of slots, or models that pass 63 bits");
  if (slots && rows->n_rows > STEP_MAX_ROWS) return refuse(c, "delta_step", "more than 4194304 rows by slots", WPSGD_ERR_UNSUPPORTED);
  if (!slots && n_slots < rows->n_rows) return refuse(c, "delta_step", "fewer models than rows, and no slots");
  const Region to = {out, wv * es, ld_out * es, rows->n_rows}, models = block_of(W, n_slots * per_slot), places = block_of(slots, rows->n_rows * 4);
  if (meets_rows(to, rows, false) || meets_rows(models, rows, false) || meet(to, models) || meet(to, places) || meet(models, places)) return refuse(c, "delta_step", "an output overlaps an input or another output");
  if (rows->n_rows == 0) return WPSGD_OK;
  DeviceGuard guard(c->device);
  DeltaRowsParams p = rows_params(c, rows, out, ld_out, nullptr, W);
  p.slots = slots;
  p.n_slots = n_slots;
  return rows->type == WPSGD_X_F32 ? run_step<float>(c, p) : run_step<__nv_bfloat16>(c, p);
}

}  // extern "C"
