// C ABI of the operators that lay rows out by node and bring them back (see include/wpsgd.h). Argument checks, choice of forms, launches.
#include <algorithm>

#include "nodes.cuh"
#include "rows_host.cuh"

using namespace wpsgd;

namespace {

// The rows and places that all of these calls name
const char* check_places(const int32_t* where, int64_t n_rows, int32_t top) {
  if (n_rows < 0 || top < 1) return "negative row count, or less than one place a row";
  if (n_rows > INT32_MAX / top) return "2^31 places and more";
  if (n_rows > 0 && !where) return "positions are NULL";
  if ((uintptr_t)where % 4) return "positions are not aligned to their elements";
  return nullptr;
}
const char* check_rows(const void* p, wpsgd_xtype xt, int64_t ld, int64_t d, int64_t n) {
  if (!known(xt)) return "unknown type";
  if (d < 1 || ld < d || n < 0) return "rows need at least one column, a stride of at least d and no negative count";
  if (d > INT64_MAX / 8 / std::max<int64_t>(n, 1) || ld > INT64_MAX / 8 / std::max<int64_t>(n, 1)) return "rows that pass 63 bits";
  if (n > INT32_MAX || d > INT32_MAX / 8) return "2^31 rows and more, or rows of 2^31 bytes";
  if (n > 0 && !p) return "rows are NULL";
  if ((uintptr_t)p % element_size(xt)) return "rows are not aligned to their elements";
  return nullptr;
}
Region rows_region(const void* p, wpsgd_xtype xt, int64_t ld, int64_t d, int64_t n) {
  return {p, (long long)(d * element_size(xt)), (long long)(ld * element_size(xt)), n};
}
bool on16(const void* p, long long ld_bytes) { return aligned16(p) && ld_bytes % 16 == 0; }

// Threads of a row: four units of 16 bytes for each, or one where the rows are too few to fill the GPU that way
void choose_group(NodesParams* p) {
  const long long units = (p->width + 15) / 16;
  int lg = 2;
  while (lg < 8 && (4ll << lg) < units) ++lg;
  while (lg < 8 && (1ll << lg) < units && p->n_rows << lg < 148 * 1024) ++lg;
  p->lg = lg;
}
unsigned rows_grid(const NodesParams& p) { return (unsigned)grid_for(p.n_rows, NODES_THREADS >> p.lg, 1 << 20); }

#define NODES_LAUNCH(kernel, ...) launch(kernel<__VA_ARGS__>, rows_grid(p), NODES_THREADS, 0, c->stream, p)
#define NODES_LAUNCH_ANY(kernel, ...)                                                                                                                \
  (xt == WPSGD_X_F32 ? (aligned ? NODES_LAUNCH(kernel, float, true, ##__VA_ARGS__) : NODES_LAUNCH(kernel, float, false, ##__VA_ARGS__)) \
                     : (aligned ? NODES_LAUNCH(kernel, __nv_bfloat16, true, ##__VA_ARGS__) : NODES_LAUNCH(kernel, __nv_bfloat16, false, ##__VA_ARGS__)))
// by the places that are in registers at a time: as many as a row has, up to four
#define NODES_LAUNCH_PLACES(kernel) (top == 1 ? NODES_LAUNCH_ANY(kernel, 1) : top == 2 ? NODES_LAUNCH_ANY(kernel, 2) : NODES_LAUNCH_ANY(kernel, 4))

wpsgd_status refuse(wpsgd_ctx* c, const char* call, const char* why) { return fail(c, WPSGD_ERR_INVALID_ARG, std::string(call) + ": " + why); }

}  // namespace

extern "C" {

wpsgd_status wpsgd_sort_rows(wpsgd_ctx* c, const int32_t* node, int64_t n_rows, int32_t top, int32_t n_nodes, int32_t* where, int32_t* order, int64_t* shard_off) {
  if (!c) return fail(nullptr, WPSGD_ERR_INVALID_ARG, "ctx is NULL");
  if (const char* why = check_places(where, n_rows, top)) return refuse(c, "sort_rows", why);
  if (n_nodes < 1 || !shard_off || (n_rows > 0 && !node)) return refuse(c, "sort_rows", "NULL argument, or no nodes");
  if (((uintptr_t)node | (uintptr_t)order) % 4 || (uintptr_t)shard_off % 8) return refuse(c, "sort_rows", "an array is not aligned to its elements");
  if (n_nodes > SORT_MAX_NODES) return fail(c, WPSGD_ERR_UNSUPPORTED, "sort_rows: more than 16384 nodes");
  const long long places = n_rows * top;
  const size_t bytes = (size_t)places * 4, off_bytes = ((size_t)n_nodes + 1) * 8;
  if (overlap(where, bytes, node, bytes) || overlap(shard_off, off_bytes, node, bytes) || overlap(shard_off, off_bytes, where, bytes) ||
      (order && (overlap(order, bytes, node, bytes) || overlap(order, bytes, where, bytes) || overlap(shard_off, off_bytes, order, bytes))))
    return refuse(c, "sort_rows", "arrays overlap");
  DeviceGuard guard(c->device);
  SortParams p = {node, places, n_nodes, 0, 0, where, order, (long long*)shard_off, c->status};
  // Many places and blocks enough whose counts fit `order`: 131072 places on 128 nodes 30 us by a cluster of 8 blocks, 17 by the GPU. The scan over blocks is one
  // block's, so that there are fewer of them for more nodes.
  const long long many = std::min<long long>({148ll, 65536ll / n_nodes, places / 2 / n_nodes, (places + 2047) / 2048});
  if (order && places >= 32768 && many >= 12) {
    p.warps = (int)std::min<long long>(32, SORT_COUNTERS / n_nodes);
    p.run = ((places + many * p.warps - 1) / (many * p.warps) + 31) / 32 * 32;
    const size_t smem = ((size_t)n_nodes * (p.warps + 1)) * 4;
    CU_TRY(c, (allow_smem<sort_count_kernel>(c)));
    CU_TRY(c, (allow_smem<sort_place_kernel>(c)));
    CU_TRY(c, launch(sort_count_kernel, (unsigned)many, SORT_THREADS, smem, c->stream, p));
    CU_TRY(c, launch(sort_scan_kernel, 1, SORT_THREADS, 0, c->stream, p, (int)many));
    CU_TRY(c, launch(sort_place_kernel, (unsigned)many, SORT_THREADS, smem, c->stream, p));
    CU_TRY(c, launch(sort_order_kernel, (unsigned)grid_for(places, 256), 256, 0, c->stream, p));
    c->launches += 4;
    return WPSGD_OK;
  }
  // blocks: a run of 128 places for each warp before another block is worth its exchange
  const unsigned blocks = places <= 4096 ? 1 : places <= 8192 ? 2 : places <= 16384 ? 4 : 8;
  p.warps = (int)std::max(1ll, std::min<long long>({32ll, (long long)SORT_COUNTERS / n_nodes, (places + 32 * blocks - 1) / (32 * blocks)}));
  p.run = ((places + (long long)blocks * p.warps - 1) / ((long long)blocks * p.warps) + 31) / 32 * 32;
  CU_TRY(c, (allow_smem<sort_rows_kernel>(c)));
  CU_TRY(c, launch_clusters(sort_rows_kernel, blocks, SORT_THREADS, ((size_t)n_nodes * (p.warps + 1)) * 4, c->stream, blocks, p));
  c->launches++;
  return WPSGD_OK;
}

wpsgd_status wpsgd_gather_rows(wpsgd_ctx* c, const void* X, wpsgd_xtype xt, int64_t ld_x, int64_t d, const int32_t* where, int64_t n_rows, int32_t top, void* out, int64_t ld_out,
                               int64_t n_sorted) {
  if (!c) return fail(nullptr, WPSGD_ERR_INVALID_ARG, "ctx is NULL");
  if (const char* why = check_places(where, n_rows, top)) return refuse(c, "gather_rows", why);
  if (const char* why = check_rows(X, xt, ld_x, d, n_rows)) return refuse(c, "gather_rows", why);
  if (const char* why = check_rows(out, xt, ld_out, d, n_sorted)) return refuse(c, "gather_rows", why);
  const Region to = rows_region(out, xt, ld_out, d, n_sorted);
  if (meet(to, rows_region(X, xt, ld_x, d, n_rows)) || meet(to, {where, n_rows * top * 4ll, n_rows * top * 4ll, n_rows > 0})) return refuse(c, "gather_rows", "out overlaps X or the positions");
  if (n_rows == 0) return WPSGD_OK;
  DeviceGuard guard(c->device);
  const long long es = (long long)element_size(xt);
  NodesParams p = {where, nullptr, n_rows, n_sorted, top, 0, (int)(d * es), (const char*)X, ld_x * es, nullptr, 0, (char*)out, ld_out * es, nullptr, c->status};
  choose_group(&p);
  const bool aligned = p.width % 16 == 0 && on16(X, p.ld_rows) && on16(out, p.ld_out);
  CU_TRY(c, NODES_LAUNCH_ANY(gather_rows_kernel));
  c->launches++;
  return WPSGD_OK;
}

wpsgd_status wpsgd_combine_rows(wpsgd_ctx* c, const void* Y, wpsgd_xtype xt, int64_t ld_y, int64_t d, int64_t n_sorted, const int32_t* where, const float* weights, int64_t n_rows,
                                int32_t top, void* out, int64_t ld_out) {
  if (!c) return fail(nullptr, WPSGD_ERR_INVALID_ARG, "ctx is NULL");
  if (const char* why = check_places(where, n_rows, top)) return refuse(c, "combine_rows", why);
  if (const char* why = check_rows(Y, xt, ld_y, d, n_sorted)) return refuse(c, "combine_rows", why);
  if (const char* why = check_rows(out, xt, ld_out, d, n_rows)) return refuse(c, "combine_rows", why);
  if ((uintptr_t)weights % 4) return refuse(c, "combine_rows", "weights are not aligned to their elements");
  const Region to = rows_region(out, xt, ld_out, d, n_rows);
  const long long places = n_rows * top * 4ll;
  if (meet(to, rows_region(Y, xt, ld_y, d, n_sorted)) || meet(to, {where, places, places, n_rows > 0}) || (weights && meet(to, {weights, places, places, n_rows > 0})))
    return refuse(c, "combine_rows", "out overlaps Y, the positions or the weights");
  if (n_rows == 0) return WPSGD_OK;
  DeviceGuard guard(c->device);
  const long long es = (long long)element_size(xt);
  NodesParams p = {where, weights, n_rows, n_sorted, top, 0, (int)(d * es), nullptr, 0, (const char*)Y, ld_y * es, (char*)out, ld_out * es, nullptr, c->status};
  choose_group(&p);
  const bool aligned = p.width % 16 == 0 && on16(Y, p.ld_sorted) && on16(out, p.ld_out);
  CU_TRY(c, NODES_LAUNCH_PLACES(combine_rows_kernel));
  c->launches++;
  return WPSGD_OK;
}

wpsgd_status wpsgd_combine_rows_grad(wpsgd_ctx* c, const void* dout, int64_t ld_dout, const void* Y, int64_t ld_y, wpsgd_xtype xt, int64_t d, int64_t n_sorted, const int32_t* where,
                                     const float* weights, int64_t n_rows, int32_t top, void* dY, int64_t ld_dy, float* dweights) {
  if (!c) return fail(nullptr, WPSGD_ERR_INVALID_ARG, "ctx is NULL");
  if (const char* why = check_places(where, n_rows, top)) return refuse(c, "combine_rows_grad", why);
  if (const char* why = check_rows(dout, xt, ld_dout, d, n_rows)) return refuse(c, "combine_rows_grad", why);
  if (const char* why = check_rows(Y, xt, ld_y, d, n_sorted)) return refuse(c, "combine_rows_grad", why);
  if (const char* why = check_rows(dY, xt, ld_dy, d, n_sorted)) return refuse(c, "combine_rows_grad", why);
  if (((uintptr_t)weights | (uintptr_t)dweights) % 4) return refuse(c, "combine_rows_grad", "weights or their gradient are not aligned to their elements");
  const long long places = n_rows * top * 4ll;
  const Region to = rows_region(dY, xt, ld_dy, d, n_sorted), in_rows = rows_region(dout, xt, ld_dout, d, n_rows), in_sorted = rows_region(Y, xt, ld_y, d, n_sorted),
               in_where = {where, places, places, n_rows > 0}, in_weights = {weights, places, places, weights ? n_rows > 0 : 0}, to_weights = {dweights, places, places, dweights ? n_rows > 0 : 0};
  for (const Region& a : {to, to_weights})
    if (meet(a, in_rows) || meet(a, in_sorted) || meet(a, in_where) || meet(a, in_weights)) return refuse(c, "combine_rows_grad", "an output overlaps an input");
  if (meet(to, to_weights)) return refuse(c, "combine_rows_grad", "outputs overlap");
  if (n_rows == 0) return WPSGD_OK;
  DeviceGuard guard(c->device);
  const long long es = (long long)element_size(xt);
  NodesParams p = {where, weights, n_rows, n_sorted, top, 0, (int)(d * es), (const char*)dout, ld_dout * es, (const char*)Y, ld_y * es, (char*)dY, ld_dy * es, dweights, c->status};
  choose_group(&p);
  const bool aligned = p.width % 16 == 0 && on16(dout, p.ld_rows) && on16(Y, p.ld_sorted) && on16(dY, p.ld_out);
  // a warp to a row where the rows fill the GPU that way: its sums need no barrier of the block (65536 bf16 rows of 4096 columns: 516 -> 435 us)
  if (n_rows >= 148 * 32) p.lg = std::min(p.lg, 5);
  CU_TRY(c, NODES_LAUNCH_PLACES(combine_grad_kernel));
  c->launches++;
  return WPSGD_OK;
}

wpsgd_status wpsgd_clear_rows(wpsgd_ctx* c, const int32_t* where, int64_t n_rows, int32_t top, void* out, wpsgd_xtype xt, int64_t ld_out, int64_t d, int64_t n_sorted, uint32_t* marks) {
  if (!c) return fail(nullptr, WPSGD_ERR_INVALID_ARG, "ctx is NULL");
  if (const char* why = check_places(where, n_rows, top)) return refuse(c, "clear_rows", why);
  if (const char* why = check_rows(out, xt, ld_out, d, n_sorted)) return refuse(c, "clear_rows", why);
  if ((n_sorted > 0 && !marks) || (uintptr_t)marks % 4) return refuse(c, "clear_rows", "marks are NULL or not aligned to their elements");
  const long long es = (long long)element_size(xt), words = (n_sorted + 31) / 32 * 4, places = n_rows * top * 4ll;
  const Region to = rows_region(out, xt, ld_out, d, n_sorted), bits = {marks, words, words, 1}, in = {where, places, places, 1};
  if (meet(to, bits) || meet(to, in) || meet(bits, in)) return refuse(c, "clear_rows", "arrays overlap");
  if (n_sorted == 0) return WPSGD_OK;
  DeviceGuard guard(c->device);
  // Few bytes: all of them in one launch. 16 MB take as long as the three launches do.
  if (n_sorted * d * es <= 16 << 20 && ld_out * es <= INT32_MAX) {
    CU_TRY(c, cudaMemset2DAsync(out, ld_out * es, 0, d * es, n_sorted, c->stream));
    return WPSGD_OK;
  }
  const ClearParams p = {where, n_rows * top, n_sorted, marks, (char*)out, ld_out * es, (int)(d * es), (int)es};
  CU_TRY(c, cudaMemsetAsync(marks, 0, words, c->stream));
  CU_TRY(c, launch(mark_places_kernel, (unsigned)grid_for(std::max(p.places, 1ll), 256), 256, 0, c->stream, p));
  CU_TRY(c, launch(clear_rows_kernel, (unsigned)grid_for((n_sorted + 31) / 32, 8), 256, 0, c->stream, p));
  c->launches += 2;
  return WPSGD_OK;
}

}  // extern "C"
