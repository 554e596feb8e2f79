// C ABI of the operators on whole sets of rows (see include/wpsgd.h): 8-bit rows, margins of many models, the objective with its
// gradient, norm and clipping of gradients. Argument checks, workspaces, choice of kernels, launches.
#include <cmath>
#include <memory>
#include <new>
#include <type_traits>

#include "clip.cuh"
#include "context.cuh"
#include "gradient.cuh"
#include "margins.cuh"
#include "quantize.cuh"
#include "rows_host.cuh"

using namespace wpsgd;

namespace {

// ---- workspace -----------------------------------------------------------------------------------------------------------
// One buffer per context, allocated by the first call that needs it and never moved (a captured graph keeps its address). Its size
// depends on d alone. Calls of one context follow each other on its stream, so they can share it.
constexpr int kMaxBlocks = 148 * 8;             // of any kernel that leaves sums here
constexpr int kGradParts = 148 * 2;             // partial gradients at most
constexpr long long kCoefRows = 1 << 16;        // rows per step of the two-pass gradient
struct RowsLayout {
  int parts;
  size_t ticket, sums, coef, part, total;
  explicit RowsLayout(long long d) {
    parts = (int)std::max(1ll, std::min<long long>(kGradParts, (1ll << 23) / d));
    ticket = 0;
    sums = 256;
    coef = sums + kMaxBlocks * 2 * sizeof(double);
    part = coef + kCoefRows * sizeof(float);
    total = part + (size_t)parts * (size_t)d * sizeof(float);
  }
};
wpsgd_status rows_workspace(wpsgd_ctx* c) {
  if (c->rows_ws) return WPSGD_OK;
  cudaStreamCaptureStatus capturing = cudaStreamCaptureStatusNone;
  CU_TRY(c, cudaStreamIsCapturing(c->stream, &capturing));
  if (capturing != cudaStreamCaptureStatusNone)
    return fail(c, WPSGD_ERR_STATE, "the first call of a gradient, norm or clipping operator on a context allocates its workspace: make one before the capture");
  void* ws = nullptr;
  // another stream of the process may be under capture: an allocation does not touch it, which "relaxed" says
  cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;
  CU_TRY(c, cudaThreadExchangeStreamCaptureMode(&mode));
  const cudaError_t allocated = cudaMalloc(&ws, RowsLayout(c->d).total);
  cudaThreadExchangeStreamCaptureMode(&mode);
  CU_TRY(c, allocated);
  cudaError_t e = cudaMemsetAsync(ws, 0, RowsLayout(c->d).sums, c->stream);
  if (e != cudaSuccess) {
    cudaFree(ws);
    CU_TRY(c, e);
  }
  c->rows_ws = ws;
  return WPSGD_OK;
}

long long blocks_of(long long d) { return (d + Q_BLOCK - 1) / Q_BLOCK; }

// 8-bit rows as every entry point takes them
const char* check_rows8(const uint8_t* Q, int64_t ld_q, const float* scales, int64_t ld_s, int64_t n, long long d) {
  if (n < 0) return "negative row count";
  if (n > 0 && (!Q || !scales)) return "8-bit rows or scales are NULL";
  if (ld_q < d || ld_q % 16) return "8-bit rows need a stride of at least d and a multiple of 16 bytes";
  if (n > 0 && !aligned16(Q)) return "8-bit rows must start on 16 bytes";
  if ((uintptr_t)scales % sizeof(float)) return "scales are not aligned to their elements";
  if (ld_s < blocks_of(d)) return "scales need a stride of at least ceil(d / 128)";
  return nullptr;
}

// ---- margins -------------------------------------------------------------------------------------------------------------
struct MarginsCall {
  const uint8_t* Q;
  long long ld_q;
  const uint8_t* M;
  long long ld_m, d;
  MarginsParams p;
};

// Boxes of 128 columns and `box_rows` rows of an 8-bit matrix; what lies outside it reads as zeros.
bool encode_rows8(CUtensorMap* map, const uint8_t* base, long long d, long long rows, long long ld, int box_rows) {
  const cuuint64_t dims[2] = {(cuuint64_t)d, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld};
  const cuuint32_t box[2] = {Q_BLOCK, (cuuint32_t)box_rows}, steps[2] = {1, 1};
  return tensor_map_encoder()(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, (void*)base, dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename OT, int BN>
wpsgd_status launch_margins(wpsgd_ctx* c, const MarginsCall& call, int splits) {
  using Shape = MarginsShape<BN>;
  static_assert(Shape::stages >= 3 && Shape::smem <= (int)kSmemMax, "a ring of three stages must fit");
  CUtensorMap map_q, map_m;
  MarginsParams p = call.p;
  if (!tensor_map_encoder()) return fail(c, WPSGD_ERR_CUDA, "margins_fp8: the driver has no cuTensorMapEncodeTiled");
  if (!encode_rows8(&map_q, call.Q, call.d, p.n_rows, call.ld_q, MG_ROWS) || !encode_rows8(&map_m, call.M, call.d, p.n_models, call.ld_m, BN))
    return fail(c, WPSGD_ERR_UNSUPPORTED, "margins_fp8: sizes or strides that a tensor map cannot describe");
  p.tiles_m = (p.n_models + BN - 1) / BN;
  const long long tiles = (long long)((p.n_rows + MG_ROWS - 1) / MG_ROWS) * p.tiles_m;
  if (tiles > INT32_MAX - 148 || tiles / 148 * p.blocks > INT32_MAX) return fail(c, WPSGD_ERR_UNSUPPORTED, "margins_fp8: too many tiles");
  p.tiles = (int)tiles;
  p.splits = splits;
  if (splits == 1) {
    CU_TRY(c, (allow_smem<margins_kernel<OT, BN, false>>(c)));
    CU_TRY(c, launch(margins_kernel<OT, BN, false>, (unsigned)std::min<long long>(tiles, 148), Shape::threads, Shape::smem, c->stream, map_q, map_m, p));
  } else if constexpr (Shape::max_splits > 1) {
    CU_TRY(c, (allow_smem<margins_kernel<OT, BN, true>>(c)));
    CU_TRY(c, launch_clusters(margins_kernel<OT, BN, true>, (unsigned)(tiles * splits), Shape::threads, Shape::smem, c->stream, (unsigned)splits, map_q, map_m, p));
  }
  c->launches++;
  return WPSGD_OK;
}

template <typename OT>
wpsgd_status margins_of(wpsgd_ctx* c, const MarginsCall& call) {
  // Width of a tile and CTAs per tile by the time of the busiest SM, in cycles: per tile and block of columns the products (2 per
  // model), the copies (16 KB of rows and 128 bytes per model at about 40 bytes a cycle) or the hand-over from role to role (600),
  // whichever is longest; 5000 for the sums of a cluster to meet. 2047 rows of 999 columns on 37 models, 48 tiles of 16: 5.3 us, in pairs
  // of CTAs 6.6; 2 rows of 5918 columns on 15 models, one tile: 16.1 us by one CTA, 6.6 by eight.
  struct Choice {
    long long bn, splits, cycles;
  } best = {0, 1, 0};
  for (long long bn : {16, 32, 64, 128, 256}) {
    const long long tiles = ((call.p.n_rows + MG_ROWS - 1) / MG_ROWS) * ((call.p.n_models + bn - 1) / bn), rounds = (tiles + 147) / 148;
    const long long step = std::max({2 * bn, (MG_ROWS + bn) * Q_BLOCK / 40, 600ll});
    const int most = bn == 16 ? MarginsShape<16>::max_splits : bn == 32 ? MarginsShape<32>::max_splits : bn == 64 ? MarginsShape<64>::max_splits : bn == 128 ? MarginsShape<128>::max_splits : 1;
    for (long long splits : {1, 2, 4, 8}) {
      if (splits > 1 && (splits > most || tiles * splits > 148 || call.p.blocks < 2 * splits)) continue;
      const long long cycles = rounds * ((call.p.blocks + splits - 1) / splits * step + 12 * bn) + (splits > 1 ? 5000 : 0);
      if (best.bn == 0 || cycles < best.cycles) best = {bn, splits, cycles};
    }
  }
  const int splits = (int)best.splits;
  if (best.bn == 16) return launch_margins<OT, 16>(c, call, splits);
  if (best.bn == 32) return launch_margins<OT, 32>(c, call, splits);
  if (best.bn == 64) return launch_margins<OT, 64>(c, call, splits);
  if (best.bn == 128) return launch_margins<OT, 128>(c, call, splits);
  return launch_margins<OT, 256>(c, call, splits);
}

// ---- gradient ------------------------------------------------------------------------------------------------------------
template <typename RT>
wpsgd_status gradient_any_width(wpsgd_ctx* c, GradParams p, int* parts, int* n_sums) {
  const RowsLayout lay(c->d);
  float* coef = (float*)((char*)c->rows_ws + lay.coef);
  const int slabs = (int)((p.d + GRAD_THREADS - 1) / GRAD_THREADS);
  const long long first = std::min(p.n_rows, kCoefRows);
  *parts = (int)std::max(1ll, std::min<long long>({(long long)lay.parts, (long long)(kMaxBlocks / slabs), (first + 31) / 32}));
  *n_sums = grid_for(first, GRAD_THREADS / 32, kMaxBlocks);
  for (long long row0 = 0; row0 < p.n_rows; row0 += kCoefRows) {
    const long long count = std::min(p.n_rows - row0, kCoefRows);
    launch(gradient_margins_kernel<RT>, *n_sums, GRAD_THREADS, 0, c->stream, p, row0, count, row0 == 0, coef);
    CU_TRY(c, cudaGetLastError());
    launch(gradient_columns_kernel<RT>, dim3(slabs, *parts), GRAD_THREADS, 0, c->stream, p, row0, count, row0 == 0, coef);
    CU_TRY(c, cudaGetLastError());
    c->launches += 2;
  }
  return WPSGD_OK;
}

// One pass with G threads per row and CH units per thread; false: the rows are wider.
template <typename RT, int FEED, int G, int CH, int R>
wpsgd_status gradient_one_pass(wpsgd_ctx* c, GradParams& p, int* parts) {
  using Shape = GradShape<RT, FEED, G, CH, R>;
  const long long batches = (p.n_rows + R - 1) / R, blocks = (batches + Shape::groups - 1) / Shape::groups;
  *parts = (int)std::min<long long>({blocks, (long long)RowsLayout(c->d).parts, 148ll * Shape::per_sm});
  const long long row_bytes = p.d * (16 / Shape::V);
  p.slots = FEED == FEED_BULK ? Shape::bulk_slots(row_bytes) : 0;
  const int smem = Shape::smem(row_bytes);
  if (FEED == FEED_BULK && p.slots < 2) return fail(c, WPSGD_ERR_STATE, "gradient: a ring of two slots must fit");
  CU_TRY(c, (allow_smem<gradient_rows_kernel<RT, FEED, G, CH, R>>(c)));
  if ((long long)*parts * p.d <= GRAD_LAST_BLOCK) p.ticket = (unsigned*)((char*)c->rows_ws + RowsLayout(c->d).ticket);
  CU_TRY(c, launch(gradient_rows_kernel<RT, FEED, G, CH, R>, *parts, Shape::threads, smem, c->stream, p));
  c->launches++;
  return WPSGD_OK;
}
template <typename RT, int FEED>
wpsgd_status gradient_by_width(wpsgd_ctx* c, GradParams& p, int* parts, int* n_sums) {
  constexpr int V = RowUnit<RT>::V, R = V == 16 || (V == 8 && FEED == FEED_ELEMENTS) ? 4 : 8;
  const long long units = (p.d + V - 1) / V;
  auto run = [&](auto g, auto ch, auto r) {
    const wpsgd_status s = gradient_one_pass<RT, FEED, decltype(g)::value, decltype(ch)::value, decltype(r)::value>(c, p, parts);
    *n_sums = *parts;
    return s;
  };
#define GRAD_RUN(G, CH, R_) run(std::integral_constant<int, G>(), std::integral_constant<int, CH>(), std::integral_constant<int, R_>())
  if (units <= 4) return GRAD_RUN(4, 1, 4);
  if (units <= 8) return GRAD_RUN(8, 1, R);
  if (units <= 16) return GRAD_RUN(16, 1, R);
  if (units <= 32) return GRAD_RUN(32, 1, R);
  if (units <= 64) return GRAD_RUN(64, 1, R);
  if (units <= 128) return GRAD_RUN(128, 1, R);
  if (units <= 256) return GRAD_RUN(256, 1, R);
  if (units <= 512) {  // bf16 by elements: two units of a row do not fit a thread's registers beside the next rows (65536 x 3230: 295 us, 228 this way)
    if constexpr (V == 8 && FEED == FEED_ELEMENTS) return GRAD_RUN(512, 1, R);
    else return GRAD_RUN(256, 2, R / 2);
  }
  if (units <= 1024) return GRAD_RUN(512, 2, R / 2);
  if constexpr (V < 16)
    if (units <= 2048) return GRAD_RUN(512, 4, 2);
#undef GRAD_RUN
  return gradient_any_width<RT>(c, p, parts, n_sums);
}

template <typename RT>
wpsgd_status gradient(wpsgd_ctx* c, GradParams p) {
  wpsgd_status s = rows_workspace(c);
  if (s != WPSGD_OK) return s;
  const RowsLayout lay(c->d);
  p.sums = (double*)((char*)c->rows_ws + lay.sums);
  p.part = (float*)((char*)c->rows_ws + lay.part);
  int parts = 0, n_sums = 0;
  if (p.n_rows > 0) {
    const bool units = aligned16(p.X) && p.ld % RowUnit<RT>::V == 0;
    if constexpr (std::is_same<RT, Row8>::value) s = gradient_by_width<RT, FEED_UNITS>(c, p, &parts, &n_sums);
    else if (units && p.d % RowUnit<RT>::V == 0) s = gradient_by_width<RT, FEED_BULK>(c, p, &parts, &n_sums);
    else s = units ? gradient_by_width<RT, FEED_UNITS>(c, p, &parts, &n_sums) : gradient_by_width<RT, FEED_ELEMENTS>(c, p, &parts, &n_sums);
    if (s != WPSGD_OK || p.ticket) return s;
  }
  launch(gradient_finish_kernel, (unsigned)((p.d + 31) / 32), 32 * GRAD_FINISH_WARPS, 0, c->stream, p, parts, n_sums);
  CU_TRY(c, cudaGetLastError());
  c->launches++;
  return WPSGD_OK;
}

const char* check_gradient(const wpsgd_ctx* c, const float* y, int64_t n_rows, const float* w, float lambda, wpsgd_loss loss, const float* grad, const float* out) {
  if (!w || !grad || !out || (n_rows > 0 && !y)) return "NULL argument";
  if (((uintptr_t)y | (uintptr_t)w | (uintptr_t)grad | (uintptr_t)out) % sizeof(float)) return "y, w, grad or out is not aligned to its elements";
  if ((int)loss < 0 || (int)loss > 2) return "unknown loss";
  if (!std::isfinite(lambda)) return "lambda is not finite";
  const size_t nd = (size_t)c->d * 4;
  if (overlap(grad, nd, w, nd) || overlap(out, 8, w, nd) || overlap(out, 8, grad, nd)) return "grad, out and w overlap";
  return nullptr;
}

// ---- norm and clipping ---------------------------------------------------------------------------------------------------
constexpr int kFewTensors = 32, kManyTensors = 1072;  // per launch: 3 and 32 KB of kernel arguments (of which 32764 bytes are allowed)

struct Range {
  uintptr_t lo, hi;
  bool out;
};

}  // namespace

// What wpsgd_grad_list_create makes of its arguments: the kernels' arguments, launch by launch, and the address ranges by address.
struct wpsgd_grad_list {
  std::vector<TensorList<kFewTensors>> few;  // one of the two: `few` where one launch of it is enough
  std::vector<TensorList<kManyTensors>> many;
  std::vector<Range> ranges;
  uintptr_t longest = 0;   // range, bytes
  long long chunks = 0;    // of the launch with most
  int blocks = 1;
  bool in_place = true;
};

namespace {

template <int N>
void add_tensor(std::vector<TensorList<N>>& lists, const void* src, void* dst, long long n, bool bf16) {
  const long long chunks = (n + CLIP_CHUNK - 1) / CLIP_CHUNK;
  if (lists.empty() || lists.back().n == N || lists.back().first_chunk[lists.back().n] + chunks > INT32_MAX) {
    lists.emplace_back();
    lists.back().n = 0;
    lists.back().first_chunk[0] = 0;
  }
  TensorList<N>& l = lists.back();
  l.src[l.n] = src;
  l.dst[l.n] = dst;
  l.elems_type[l.n] = n * 2 + (bf16 ? 1 : 0);
  l.first_chunk[l.n + 1] = l.first_chunk[l.n] + (int)chunks;
  l.n++;
}

// The first tensor of each block's share, so that no block has to search for it
template <int N>
void set_starts(std::vector<TensorList<N>>& lists, int blocks) {
  for (TensorList<N>& l : lists) {
    const long long total = l.first_chunk[l.n];
    int i = 0;
    for (int b = 0; b < blocks; ++b) {
      const int c0 = (int)(total * b / blocks);
      while (i + 1 < l.n && l.first_chunk[i + 1] <= c0) ++i;
      l.start[b] = (uint16_t)i;
    }
  }
}

// nullptr, or what is wrong
const char* make_list(wpsgd_grad_list* list, const void* const* src, void* const* dst, const int64_t* n_elems, const wpsgd_xtype* types, int32_t n_tensors) {
  int filled = 0;
  for (int i = 0; i < n_tensors; ++i) {
    if (!known(types[i])) return "unknown element type";
    if (n_elems[i] < 0 || n_elems[i] > (1ll << 43)) return "element count out of range";
    filled += n_elems[i] > 0;
  }
  list->ranges.reserve(2 * (size_t)filled);
  for (int i = 0; i < n_tensors; ++i) {
    const long long n = n_elems[i];
    if (n == 0) continue;
    const size_t es = element_size(types[i]);
    void* to = dst ? dst[i] : const_cast<void*>(src[i]);
    if (!src[i] || !to) return "a tensor is NULL";
    if ((uintptr_t)src[i] % es || (uintptr_t)to % es) return "a tensor is not aligned to its elements";
    if (filled <= kFewTensors) add_tensor(list->few, src[i], to, n, types[i] == WPSGD_X_BF16);
    else add_tensor(list->many, src[i], to, n, types[i] == WPSGD_X_BF16);
    list->in_place = list->in_place && src[i] == to;
    list->ranges.push_back({(uintptr_t)to, (uintptr_t)to + (size_t)n * es, true});
    if (src[i] != to) list->ranges.push_back({(uintptr_t)src[i], (uintptr_t)src[i] + (size_t)n * es, false});
    list->longest = std::max<uintptr_t>(list->longest, (size_t)n * es);
  }
  for (const auto& l : list->few) list->chunks = std::max<long long>(list->chunks, l.first_chunk[l.n]);
  for (const auto& l : list->many) list->chunks = std::max<long long>(list->chunks, l.first_chunk[l.n]);
  list->blocks = list->few.size() == 1 && list->chunks <= CLIP_SMALL_CHUNKS ? CLIP_CLUSTER : (int)std::max(1ll, std::min<long long>(CLIP_BLOCKS, list->chunks));
  set_starts(list->few, list->blocks);
  set_starts(list->many, list->blocks);
  // every element is written by one thread and read by no other: outputs are disjoint, and each is its own input or apart from all
  std::sort(list->ranges.begin(), list->ranges.end(), [](const Range& a, const Range& b) { return a.lo < b.lo; });
  uintptr_t end_all = 0, end_out = 0;  // ends of what lies before: of all ranges, of outputs
  for (const Range& q : list->ranges) {
    if (q.lo < end_out || (q.out && q.lo < end_all)) return "an output overlaps another output or another tensor's input";
    end_all = std::max(end_all, q.hi);
    if (q.out) end_out = std::max(end_out, q.hi);
  }
  return nullptr;
}

template <int N>
wpsgd_status norm_and_scale(wpsgd_ctx* c, const std::vector<TensorList<N>>& lists, int blocks, bool scale, bool in_place, double max_norm, float* norm_out) {
  double* part = (double*)((char*)c->rows_ws + RowsLayout(c->d).sums);
  static_assert(CLIP_BLOCKS <= 2 * kMaxBlocks, "block sums must fit the workspace");
  for (size_t i = 0; i < lists.size(); ++i) {
    launch(squares_kernel<N>, blocks, CLIP_THREADS, 0, c->stream, lists[i], i == 0, part);
    CU_TRY(c, cudaGetLastError());
    c->launches++;
  }
  if (!scale || lists.empty()) {
    launch(norm_kernel, 1, CLIP_THREADS, 0, c->stream, part, lists.empty() ? 0 : blocks, norm_out);
    CU_TRY(c, cudaGetLastError());
    c->launches++;
    return WPSGD_OK;
  }
  for (size_t i = lists.size(); i-- > 0;) {
    launch(scale_kernel<N>, blocks, CLIP_THREADS, 0, c->stream, lists[i], part, blocks, max_norm, in_place, norm_out);
    CU_TRY(c, cudaGetLastError());
    c->launches++;
  }
  return WPSGD_OK;
}

wpsgd_status run_list(wpsgd_ctx* c, const wpsgd_grad_list* list, bool scale, double max_norm, float* norm_out) {
  if (!list || !norm_out) return fail(c, WPSGD_ERR_INVALID_ARG, "the list or norm_out is NULL");
  if ((uintptr_t)norm_out % sizeof(float)) return fail(c, WPSGD_ERR_INVALID_ARG, "norm_out is not aligned to its element");
  // norm_out in no range: of those that start before its end, only such as start less than the longest before it can reach it
  const uintptr_t lo = (uintptr_t)norm_out, hi = lo + sizeof(float);
  auto it = std::lower_bound(list->ranges.begin(), list->ranges.end(), hi, [](const Range& r, uintptr_t v) { return r.lo < v; });
  while (it != list->ranges.begin()) {
    --it;
    if (it->hi > lo) return fail(c, WPSGD_ERR_INVALID_ARG, "norm_out overlaps a tensor of the list");
    if (it->lo + list->longest <= lo) break;
  }
  DeviceGuard guard(c->device);
  if (list->few.size() == 1 && list->chunks <= CLIP_SMALL_CHUNKS) {
    CU_TRY(c, launch(clip_small_kernel<kFewTensors>, CLIP_CLUSTER, CLIP_THREADS, 0, c->stream, list->few[0], scale, max_norm, list->in_place, norm_out));
    c->launches++;
    return WPSGD_OK;
  }
  wpsgd_status s = rows_workspace(c);
  if (s != WPSGD_OK) return s;
  const int blocks = list->blocks;
  return list->many.empty() ? norm_and_scale(c, list->few, blocks, scale, list->in_place, max_norm, norm_out)
                            : norm_and_scale(c, list->many, blocks, scale, list->in_place, max_norm, norm_out);
}

}  // namespace

extern "C" {

wpsgd_status wpsgd_quantize_rows(wpsgd_ctx* c, const void* X, wpsgd_xtype xt, int64_t ld_elems, int64_t n_rows, uint8_t* Q, int64_t ld_q, float* scales, int64_t ld_s) {
  if (!c) return fail(nullptr, WPSGD_ERR_INVALID_ARG, "ctx is NULL");
  if (!known(xt)) return fail(c, WPSGD_ERR_INVALID_ARG, "unknown feature type");
  if (ld_elems < c->d || (n_rows > 0 && !X)) return fail(c, WPSGD_ERR_INVALID_ARG, "quantize_rows: bad argument");
  if (const char* why = check_rows8(Q, ld_q, scales, ld_s, n_rows, c->d)) return fail(c, WPSGD_ERR_INVALID_ARG, std::string("quantize_rows: ") + why);
  if (n_rows == 0) return WPSGD_OK;
  const size_t es = element_size(xt);
  if ((uintptr_t)X % es) return fail(c, WPSGD_ERR_INVALID_ARG, "quantize_rows: X is not aligned to its elements");
  const long long nb = blocks_of(c->d);
  if (c->d > INT32_MAX - Q_BLOCK || n_rows > INT64_MAX / nb / 64) return fail(c, WPSGD_ERR_UNSUPPORTED, "quantize_rows: 2^31 columns or 2^57 blocks and more");
  const Region x = {X, (long long)(c->d * es), (long long)(ld_elems * es), n_rows}, q = {Q, c->d, ld_q, n_rows}, s = {scales, nb * 4, ld_s * 4, n_rows};
  if (meet(x, q) || meet(x, s) || meet(q, s)) return fail(c, WPSGD_ERR_INVALID_ARG, "quantize_rows: X, Q and scales overlap");
  DeviceGuard guard(c->device);
  const bool vec = aligned16(X) && ((size_t)ld_elems * es) % 16 == 0 && ((size_t)c->d * es) % 16 == 0;
  auto go = [&](auto tag) {
    using XT = decltype(tag);
    constexpr int U = 4, per_warp = 32 / (Q_BLOCK / XVec<XT>::V);
    if (vec) launch(quantize_rows_kernel<XT, U>, grid_for(n_rows * nb, 8 * U * per_warp, 148 * 4), 256, 0, c->stream, (const XT*)X, ld_elems, n_rows, c->d, (int)nb, Q, ld_q, scales, ld_s);
    else launch(quantize_elements_kernel<XT, U>, grid_for(n_rows * nb, 8 * U, 148 * 4), 256, 0, c->stream, (const XT*)X, ld_elems, n_rows, c->d, (int)nb, Q, ld_q, scales, ld_s);
  };
  if (xt == WPSGD_X_F32) go(float());
  else go(__nv_bfloat16());
  CU_TRY(c, cudaGetLastError());
  c->launches++;
  return WPSGD_OK;
}

wpsgd_status wpsgd_margins_fp8(wpsgd_ctx* c, const uint8_t* Q, int64_t ld_q, const float* q_scales, int64_t ld_qs, int64_t n_rows, const uint8_t* M, int64_t ld_m,
                               const float* m_scales, int64_t ld_ms, int64_t n_models, void* Z, wpsgd_xtype zt, int64_t ld_z) {
  if (!c) return fail(nullptr, WPSGD_ERR_INVALID_ARG, "ctx is NULL");
  if (!known(zt)) return fail(c, WPSGD_ERR_INVALID_ARG, "margins_fp8: unknown output type");
  if (const char* why = check_rows8(Q, ld_q, q_scales, ld_qs, n_rows, c->d)) return fail(c, WPSGD_ERR_INVALID_ARG, std::string("margins_fp8: rows: ") + why);
  if (const char* why = check_rows8(M, ld_m, m_scales, ld_ms, n_models, c->d)) return fail(c, WPSGD_ERR_INVALID_ARG, std::string("margins_fp8: models: ") + why);
  if (n_rows > INT32_MAX - 256 || n_models > INT32_MAX - 256) return fail(c, WPSGD_ERR_UNSUPPORTED, "margins_fp8: 2^31 - 256 rows or models and more");
  if (c->d > INT32_MAX - Q_BLOCK) return fail(c, WPSGD_ERR_UNSUPPORTED, "margins_fp8: 2^31 columns and more");  // columns of a tile are 32-bit coordinates
  if (n_rows == 0 || n_models == 0) return WPSGD_OK;
  if (!Z || ld_z < n_models || (uintptr_t)Z % element_size(zt)) return fail(c, WPSGD_ERR_INVALID_ARG, "margins_fp8: Z is NULL, not aligned to its elements, or its stride is below n_models");
  const long long zs = (long long)element_size(zt), nb = blocks_of(c->d);
  const Region z = {Z, n_models * zs, ld_z * zs, n_rows};
  if (meet(z, {Q, c->d, ld_q, n_rows}) || meet(z, {q_scales, nb * 4, ld_qs * 4, n_rows}) || meet(z, {M, c->d, ld_m, n_models}) || meet(z, {m_scales, nb * 4, ld_ms * 4, n_models}))
    return fail(c, WPSGD_ERR_INVALID_ARG, "margins_fp8: Z overlaps rows, models or their scales");
  DeviceGuard guard(c->device);
  const MarginsCall call = {Q, ld_q, M, ld_m, c->d, {q_scales, ld_qs, m_scales, ld_ms, Z, ld_z, (int)n_rows, (int)n_models, (int)blocks_of(c->d), 0, 0, 1,
                            ld_z % 2 == 0 && (uintptr_t)Z % (2 * element_size(zt)) == 0, c->opt_spin_limit, c->opt_drop_block, c->status}};
  return zt == WPSGD_X_F32 ? margins_of<float>(c, call) : margins_of<__nv_bfloat16>(c, call);
}

wpsgd_status wpsgd_objective_grad(wpsgd_ctx* c, const void* X, wpsgd_xtype xt, int64_t ld_elems, const float* y, int64_t n_rows, const float* w, float lambda,
                                  wpsgd_loss loss, float* grad, float* out) {
  if (!c) return fail(nullptr, WPSGD_ERR_INVALID_ARG, "ctx is NULL");
  if (!known(xt)) return fail(c, WPSGD_ERR_INVALID_ARG, "unknown feature type");
  if (n_rows < 0 || ld_elems < c->d || (n_rows > 0 && !X)) return fail(c, WPSGD_ERR_INVALID_ARG, "objective_grad: bad argument");
  if (const char* why = check_gradient(c, y, n_rows, w, lambda, loss, grad, out)) return fail(c, WPSGD_ERR_INVALID_ARG, std::string("objective_grad: ") + why);
  if ((uintptr_t)X % element_size(xt)) return fail(c, WPSGD_ERR_INVALID_ARG, "objective_grad: X is not aligned to its elements");
  DeviceGuard guard(c->device);
  const GradParams p = {X, ld_elems, nullptr, 0, y, w, n_rows, c->d, (int)loss, lambda, grad, out, nullptr, nullptr, nullptr, 0, c->opt_spin_limit, c->opt_drop_block, c->status};
  return xt == WPSGD_X_F32 ? gradient<float>(c, p) : gradient<__nv_bfloat16>(c, p);
}

wpsgd_status wpsgd_objective_grad_fp8(wpsgd_ctx* c, const uint8_t* Q, int64_t ld_q, const float* scales, int64_t ld_s, const float* y, int64_t n_rows, const float* w,
                                      float lambda, wpsgd_loss loss, float* grad, float* out) {
  if (!c) return fail(nullptr, WPSGD_ERR_INVALID_ARG, "ctx is NULL");
  if (const char* why = check_rows8(Q, ld_q, scales, ld_s, n_rows, c->d)) return fail(c, WPSGD_ERR_INVALID_ARG, std::string("objective_grad_fp8: ") + why);
  if (const char* why = check_gradient(c, y, n_rows, w, lambda, loss, grad, out)) return fail(c, WPSGD_ERR_INVALID_ARG, std::string("objective_grad_fp8: ") + why);
  DeviceGuard guard(c->device);
  const GradParams p = {Q, ld_q, scales, ld_s, y, w, n_rows, c->d, (int)loss, lambda, grad, out, nullptr, nullptr, nullptr, 0, c->opt_spin_limit, c->opt_drop_block, c->status};
  return gradient<Row8>(c, p);
}

wpsgd_status wpsgd_grad_list_create(const void* const* grads, void* const* out, const int64_t* n_elems, const wpsgd_xtype* types, int32_t n_tensors,
                                    wpsgd_grad_list** list) {
  if (!list) return fail(nullptr, WPSGD_ERR_INVALID_ARG, "list is NULL");
  *list = nullptr;
  if (n_tensors < 0 || (n_tensors > 0 && (!grads || !n_elems || !types))) return fail(nullptr, WPSGD_ERR_INVALID_ARG, "grad_list_create: bad argument");
  try {
    std::unique_ptr<wpsgd_grad_list> l(new wpsgd_grad_list());
    if (const char* why = make_list(l.get(), grads, out, n_elems, types, n_tensors)) return fail(nullptr, WPSGD_ERR_INVALID_ARG, std::string("grad_list_create: ") + why);
    *list = l.release();
  } catch (const std::bad_alloc&) {
    return fail(nullptr, WPSGD_ERR_ALLOC, "grad_list_create: no memory");
  }
  return WPSGD_OK;
}

wpsgd_status wpsgd_grad_list_destroy(wpsgd_grad_list* list) {
  delete list;
  return WPSGD_OK;
}

wpsgd_status wpsgd_grad_norm(wpsgd_ctx* c, const wpsgd_grad_list* list, float* norm_out) {
  if (!c) return fail(nullptr, WPSGD_ERR_INVALID_ARG, "ctx is NULL");
  return run_list(c, list, false, 0.0, norm_out);
}

wpsgd_status wpsgd_clip_grad_norm(wpsgd_ctx* c, const wpsgd_grad_list* list, double max_norm, float* norm_out) {
  if (!c) return fail(nullptr, WPSGD_ERR_INVALID_ARG, "ctx is NULL");
  if (!(max_norm >= 0.0)) return fail(c, WPSGD_ERR_INVALID_ARG, "clip_grad_norm: max_norm must be >= 0");
  return run_list(c, list, true, max_norm, norm_out);
}

}  // extern "C"
