// Rows that go to several nodes: sorted by node, laid out in that order, and brought back with weights (see include/wpsgd.h).
//
// A row i has `top` places, each with a node (negative: none). A place is a pair (i, j), numbered i top + j; its position is where its row
// stands among all rows sorted by node, equal nodes in the order of their places.
#pragma once

#include "common.cuh"

namespace wpsgd {

// ---- sorting ---------------------------------------------------------------------------------------------------------------
// A stable counting sort, by one of two forms. Up to 32767 places, without `order`, or with more nodes than many blocks' counts fit: one launch, a cluster of up to 8 blocks, each warp with a run
// of places and a counter per node in shared memory. Count; add up over warps, blocks (through distributed shared memory, about 2 us) and nodes; go over the places again and hand the positions out.
// More places: the same over up to 148 blocks in four launches (count, scan, place, order), whose latencies are less than what 8 blocks need for so many (131072 places on 128 nodes: 30 us by the
// cluster, 17 by four launches). Lanes with the same node find each other with one match instruction, so no counter is reached twice at a time and positions do not depend on timing.
//
// Bounds: latency. The places are read twice and the positions written once (1.5 MB for 131072 places).
constexpr int SORT_THREADS = 1024;
constexpr int SORT_COUNTERS = 32768;      // of all warps of a block
constexpr int SORT_MAX_NODES = 16384;     // counters of two warps, and a total per node beside them

struct SortParams {
  const int* node;
  long long places;
  int nodes, warps;  // warps of a block that count
  long long run;     // places of a warp, a multiple of 32
  int *where, *order;
  long long* shard_off;
  DevStatus* status;
};

__device__ __forceinline__ void cluster_barrier() { asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// A warp's places in order: f(place, node as given, node or -1, lanes with the same node)
template <typename F>
__device__ __forceinline__ void go_over_places(const int* node, long long begin, long long end, int n, int lane, F f) {
  constexpr int AHEAD = 8;  // loads in flight: one at a time would wait 600 cycles for each 32 places
  for (long long at = begin; at < end; at += 32 * AHEAD) {
    int key[AHEAD];
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
      const long long e = at + a * 32 + lane;
      key[a] = e < end ? node[e] : -1;
    }
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
      if (at + a * 32 >= end) break;
      const int k = key[a] >= 0 && key[a] < n ? key[a] : -1;
      f(at + a * 32 + lane, key[a], k, __match_any_sync(0xffffffffu, k));
      __syncwarp();
    }
  }
}
// Counts of a warp's places by node
__device__ __forceinline__ void count_places(const SortParams& p, unsigned* mine, long long begin, long long end, int lane) {
  go_over_places(p.node, begin, end, p.nodes, lane, [&](long long e, int given, int k, unsigned same) {
    if (k >= 0 && lane == __ffs(same) - 1) mine[k] += __popc(same);
    if (given >= p.nodes) set_status(p.status, DEV_BOUNDS, 20, e);
  });
}
// Positions handed out from a warp's counters, which hold the next position of each node
__device__ __forceinline__ void place_rows(const SortParams& p, unsigned* mine, long long begin, long long end, int lane, int* order) {
  go_over_places(p.node, begin, end, p.nodes, lane, [&](long long e, int, int k, unsigned same) {
    int pos = -1;
    if (k >= 0) pos = (int)(mine[k] + __popc(same & ((1u << lane) - 1)));
    __syncwarp();
    if (k >= 0 && lane == __ffs(same) - 1) mine[k] += __popc(same);
    if (e < end) p.where[e] = pos;
    if (k >= 0 && order) order[pos] = (int)e;
  });
}
// Counters of a block's warps: of each node those of earlier warps; returns into totals[] those of all
__device__ __forceinline__ void add_up_warps(const SortParams& p, unsigned* counters, unsigned* totals, int tid) {
  for (int k = tid; k < p.nodes; k += SORT_THREADS) {
    unsigned sum = 0;
    for (int w = 0; w < p.warps; ++w) {
      const unsigned c = counters[(size_t)w * p.nodes + k];
      counters[(size_t)w * p.nodes + k] = sum;
      sum += c;
    }
    totals[k] = sum;
  }
}
// Exclusive sums of `value` over the threads of a block, and `carry` moved on by all of them
__device__ __forceinline__ unsigned block_scan(unsigned value, unsigned& carry, unsigned* warp_sums, int warp, int lane) {
  unsigned sum = value;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned v = __shfl_up_sync(0xffffffffu, sum, o);
    if (lane >= o) sum += v;
  }
  if (lane == 31) warp_sums[warp] = sum;
  __syncthreads();
  const unsigned w = warp_sums[lane];
  unsigned ws = w;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned v = __shfl_up_sync(0xffffffffu, ws, o);
    if (lane >= o) ws += v;
  }
  const unsigned before = carry + __shfl_sync(0xffffffffu, ws - w, warp) + sum - value;
  carry += __shfl_sync(0xffffffffu, ws, 31);
  __syncthreads();
  return before;
}

__global__ void __launch_bounds__(SORT_THREADS) sort_rows_kernel(const __grid_constant__ SortParams p) {
  extern __shared__ unsigned sort_smem[];
  unsigned* totals = sort_smem;                // [nodes] of this block
  unsigned* counters = sort_smem + p.nodes;    // [warps][nodes]
  __shared__ unsigned warp_sums[32];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, n = p.nodes;
  unsigned rank, blocks;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(blocks));
  kernel_started();
  for (int i = tid; i < p.warps * n; i += SORT_THREADS) counters[i] = 0;
  kernel_inputs_ready();
  __syncthreads();

  const long long begin = ((long long)rank * p.warps + warp) * p.run, end = min(begin + p.run, p.places);
  unsigned* mine = counters + (size_t)warp * n;
  if (warp < p.warps) count_places(p, mine, begin, end, lane);
  __syncthreads();
  add_up_warps(p, counters, totals, tid);
  cluster_barrier();

  unsigned carry = 0;  // places of lower nodes
  for (int base = 0; base < n; base += SORT_THREADS) {
    const int k = base + tid;
    unsigned all = 0, before = 0;
    if (k < n)
      for (unsigned r = 0; r < blocks; ++r) {
        uint32_t from, c;
        asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(from) : "r"((uint32_t)__cvta_generic_to_shared(totals + k)), "r"(r));
        asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(c) : "r"(from) : "memory");
        if (r < rank) before += c;
        all += c;
      }
    const unsigned first = block_scan(all, carry, warp_sums, warp, lane);
    if (k < n) {
      if (rank == 0) p.shard_off[k] = first;
      for (int v = 0; v < p.warps; ++v) counters[(size_t)v * n + k] += first + before;
    }
  }
  __syncthreads();
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");  // this block has read the others' totals
  if (rank == 0 && tid == 0) p.shard_off[n] = carry;

  if (warp < p.warps) place_rows(p, mine, begin, end, lane, p.order);
  if (p.order)
    for (long long i = carry + (long long)rank * SORT_THREADS + tid; i < p.places; i += (long long)blocks * SORT_THREADS) p.order[i] = -1;
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");  // no block leaves while its totals are read
}

// Many places: blocks all over the GPU, in four steps. The counts of the blocks, [blocks][nodes], stand in `order` until the positions are known, which is why it
// has to be there: no memory beyond the arguments is used.
__global__ void __launch_bounds__(SORT_THREADS) sort_count_kernel(const __grid_constant__ SortParams p) {
  extern __shared__ unsigned sort_smem[];
  unsigned* counters = sort_smem + p.nodes;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, n = p.nodes;
  kernel_started();
  for (int i = tid; i < p.warps * n; i += SORT_THREADS) counters[i] = 0;
  kernel_inputs_ready();
  __syncthreads();
  const long long begin = ((long long)blockIdx.x * p.warps + warp) * p.run, end = min(begin + p.run, p.places);
  if (warp < p.warps) count_places(p, counters + (size_t)warp * n, begin, end, lane);
  __syncthreads();
  for (int k = tid; k < n; k += SORT_THREADS) {
    unsigned sum = 0;
    for (int w = 0; w < p.warps; ++w) sum += counters[(size_t)w * n + k];
    p.order[(size_t)blockIdx.x * n + k] = (int)sum;
  }
}
// First position of each node in each block, from its counts
__global__ void __launch_bounds__(SORT_THREADS) sort_scan_kernel(const __grid_constant__ SortParams p, int blocks) {
  __shared__ unsigned warp_sums[32];
  const int tid = threadIdx.x, n = p.nodes;
  kernel_started();
  kernel_inputs_ready();
  unsigned carry = 0;
  for (int base = 0; base < n; base += SORT_THREADS) {
    const int k = base + tid;
    unsigned all = 0;
    if (k < n)
      for (int b0 = 0; b0 < blocks; b0 += 16) {  // read before written: loads behind a store to the same array would wait for each other
        unsigned c[16];
#pragma unroll
        for (int b = 0; b < 16; ++b) c[b] = b0 + b < blocks ? (unsigned)p.order[(size_t)(b0 + b) * n + k] : 0;
#pragma unroll
        for (int b = 0; b < 16; ++b) {
          if (b0 + b < blocks) p.order[(size_t)(b0 + b) * n + k] = (int)all;
          all += c[b];
        }
      }
    const unsigned first = block_scan(all, carry, warp_sums, tid >> 5, tid & 31);
    if (k < n) p.shard_off[k] = first;
  }
  if (tid == 0) p.shard_off[n] = carry;
}
__global__ void __launch_bounds__(SORT_THREADS) sort_place_kernel(const __grid_constant__ SortParams p) {
  extern __shared__ unsigned sort_smem[];
  unsigned *totals = sort_smem, *counters = sort_smem + p.nodes;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, n = p.nodes;
  kernel_started();
  for (int i = tid; i < p.warps * n; i += SORT_THREADS) counters[i] = 0;
  kernel_inputs_ready();
  __syncthreads();
  const long long begin = ((long long)blockIdx.x * p.warps + warp) * p.run, end = min(begin + p.run, p.places);
  unsigned* mine = counters + (size_t)warp * n;
  if (warp < p.warps) go_over_places(p.node, begin, end, n, lane, [&](long long, int, int k, unsigned same) {
    if (k >= 0 && lane == __ffs(same) - 1) mine[k] += __popc(same);
  });
  __syncthreads();
  add_up_warps(p, counters, totals, tid);
  for (int k = tid; k < n; k += SORT_THREADS) {
    const unsigned first = (unsigned)p.shard_off[k] + (unsigned)p.order[(size_t)blockIdx.x * n + k];
    for (int v = 0; v < p.warps; ++v) counters[(size_t)v * n + k] += first;
  }
  __syncthreads();
  if (warp < p.warps) place_rows(p, mine, begin, end, lane, nullptr);
}
__global__ void __launch_bounds__(256) sort_order_kernel(const __grid_constant__ SortParams p) {
  kernel_started();
  kernel_inputs_ready();
  const long long kept = p.shard_off[p.nodes];
  for (long long e = (long long)blockIdx.x * 256 + threadIdx.x; e < p.places; e += (long long)gridDim.x * 256) {
    const int pos = p.where[e];
    if (pos >= 0) p.order[pos] = (int)e;
    if (e >= kept) p.order[e] = -1;
  }
}

// ---- rows at any place in memory, by 16 bytes ----------------------------------------------------------------------------------
// A row as units of 16 bytes that start where those of another row do that lies elsewhere: unit u has the bytes from `skew` + 16 u on (skew -15 to 0, so the first and the
// last unit may reach outside the row: those bytes are anything). Where they do not start on 16 in memory, the two aligned units around them are read, if any byte
// of the row lies in them, and shifted together; what is the same for all units of a row is worked out once.
// Read-only 16 bytes where `yes`, zeros elsewhere: a predicate, not a branch. Neighbouring units of a shifted row share them in L1.
__device__ __forceinline__ uint4 ld16_if(const void* p, bool yes) {
  uint4 r = make_uint4(0u, 0u, 0u, 0u);
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.s32 p, %5, 0;\n\t@p ld.global.nc.v4.u32 {%0,%1,%2,%3}, [%4];\n\t}"
               : "+r"(r.x), "+r"(r.y), "+r"(r.z), "+r"(r.w)
               : "l"(p), "r"((int)yes));
  return r;
}
template <typename XT>
struct ShiftedRow {
  const uint4* at;  // the aligned unit in which unit 0 starts
  unsigned off;     // and how far into it
  int lo, n;        // aligned units lo to lo + n - 1 have bytes of the row
  __device__ __forceinline__ void find(const char* row, int width, int skew) {
    const char* start = row + skew;
    off = (unsigned)((uintptr_t)start & 15);
    at = (const uint4*)(start - off);
    lo = (int)(row - (const char*)at) >> 4;
    n = ((int)(row - (const char*)at) + width - 1 >> 4) - lo + 1;
  }
  // the two aligned units of unit u, asked for; and the unit itself, once they are there. Apart, so that several can be under way
  struct Raw {
    uint4 a, b;
  };
  __device__ __forceinline__ Raw ask(int u, bool yes) const {
    return {ld16_if(at + u, yes && (unsigned)(u - lo) < (unsigned)n), ld16_if(at + u + 1, yes && off != 0 && (unsigned)(u + 1 - lo) < (unsigned)n)};
  }
  __device__ __forceinline__ uint4 unit(const Raw& raw) const {
    unsigned w0 = raw.a.x, w1 = raw.a.y, w2 = raw.a.z, w3 = raw.a.w, w4 = raw.b.x, w5 = raw.b.y, w6 = raw.b.z, w7 = raw.b.w;
    if (off & 8) w0 = w2, w1 = w3, w2 = w4, w3 = w5, w4 = w6, w5 = w7;
    if (off & 4) w0 = w1, w1 = w2, w2 = w3, w3 = w4, w4 = w5;
    if (sizeof(XT) == 4) return make_uint4(w0, w1, w2, w3);
    const unsigned bits = (off & 3) * 8;
    return make_uint4(__funnelshift_r(w0, w1, bits), __funnelshift_r(w1, w2, bits), __funnelshift_r(w2, w3, bits), __funnelshift_r(w3, w4, bits));
  }
};
// 16 bytes to a row from byte `c` on, a multiple of 16 in memory; those that lie in the row are written.
template <typename XT, bool ALIGNED>
__device__ __forceinline__ void put16(char* row, int c, int width, uint4 v) {
  if (ALIGNED || (c >= 0 && c + 16 <= width)) {
    *(uint4*)(row + c) = v;
  } else {
    const unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 16 / (int)sizeof(XT); ++i) {
      const int at = c + i * (int)sizeof(XT);
      if (at < 0 || at >= width) continue;
      if constexpr (sizeof(XT) == 4) *(unsigned*)(row + at) = w[i];
      else *(unsigned short*)(row + at) = (unsigned short)(w[i / 2] >> (16 * (i % 2)));
    }
  }
}
template <typename XT>
__device__ __forceinline__ uint4 narrow16(const float (&f)[XVec<XT>::V]) {
  if constexpr (sizeof(XT) == 4) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  } else {
    uint4 r;
    unsigned* w = &r.x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
      w[i] = *(const unsigned*)&h;
    }
    return r;
  }
}

// A group of 2^lg threads has a row; a thread's units of 16 bytes are 2^lg apart. Several rows to a block of 256 threads.
constexpr int NODES_THREADS = 256;

struct NodesParams {
  const int* where;      // [n_rows, top]
  const float* weights;  // [n_rows, top], or NULL: all 1
  long long n_rows, n_sorted;
  int top, lg;
  int width;                  // bytes of a row
  const char* rows;           // [n_rows]: read by gather and by the gradient
  long long ld_rows;          // strides in bytes
  const char* sorted;         // [n_sorted]: read by combine and by the gradient
  long long ld_sorted;
  char* out;                  // [n_rows] of combine, [n_sorted] of gather and the gradient
  long long ld_out;
  float* dweights;            // [n_rows, top]
  DevStatus* status;
};

// A place's position, -1 where it has none or one outside the sorted rows (reported)
__device__ __forceinline__ int position(const NodesParams& p, long long place, bool report) {
  const int pos = __ldg(p.where + place);
  if (pos >= p.n_sorted) {
    if (report) set_status(p.status, DEV_BOUNDS, 21, place);
    return -1;
  }
  return pos;
}

// out[where[i, j]] = rows[i]: every row is read once and written `top` times. Bounds: bytes.
template <typename XT, bool ALIGNED>
__global__ void __launch_bounds__(NODES_THREADS) gather_rows_kernel(const __grid_constant__ NodesParams p) {
  kernel_started();
  kernel_inputs_ready();
  const int per = NODES_THREADS >> p.lg, t = threadIdx.x & ((1 << p.lg) - 1), step = 16 << p.lg;
  for (long long i = (long long)blockIdx.x * per + (threadIdx.x >> p.lg); i < p.n_rows; i += (long long)gridDim.x * per) {
    const char* row = p.rows + i * p.ld_rows;
    if constexpr (ALIGNED) {
      for (int c = t * 16; c < p.width; c += 4 * step) {
        uint4 v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (c + u * step < p.width) v[u] = ld_stream16(row + c + u * step);
        for (int j = 0; j < p.top; ++j) {
          const int pos = position(p, i * p.top + j, c == 0);
          if (pos < 0) continue;
          char* out = p.out + pos * p.ld_out + c;
#pragma unroll
          for (int u = 0; u < 4; ++u)
            if (c + u * step < p.width) *(uint4*)(out + u * step) = v[u];
        }
      }
    } else {  // units of the output, whose rows start anywhere
      for (int j = 0; j < p.top; ++j) {
        const int pos = position(p, i * p.top + j, t == 0);
        if (pos < 0) continue;
        char* out = p.out + pos * p.ld_out;
        const int skew = -(int)((uintptr_t)out & 15);
        ShiftedRow<XT> from;
        from.find(row, p.width, skew);
        for (int u0 = t; skew + u0 * 16 < p.width; u0 += 4 << p.lg) {
          typename ShiftedRow<XT>::Raw v[4];
#pragma unroll
          for (int u = 0; u < 4; ++u) v[u] = from.ask(u0 + (u << p.lg), true);
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const int c = skew + (u0 + (u << p.lg)) * 16;
            if (c < p.width) put16<XT, false>(out, c, p.width, from.unit(v[u]));
          }
        }
      }
    }
  }
}

// out[i] = sum_j weights[i, j] sorted[where[i, j]], j ascending, in fp32. Places without a position are left out, whatever their weight.
// Units under way at a time, of PLACES places each: four where a row has one place, two where it has more, one where rows start off 16 bytes, each read as two aligned ones (rows of more than
// PLACES places have them found anew for each unit). Bounds: bytes.
template <typename XT, bool ALIGNED, int PLACES>
__global__ void __launch_bounds__(NODES_THREADS, 4) combine_rows_kernel(const __grid_constant__ NodesParams p) {
  constexpr int V = XVec<XT>::V, UNITS = !ALIGNED ? 1 : PLACES == 1 ? 4 : 2;
  kernel_started();
  kernel_inputs_ready();
  const int per = NODES_THREADS >> p.lg, g = 1 << p.lg, t = threadIdx.x & (g - 1);
  for (long long i = (long long)blockIdx.x * per + (threadIdx.x >> p.lg); i < p.n_rows; i += (long long)gridDim.x * per) {
    char* out = p.out + i * p.ld_out;
    const int skew = ALIGNED ? 0 : -(int)((uintptr_t)out & 15);
    const char* at[PLACES];
    ShiftedRow<XT> from[PLACES];
    float w[PLACES];
    auto find = [&](int j) {  // places from j on; at NULL: none
#pragma unroll
      for (int a = 0; a < PLACES; ++a) {
        const int pos = j + a < p.top ? position(p, i * p.top + j + a, t == 0) : -1;
        at[a] = pos >= 0 ? p.sorted + pos * p.ld_sorted : nullptr;
        w[a] = pos >= 0 && p.weights ? __ldg(p.weights + i * p.top + j + a) : 1.0f;
        if (!ALIGNED) from[a].find(pos >= 0 ? at[a] : p.sorted, p.width, skew);
      }
    };
    if (p.top <= PLACES) find(0);
    for (int u0 = t; skew + u0 * 16 < p.width; u0 += UNITS * g) {
      float acc[UNITS][V];
#pragma unroll
      for (int u = 0; u < UNITS; ++u)
#pragma unroll
        for (int e = 0; e < V; ++e) acc[u][e] = 0.0f;
      for (int j = 0; j < p.top; j += PLACES) {
        if (p.top > PLACES) find(j);
        uint4 v[UNITS][PLACES];
        if constexpr (ALIGNED) {
#pragma unroll
          for (int u = 0; u < UNITS; ++u)
#pragma unroll
            for (int a = 0; a < PLACES; ++a) v[u][a] = ld_stream16_if(at[a] + (u0 + u * g) * 16, at[a] != nullptr && (u0 + u * g) * 16 < p.width);
        } else {
          typename ShiftedRow<XT>::Raw raw[UNITS][PLACES];
#pragma unroll
          for (int u = 0; u < UNITS; ++u)
#pragma unroll
            for (int a = 0; a < PLACES; ++a) raw[u][a] = from[a].ask(u0 + u * g, at[a] != nullptr);
#pragma unroll
          for (int u = 0; u < UNITS; ++u)
#pragma unroll
            for (int a = 0; a < PLACES; ++a) v[u][a] = from[a].unit(raw[u][a]);
        }
#pragma unroll
        for (int a = 0; a < PLACES; ++a) {
          if (!at[a]) continue;
#pragma unroll
          for (int u = 0; u < UNITS; ++u) {
            float f[V];
            XVec<XT>::widen(v[u][a], f);
#pragma unroll
            for (int e = 0; e < V; ++e) acc[u][e] = fmaf(w[a], f[e], acc[u][e]);
          }
        }
      }
#pragma unroll
      for (int u = 0; u < UNITS; ++u) {
        const int c = skew + (u0 + u * g) * 16;
        if (c < p.width) put16<XT, ALIGNED>(out, c, p.width, narrow16<XT>(acc[u]));
      }
    }
  }
}

// out[where[i, j]] = weights[i, j] rows[i] and dweights[i, j] = rows[i] . sorted[where[i, j]], with rows the gradient of combine's result.
// All three are gone through once; BATCH places have their sums in registers at a time, and four units of theirs are under way. The sums of a group's threads
// are added in a fixed order. Bounds: bytes (65536 bf16 rows of 4096 columns with two places each: one unit of four places at a time 530 us).
template <typename XT, bool ALIGNED, int BATCH>
__global__ void __launch_bounds__(NODES_THREADS) combine_grad_kernel(const __grid_constant__ NodesParams p) {
  constexpr int V = XVec<XT>::V, UNITS = 4 / BATCH;
  __shared__ float sums[NODES_THREADS / 32][BATCH];
  kernel_started();
  kernel_inputs_ready();
  const int per = NODES_THREADS >> p.lg, g = 1 << p.lg, t = threadIdx.x & (g - 1), step = 16 << p.lg, warp = threadIdx.x >> 5;
  // all threads of a block go round together: groups of more than a warp meet at barriers
  for (long long i0 = (long long)blockIdx.x * per; i0 < p.n_rows; i0 += (long long)gridDim.x * per) {
    const long long i = i0 + (threadIdx.x >> p.lg);
    const bool row_there = i < p.n_rows;
    const char* row = p.rows + i * p.ld_rows;
    for (int j = 0; j < p.top; j += BATCH) {
      int pos[BATCH];
      float w[BATCH], dot[BATCH];
#pragma unroll
      for (int a = 0; a < BATCH; ++a) {
        const long long place = i * p.top + j + a;
        pos[a] = row_there && j + a < p.top ? position(p, place, t == 0) : -1;
        w[a] = pos[a] >= 0 && p.weights ? __ldg(p.weights + place) : 1.0f;
        dot[a] = 0.0f;
      }
      if constexpr (ALIGNED) {
        if (row_there)
          for (int c = t * 16; c < p.width; c += UNITS * step) {
            uint4 dv[UNITS], v[UNITS][BATCH];
#pragma unroll
            for (int u = 0; u < UNITS; ++u) {
              const bool in = c + u * step < p.width;
              dv[u] = ld_stream16_if(row + c + u * step, in);
#pragma unroll
              for (int a = 0; a < BATCH; ++a) v[u][a] = ld_stream16_if(p.sorted + (pos[a] < 0 ? 0 : pos[a]) * p.ld_sorted + c + u * step, in && pos[a] >= 0);
            }
#pragma unroll
            for (int u = 0; u < UNITS; ++u) {
              if (c + u * step >= p.width) break;
              float d[V], f[V];
              XVec<XT>::widen(dv[u], d);
#pragma unroll
              for (int a = 0; a < BATCH; ++a) {
                if (pos[a] < 0) continue;
                XVec<XT>::widen(v[u][a], f);
                float o[V];
#pragma unroll
                for (int e = 0; e < V; ++e) {
                  dot[a] = fmaf(d[e], f[e], dot[a]);
                  o[e] = w[a] * d[e];
                }
                *(uint4*)(p.out + pos[a] * p.ld_out + c + u * step) = narrow16<XT>(o);
              }
            }
          }
      } else {
#pragma unroll
        for (int a = 0; a < BATCH; ++a) {
          if (pos[a] < 0) continue;
          char* out = p.out + pos[a] * p.ld_out;
          const int skew = -(int)((uintptr_t)out & 15);
          ShiftedRow<XT> ds, fs;
          ds.find(row, p.width, skew);
          fs.find(p.sorted + pos[a] * p.ld_sorted, p.width, skew);
          for (int u0 = t; skew + u0 * 16 < p.width; u0 += 2 * g) {
            typename ShiftedRow<XT>::Raw dr[2], fr[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) dr[u] = ds.ask(u0 + u * g, true), fr[u] = fs.ask(u0 + u * g, true);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              const int c = skew + (u0 + u * g) * 16;
              if (c >= p.width) break;
              float d[V], f[V], o[V];
              XVec<XT>::widen(ds.unit(dr[u]), d);
              XVec<XT>::widen(fs.unit(fr[u]), f);
#pragma unroll
              for (int e = 0; e < V; ++e) {
                const bool in = (unsigned)(c + e * (int)sizeof(XT)) < (unsigned)p.width;
                dot[a] = fmaf(in ? d[e] : 0.0f, in ? f[e] : 0.0f, dot[a]);
                o[e] = w[a] * d[e];
              }
              put16<XT, false>(out, c, p.width, narrow16<XT>(o));
            }
          }
        }
      }
#pragma unroll
      for (int a = 0; a < BATCH; ++a)
        for (int o = min(g, 32) / 2; o > 0; o >>= 1) dot[a] += __shfl_xor_sync(0xffffffffu, dot[a], o);
      if (g > 32) {
        __syncthreads();
        if ((threadIdx.x & 31) == 0)
#pragma unroll
          for (int a = 0; a < BATCH; ++a) sums[warp][a] = dot[a];
        __syncthreads();
        if (t < BATCH) {
          float sum = 0.0f;
          for (int v = 0; v < g / 32; ++v) sum += sums[warp + v][t];
#pragma unroll
          for (int a = 0; a < BATCH; ++a)
            if (a == t) dot[a] = sum;
        }
      }
      if (row_there && p.dweights) {
        if (g >= BATCH) {
#pragma unroll
          for (int a = 0; a < BATCH; ++a)
            if (t == a && j + a < p.top) p.dweights[i * p.top + j + a] = pos[a] >= 0 ? dot[a] : 0.0f;
        }
      }
    }
  }
}

// ---- rows that no place has ------------------------------------------------------------------------------------------------------
// A bit for each sorted row that a place has; then zeros in the rows without one, a warp to 32 rows. Bounds: three short launches (with the one that clears the bits). All rows filled
// instead cost 0.27 ms for each GB, and the gradient of 65536 rows that writes this GB takes 0.41.
struct ClearParams {
  const int* where;
  long long places, n_sorted;
  unsigned* marks;  // [(n_sorted + 31) / 32]
  char* out;
  long long ld_out;  // bytes
  int width, es;     // bytes of a row and of an element
};
__global__ void __launch_bounds__(256) mark_places_kernel(const __grid_constant__ ClearParams p) {
  kernel_started();
  kernel_inputs_ready();
  for (long long e = (long long)blockIdx.x * 256 + threadIdx.x; e < p.places; e += (long long)gridDim.x * 256) {
    const int pos = __ldg(p.where + e);
    if (pos >= 0 && pos < p.n_sorted) atomicOr(p.marks + pos / 32, 1u << (pos % 32));
  }
}
__global__ void __launch_bounds__(256) clear_rows_kernel(const __grid_constant__ ClearParams p) {
  kernel_started();
  kernel_inputs_ready();
  const int lane = threadIdx.x & 31;
  for (long long word = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); word * 32 < p.n_sorted; word += (long long)gridDim.x * 8) {
    const long long left = p.n_sorted - word * 32;
    unsigned without = ~p.marks[word] & (left < 32 ? (1u << left) - 1 : 0xffffffffu);
    for (; without; without &= without - 1) {
      char* row = p.out + (word * 32 + __ffs(without) - 1) * p.ld_out;
      const int ahead = min((int)(-(uintptr_t)row & 15), p.width), units = (p.width - ahead) / 16;  // elements before the first whole 16 bytes, and those
      for (int u = lane; u < units; u += 32) *(uint4*)(row + ahead + u * 16) = make_uint4(0u, 0u, 0u, 0u);
      const int before = ahead / p.es, edges = (p.width - units * 16) / p.es;  // elements before and behind them
      for (int i = lane; i < edges; i += 32) {
        char* at = row + i * p.es + (i < before ? 0 : units * 16);
        if (p.es == 4) *(unsigned*)at = 0;
        else *(unsigned short*)at = 0;
      }
    }
  }
}

}  // namespace wpsgd
