// The places of it_experts_forward sorted by expert, and fp32 operands split into bf16 parts.
//
// A counting sort: counts per block and expert, their prefix sums, places written where they belong.  Few places take one block, more a cluster
// whose blocks read one another's counts, both in one launch; many a grid, in three.  The order of the places inside an expert differs from run to
// run (shared-memory atomics); no result depends on it: a row of a product is the same wherever in a tile it lies, and the places of a vertex are
// added in their own order.
#include <cooperative_groups.h>

#include "experts.cuh"

namespace cg = cooperative_groups;

namespace {

constexpr int PLAN_THREADS = 1024, PLAN_TILE = 128;
constexpr int PLAN_CLUSTER = 8, PLAN_CLUSTER_EXPERTS = 1024;   // (a cluster's blocks keep four words of shared memory an expert)
constexpr int PLAN_BLOCKS = 256;

struct PlanParams {
  int64_t places, per_block;
  int n_experts, blocks;
  const int32_t *ids;
  it_experts_plan q;
  int *status;
  char *zero_rows;        // out, where rows of no expert have to be zeroed here; else NULL
  int row_bytes;
};

// Exclusive prefix sum over the block's threads; *total: the sum.
__device__ __forceinline__ int block_scan(int v, int *warp_sums, int *total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int s = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, s, o);
    if (lane >= o) s += u;
  }
  __syncthreads();   // warp_sums of an earlier call have been read
  if (lane == 31) warp_sums[warp] = s;
  __syncthreads();
  if (warp == 0) {
    int w = warp_sums[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int u = __shfl_up_sync(0xffffffffu, w, o);
      if (lane >= o) w += u;
    }
    warp_sums[lane] = w;
  }
  __syncthreads();
  *total = warp_sums[31];
  return s - v + (warp ? warp_sums[warp - 1] : 0);
}

// count[e] (shared): places of every expert -> first position of every expert; tiles, padding and the number of tiles are written.
// first: as many words of shared memory.  part of parts: the share of the writing that this block does.
__device__ void lay_out(const PlanParams &p, int *count, int *first, int *warp_sums, int part = 0, int parts = 1) {
  int tiles_before = 0;
  for (int e0 = 0; e0 < p.n_experts; e0 += PLAN_THREADS) {
    const int e = e0 + threadIdx.x, tiles = e < p.n_experts ? (count[e] + PLAN_TILE - 1) / PLAN_TILE : 0;
    int total;
    const int at = tiles_before + block_scan(tiles, warp_sums, &total);
    if (e < p.n_experts) first[e] = at;
    tiles_before += total;
  }
  if (threadIdx.x == 0 && part == 0) *p.q.n_tiles = tiles_before;
  __syncthreads();
  for (int e = part + parts * (threadIdx.x >> 5); e < p.n_experts; e += parts * (PLAN_THREADS / 32)) {
    const int lane = threadIdx.x & 31, c = count[e], t0 = first[e], t1 = t0 + (c + PLAN_TILE - 1) / PLAN_TILE;
    for (int t = t0 + lane; t < t1; t += 32) p.q.tile_expert[t] = e;
    for (int64_t i = (int64_t)t0 * PLAN_TILE + c + lane; i < (int64_t)t1 * PLAN_TILE; i += 32) p.q.order[i] = -1;
  }
  __syncthreads();
  for (int e = threadIdx.x; e < p.n_experts; e += PLAN_THREADS) count[e] = first[e] * PLAN_TILE;
}

__device__ __forceinline__ void zero_row(const PlanParams &p, int64_t v) {
  uint4 *row = reinterpret_cast<uint4 *>(p.zero_rows + v * p.row_bytes);
  for (int i = 0; i < p.row_bytes / 16; ++i) row[i] = make_uint4(0, 0, 0, 0);
}

__global__ void __launch_bounds__(PLAN_THREADS) plan_one_kernel(const PlanParams p) {
  it_wait_prior();
  it_allow_next();
  extern __shared__ int plan_smem[];
  int *count = plan_smem;
  __shared__ int warp_sums[32];
  if (threadIdx.x == 0) *p.status = 0;
  for (int e = threadIdx.x; e < p.n_experts; e += PLAN_THREADS) count[e] = 0;
  __syncthreads();
  for (int64_t i = threadIdx.x; i < p.places; i += PLAN_THREADS) {
    const int e = p.ids[i];
    if ((unsigned)e < (unsigned)p.n_experts) atomicAdd(&count[e], 1);
  }
  __syncthreads();
  lay_out(p, count, count + p.n_experts, warp_sums);
  __syncthreads();
  for (int64_t i = threadIdx.x; i < p.places; i += PLAN_THREADS) {
    const int e = p.ids[i];
    if ((unsigned)e < (unsigned)p.n_experts) {
      const int at = atomicAdd(&count[e], 1);
      p.q.order[at] = (int32_t)i;
      p.q.position[i] = at;
    } else if (p.zero_rows) {
      zero_row(p, i);
    }
  }
}

// f(place, its id, whether it is one) for the places of this block, by whole warps; the ids of four rounds are fetched at once.
template <typename F>
__device__ __forceinline__ void walk_places(const PlanParams &p, F f) {
  constexpr int AHEAD = 4;
  const int lane = threadIdx.x & 31;
  const int64_t lo = blockIdx.x * p.per_block, hi = lo + p.per_block < p.places ? lo + p.per_block : p.places;
  for (int64_t i0 = lo + (threadIdx.x & ~31); i0 < hi; i0 += AHEAD * PLAN_THREADS) {
    int e[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int64_t i = i0 + u * PLAN_THREADS + lane;
      e[u] = i < hi ? p.ids[i] : -1;
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int64_t i = i0 + u * PLAN_THREADS + lane;
      if (i - lane < hi) f(i, e[u], i < hi);
    }
  }
}

// Adds the places of this block to count[e] (shared).
__device__ __forceinline__ void count_block(const PlanParams &p, int *count) {
  const int lane = threadIdx.x & 31;
  walk_places(p, [&](int64_t, int e, bool) {
    const unsigned same = __match_any_sync(0xffffffffu, e);   // one addition per expert and warp
    if ((unsigned)e < (unsigned)p.n_experts && lane == __ffs(same) - 1) atomicAdd(&count[e], __popc(same));
  });
}

// Writes the places of this block where they belong: next[e] (shared) is the next position of expert e.
__device__ __forceinline__ void place_block(const PlanParams &p, int *next) {
  const int lane = threadIdx.x & 31;
  walk_places(p, [&](int64_t i, int e, bool in) {
    const bool real = (unsigned)e < (unsigned)p.n_experts;
    const unsigned same = __match_any_sync(0xffffffffu, e);
    const int leader = __ffs(same) - 1;
    int at = 0;
    if (real && lane == leader) at = atomicAdd(&next[e], __popc(same));
    at = __shfl_sync(0xffffffffu, at, leader) + __popc(same & ((1u << lane) - 1u));
    if (real) {
      p.q.order[at] = (int32_t)i;
      p.q.position[i] = at;
    } else if (p.zero_rows && in) {
      zero_row(p, i);
    }
  });
}

// counts | of all blocks | first tiles | places of the blocks before, in shared memory.
__global__ void __launch_bounds__(PLAN_THREADS) plan_cluster_kernel(const PlanParams p) {
  it_allow_next();
  it_wait_prior();
  extern __shared__ int plan_smem[];
  __shared__ int warp_sums[32];
  cg::cluster_group cluster = cg::this_cluster();
  int *count = plan_smem, *total = count + p.n_experts, *first = total + p.n_experts, *before = first + p.n_experts;
  if (blockIdx.x == 0 && threadIdx.x == 0) *p.status = 0;
  for (int e = threadIdx.x; e < p.n_experts; e += PLAN_THREADS) count[e] = 0;
  __syncthreads();
  count_block(p, count);
  cluster.sync();
  for (int e = threadIdx.x; e < p.n_experts; e += PLAN_THREADS) {
    int sum = 0, mine = 0;
#pragma unroll
    for (int b = 0; b < PLAN_CLUSTER; ++b) {
      if (b == (int)blockIdx.x) mine = sum;
      sum += cluster.map_shared_rank(count, b)[e];
    }
    total[e] = sum;
    before[e] = mine;
  }
  cluster.sync();   // nobody's counts go before they are read
  lay_out(p, total, first, warp_sums, (int)blockIdx.x, PLAN_CLUSTER);
  __syncthreads();
  for (int e = threadIdx.x; e < p.n_experts; e += PLAN_THREADS) total[e] += before[e];
  __syncthreads();
  place_block(p, total);
}

__global__ void __launch_bounds__(PLAN_THREADS) plan_count_kernel(const PlanParams p) {
  it_allow_next();
  it_wait_prior();
  extern __shared__ int plan_smem[];
  if (blockIdx.x == 0 && threadIdx.x == 0) *p.status = 0;
  for (int e = threadIdx.x; e < p.n_experts; e += PLAN_THREADS) plan_smem[e] = 0;
  __syncthreads();
  count_block(p, plan_smem);
  __syncthreads();
  for (int e = threadIdx.x; e < p.n_experts; e += PLAN_THREADS) p.q.counts[(int64_t)blockIdx.x * p.n_experts + e] = plan_smem[e];
}

// Counts of every block -> first position of every block's places, expert by expert (a warp each).
__global__ void __launch_bounds__(PLAN_THREADS) plan_scan_kernel(const PlanParams p) {
  it_allow_next();
  it_wait_prior();
  extern __shared__ int plan_smem[];
  __shared__ int warp_sums[32];
  const int lane = threadIdx.x & 31;
  for (int e = threadIdx.x >> 5; e < p.n_experts; e += PLAN_THREADS / 32) {
    int before = 0;
    for (int b0 = 0; b0 < p.blocks; b0 += 32) {
      const int b = b0 + lane, c = b < p.blocks ? p.q.counts[(int64_t)b * p.n_experts + e] : 0;
      int s = c;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += u;
      }
      if (b < p.blocks) p.q.counts[(int64_t)b * p.n_experts + e] = before + s - c;
      before += __shfl_sync(0xffffffffu, s, 31);
    }
    if (lane == 0) plan_smem[e] = before;
  }
  __syncthreads();
  lay_out(p, plan_smem, plan_smem + p.n_experts, warp_sums);
  __syncthreads();
  for (int64_t i = threadIdx.x; i < (int64_t)p.blocks * p.n_experts; i += PLAN_THREADS) p.q.counts[i] += plan_smem[i % p.n_experts];
}

__global__ void __launch_bounds__(PLAN_THREADS) plan_place_kernel(const PlanParams p) {
  it_allow_next();
  it_wait_prior();
  extern __shared__ int plan_smem[];
  for (int e = threadIdx.x; e < p.n_experts; e += PLAN_THREADS) plan_smem[e] = p.q.counts[(int64_t)blockIdx.x * p.n_experts + e];
  __syncthreads();
  place_block(p, plan_smem);
}

// The whole of it_experts_forward on bf16 64-256-64, us (captured), one block / a cluster / a grid: 8 experts, 3000 places 19.1 / 19.9 / -, 6000
// 20.5 / 20.2 / -, 16000 25.4 / 22.1 / -, 24000 - / 30.8 / 33.1, 40000 - / 40.7 / 41.3, 80000 - / 62.0 / 59.7; 256 experts, 1400 30.7 / 27.8 / -,
// 16000 41.3 / 32.9 / -, 40000 - / 55.0 / 64.9, 80000 - / 81.5 / 86.2, 130000 - / 112.1 / 111.4.
enum PlanForm { PLAN_BLOCK, PLAN_CLUSTERED, PLAN_GRID };
PlanForm plan_form(int64_t places, int n_experts) {
  if (n_experts > PLAN_CLUSTER_EXPERTS) return places <= 16384 ? PLAN_BLOCK : PLAN_GRID;
  if (places <= 6144 && n_experts <= 32) return PLAN_BLOCK;
  return places <= 49152 + 128 * (int64_t)(n_experts < 256 ? n_experts : 256) ? PLAN_CLUSTERED : PLAN_GRID;
}

int plan_blocks(int64_t places) {
  const int64_t want = (places + 4 * PLAN_THREADS - 1) / (4 * PLAN_THREADS);
  return (int)(want < PLAN_BLOCKS ? want : PLAN_BLOCKS);
}

// ----------------------------------------------------------------------------- bf16 parts
__device__ __forceinline__ void split3(float v, uint32_t &a, uint32_t &b, uint32_t &c) {
  const uint32_t u = __float_as_uint(v);
  a = u >> 16;
  const float r1 = v - __uint_as_float(u & 0xffff0000u);   // exact (NaN of an infinity: the product is then NaN)
  const uint32_t u1 = __float_as_uint(r1);
  b = u1 >> 16;
  c = __float_as_uint(r1 - __uint_as_float(u1 & 0xffff0000u)) >> 16;
}

// Rows of x in the order of the positions: f(position, vertex, piece) for every piece of every row that has a place, a group of lanes a row.
template <typename F>
__device__ __forceinline__ void it_experts_rows_walk(const int32_t *order, const int32_t *n_tiles, int64_t tiles_max, int top_k, int pieces, F f) {
  int64_t tiles = *n_tiles;
  tiles = tiles < tiles_max ? tiles : tiles_max;
  int lanes = 1;
  while (lanes < 32 && lanes < pieces) lanes <<= 1;
  const int per_block = 256 / lanes, gl = threadIdx.x % lanes;
  for (int64_t r = blockIdx.x * (int64_t)per_block + threadIdx.x / lanes; r < tiles * PLAN_TILE; r += (int64_t)gridDim.x * per_block) {
    const int place = order[r];
    if (place < 0) continue;
    const int64_t v = place / top_k;
    for (int c = gl; c < pieces; c += lanes) f(r, v, c);
  }
}

__device__ __forceinline__ void split_store(const float4 &v, __nv_bfloat16 *dst, int64_t part) {
  uint32_t w[3][4];
  split3(v.x, w[0][0], w[1][0], w[2][0]); split3(v.y, w[0][1], w[1][1], w[2][1]);
  split3(v.z, w[0][2], w[1][2], w[2][2]); split3(v.w, w[0][3], w[1][3], w[2][3]);
#pragma unroll
  for (int k = 0; k < 3; ++k) *reinterpret_cast<uint2 *>(dst + k * part) = make_uint2(w[k][0] | (w[k][1] << 16), w[k][2] | (w[k][3] << 16));
}

// blockIdx.y: the matrix of weights, or (the last one) the rows of x.
__global__ void __launch_bounds__(256) parts_kernel(const __grid_constant__ it_experts_parts q) {
  it_allow_next();
  it_wait_prior();
  if ((int)blockIdx.y < q.count) {
    const float *src = blockIdx.y == 0 ? q.src[0] : q.src[1];
    __nv_bfloat16 *dst = blockIdx.y == 0 ? q.dst[0] : q.dst[1];
    const int64_t n = blockIdx.y == 0 ? q.elems[0] : q.elems[1];
    for (int64_t i = (blockIdx.x * (int64_t)blockDim.x + threadIdx.x) * 4; i < n; i += (int64_t)gridDim.x * blockDim.x * 4)
      split_store(*reinterpret_cast<const float4 *>(src + i), dst + i, n);
    return;
  }
  it_experts_rows_walk(q.order, q.n_tiles, q.tiles_max, q.top_k, q.row / 4, [&](int64_t r, int64_t v, int c) {
    split_store(*reinterpret_cast<const float4 *>(q.x + v * q.row + c * 4), q.x_parts + r * q.row + c * 4, q.tiles_max * PLAN_TILE * q.row);
  });
}

__global__ void __launch_bounds__(256) rows_kernel(const uint4 *x, uint4 *to, int row16, int top_k, const int32_t *order, const int32_t *n_tiles, int64_t tiles_max) {
  it_allow_next();
  it_wait_prior();
  it_experts_rows_walk(order, n_tiles, tiles_max, top_k, row16, [&](int64_t r, int64_t v, int c) { to[r * row16 + c] = x[v * row16 + c]; });
}

}  // namespace

int64_t it_experts_tiles_max(int64_t places, int n_experts) { return places / PLAN_TILE + (places < n_experts ? places : n_experts); }
size_t it_experts_count_words(int64_t places, int n_experts) {
  return plan_form(places, n_experts) != PLAN_GRID ? 0 : (size_t)plan_blocks(places) * (size_t)n_experts;
}

it_status it_launch_experts_plan(const it_experts_args &a, const it_experts_plan &q, cudaStream_t st) {
  PlanParams p{};
  p.places = a.n * a.d.top_k; p.n_experts = a.d.n_experts; p.ids = a.ids; p.q = q; p.status = a.status;
  if (a.d.top_k == 1) { p.zero_rows = (char *)a.out; p.row_bytes = a.d.out_dim * it_dtype_size(a.d.feat_dtype); }
  const size_t smem = (size_t)p.n_experts * 8;
  const double bytes = 4.0 * p.places;
  const PlanForm form = plan_form(p.places, p.n_experts);
  if (form == PLAN_BLOCK) {
    IT_LAUNCH(IT_K_EXPERT_PLAN, 3 * bytes, 0, st, IT_CUDA_TRY(it_launch_pdl(plan_one_kernel, dim3(1), dim3(PLAN_THREADS), smem, st, p)));
    return IT_OK;
  }
  if (form == PLAN_CLUSTERED) {
    p.per_block = (p.places + PLAN_CLUSTER - 1) / PLAN_CLUSTER;
    cudaLaunchAttribute attr[2] = {};
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = PLAN_CLUSTER; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(PLAN_CLUSTER); cfg.blockDim = dim3(PLAN_THREADS); cfg.dynamicSmemBytes = 2 * smem; cfg.stream = st; cfg.attrs = attr; cfg.numAttrs = 2;
    IT_LAUNCH(IT_K_EXPERT_PLAN, 3 * bytes, 0, st, IT_CUDA_TRY((cudaLaunchKernelEx(&cfg, plan_cluster_kernel, p))));
    return IT_OK;
  }
  p.blocks = plan_blocks(p.places);
  p.per_block = (p.places + p.blocks - 1) / p.blocks;
  IT_LAUNCH(IT_K_EXPERT_PLAN, bytes, 0, st, IT_CUDA_TRY(it_launch_pdl(plan_count_kernel, dim3(p.blocks), dim3(PLAN_THREADS), smem, st, p)));
  IT_LAUNCH(IT_K_EXPERT_PLAN, 0, 0, st, IT_CUDA_TRY(it_launch_pdl(plan_scan_kernel, dim3(1), dim3(PLAN_THREADS), smem, st, p)));
  IT_LAUNCH(IT_K_EXPERT_PLAN, 3 * bytes, 0, st, IT_CUDA_TRY(it_launch_pdl(plan_place_kernel, dim3(p.blocks), dim3(PLAN_THREADS), smem, st, p)));
  return IT_OK;
}

it_status it_launch_experts_parts(const it_experts_parts &q, int sms, cudaStream_t st) {
  const int64_t rows = q.tiles_max * PLAN_TILE * q.row;
  int64_t most = rows, total = rows;
  for (int i = 0; i < q.count; ++i) { most = q.elems[i] > most ? q.elems[i] : most; total += q.elems[i]; }
  const int64_t blocks = (most / 4 + 255) / 256, cap = (int64_t)sms * 8;
  IT_LAUNCH(IT_K_EXPERT_PARTS, 10.0 * total, 0, st,
            IT_CUDA_TRY(it_launch_pdl(parts_kernel, dim3((unsigned)(blocks < cap ? blocks : cap), q.count + 1), dim3(256), 0, st, q)));
  return IT_OK;
}

it_status it_launch_experts_rows(const it_experts_args &a, const it_experts_plan &q, void *to, cudaStream_t st) {
  const int row16 = a.d.in_dim * (a.d.in_dtype == IT_E4M3 ? 1 : it_dtype_size(a.d.in_dtype)) / 16;
  const int64_t blocks = (q.tiles_max * PLAN_TILE * row16 + 255) / 256, cap = (int64_t)a.sms * 16;
  IT_LAUNCH(IT_K_EXPERT_PARTS, 32.0 * a.n * a.d.top_k * row16, 0, st,
            IT_CUDA_TRY(it_launch_pdl(rows_kernel, dim3((unsigned)(blocks < cap ? blocks : cap)), dim3(256), 0, st, (const uint4 *)a.x, (uint4 *)to, row16, a.d.top_k,
                                      (const int32_t *)q.order, (const int32_t *)q.n_tiles, q.tiles_max)));
  return IT_OK;
}
