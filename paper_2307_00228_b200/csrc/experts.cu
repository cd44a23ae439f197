// it_experts_forward: checks, scratch, the form for few places (a product per place), and the sum over the places of a vertex.
#include <cooperative_groups.h>
#include <cuda_fp8.h>
#include <math.h>

#include "experts.cuh"

namespace cg = cooperative_groups;

namespace {

// ----------------------------------------------------------------------------- few places: a product per place
// A place is one (vertex, expert).  With few of them every weight is read about once and nothing else counts, so this is a matter of
// having many loads of W in flight at once: a block takes 128 bytes of a row of W (8 lanes x 16 bytes) and a share of its rows, the
// blocks of a cluster share the rows between them and add up over distributed shared memory, in their order.  fp32 throughout: the hidden row is not rounded.
constexpr int ROWS_THREADS = 256, ROWS_WARPS = ROWS_THREADS / 32, ROWS_COL_LANES = 8, ROWS_UNROLL = 4;
constexpr int ROWS_STEP = ROWS_WARPS * (32 / ROWS_COL_LANES);   // rows of W that a block reads side by side

struct RowsParams {
  int64_t units;            // places (first product) or vertices (second)
  int k, n_experts, K, cols, chunks, act, gated_at;   // gated_at: first column of the second half (0: not gated)
  const void *x;            // rows that are multiplied: of x (first product) or fp32 hidden rows
  const float *x_scale;
  const int32_t *ids;
  const float *weights;
  const void *W;
  const float *bias, *w_scale;
  int w_cols;               // columns of W
  float *hidden;            // first product: [places, cols]
  void *out;                // second product
  int *status;
};

__device__ __forceinline__ float elem_f32(const float *p) { return *p; }
__device__ __forceinline__ float elem_f32(const __nv_bfloat16 *p) { return __bfloat162float(*p); }
__device__ __forceinline__ float elem_f32(const __nv_fp8_e4m3 *p) { return float(*p); }

template <typename TW> struct WVec { static constexpr int N = 16 / (int)sizeof(TW); };
template <typename TW> __device__ __forceinline__ void w_to_f32(const uint4 &q, float (&v)[WVec<TW>::N]) {
  if constexpr (sizeof(TW) == 1) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[i >> 1] >> (16 * (i & 1))), __NV_E4M3);
      const float2 f = __half22float2(__half2(h));
      v[2 * i] = f.x; v[2 * i + 1] = f.y;
    }
  } else {
    vec_to_f32(q, v);
  }
}

// 16 bytes, or zeros: a load under a predicate, so that a thread's loads go out one behind the other without a branch in between (C++ for the same, with which
// they did not: bf16 128-512-128 64 places 12.1 us / 10.7, fp32 512-64-512 64 places 13.0 / 11.7).
__device__ __forceinline__ uint4 load_if(bool in, const void *from) {
  uint4 q = make_uint4(0, 0, 0, 0);
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %5, 0;\n\t@p ld.global.v4.b32 {%0, %1, %2, %3}, [%4];\n\t}"
               : "+r"(q.x), "+r"(q.y), "+r"(q.z), "+r"(q.w)
               : "l"(from), "r"((int)in));
  return q;
}

// (blocks an SM: fp32 256-1024-256 128 places 51.7 us with two, 48.3 with four; gated 768-1024-768 16 places 30.4 with two, 27.1 with three)
// SECOND: the rows of W follow one another place by place of the vertex: row i is row i % K of the place i / K.
template <typename TX, typename TW, bool SECOND, bool GATED, typename TO>
__global__ void __launch_bounds__(ROWS_THREADS, GATED ? 3 : 4) expert_rows_kernel(const RowsParams p) {
  constexpr int N = WVec<TW>::N, CB = ROWS_COL_LANES * N, PARTS = GATED ? 2 : 1;
  __shared__ float part[ROWS_WARPS][PARTS * CB];
  __shared__ float total[PARTS * CB];
  cg::cluster_group cluster = cg::this_cluster();
  const int share = (int)cluster.block_rank(), shares = (int)cluster.num_blocks();
  const int64_t id = blockIdx.x / shares, unit = id / p.chunks;
  const int c0 = (int)(id % p.chunks) * CB;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, cl = lane % ROWS_COL_LANES, rl = lane / ROWS_COL_LANES;
  const int col = c0 + cl * N;
  if (SECOND) {
    it_allow_next();
    // the weights are on their way while the hidden rows are made (the first product starts this kernel when all before it is over)
    // (of few vertices: of many the copies are in the way, fp32 256-1024-256, 256 places 78.6 -> 88 us)
    if (p.units <= 8 && cl == 0 && col < p.cols)
      for (int j = 0; j < p.k; ++j) {
        const int e = p.ids[unit * p.k + j];
        if ((unsigned)e >= (unsigned)p.n_experts) continue;
        const int lo = (int)((int64_t)p.K * share / shares), hi = (int)((int64_t)p.K * (share + 1) / shares);
        for (int r = lo + warp * (32 / ROWS_COL_LANES) + rl; r < hi; r += ROWS_STEP)
          asm volatile("prefetch.global.L2 [%0];" ::"l"(reinterpret_cast<const TW *>(p.W) + ((int64_t)e * p.K + r) * p.w_cols + col));
      }
    it_wait_prior();   // the hidden rows
  } else {
    it_wait_prior();
    it_allow_next();   // only now: what the next kernel reads besides the hidden rows is then there
    if (blockIdx.x == 0 && threadIdx.x == 0) *p.status = 0;
  }
  const int64_t place0 = SECOND ? unit * p.k : unit;
  if (!SECOND && (unsigned)p.ids[place0] >= (unsigned)p.n_experts) return;   // (all blocks of the cluster)

  float acc[PARTS][N];
#pragma unroll
  for (int g = 0; g < PARTS; ++g)
#pragma unroll
    for (int i = 0; i < N; ++i) acc[g][i] = 0.f;
  for (int j = 0; j < (SECOND ? p.k : 1); ++j) {
    const int64_t place = place0 + j;
    const int e = p.ids[place];
    if ((unsigned)e >= (unsigned)p.n_experts) continue;
    // this block's share of the K rows
    const int lo = (int)((int64_t)p.K * share / shares), hi = (int)((int64_t)p.K * (share + 1) / shares);
    const TX *x = reinterpret_cast<const TX *>(p.x) + (SECOND ? place : place / p.k) * p.K;
    const TW *w = reinterpret_cast<const TW *>(p.W) + (int64_t)e * p.K * p.w_cols + col;
    const float f = SECOND ? p.weights[place] : 1.f;
    for (int r0 = lo + warp * (32 / ROWS_COL_LANES) + rl; r0 < hi; r0 += ROWS_STEP * ROWS_UNROLL) {
      uint4 q[PARTS][ROWS_UNROLL];
      float xv[ROWS_UNROLL];
#pragma unroll
      for (int u = 0; u < ROWS_UNROLL; ++u) {
        const int r = r0 + u * ROWS_STEP;
        const bool in = r < hi && col < p.cols;
        xv[u] = in ? elem_f32(x + r) * f : 0.f;
#pragma unroll
        for (int g = 0; g < PARTS; ++g)
          q[g][u] = load_if(in, w + (int64_t)r * p.w_cols + g * p.gated_at);
      }
#pragma unroll
      for (int u = 0; u < ROWS_UNROLL; ++u) {
        if (r0 + u * ROWS_STEP >= hi) break;
#pragma unroll
        for (int g = 0; g < PARTS; ++g) {
          float v[N];
          w_to_f32<TW>(q[g][u], v);
#pragma unroll
          for (int i = 0; i < N; ++i) acc[g][i] = fmaf(xv[u], v[i], acc[g][i]);
        }
      }
    }
    if (SECOND && p.bias && share == 0 && warp == 0 && rl == 0 && col < p.cols) {
#pragma unroll
      for (int i = 0; i < N; ++i) acc[0][i] = fmaf(f, p.bias[(int64_t)e * p.cols + col + i], acc[0][i]);
    }
  }
#pragma unroll
  for (int g = 0; g < PARTS; ++g)
#pragma unroll
    for (int i = 0; i < N; ++i) {
#pragma unroll
      for (int o = ROWS_COL_LANES; o < 32; o <<= 1) acc[g][i] += __shfl_xor_sync(0xffffffffu, acc[g][i], o);
      if (rl == 0) part[warp][g * CB + cl * N + i] = acc[g][i];
    }
  __syncthreads();
  for (int c = threadIdx.x; c < PARTS * CB; c += ROWS_THREADS) {
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < ROWS_WARPS; ++w) s += part[w][c];
    total[c] = s;
  }
  cluster.sync();
  if (share == 0) {
    for (int c = threadIdx.x; c < CB && c0 + c < p.cols; c += ROWS_THREADS) {
      float s[PARTS];
#pragma unroll
      for (int g = 0; g < PARTS; ++g) {
        s[g] = 0.f;
        for (int b = 0; b < shares; ++b) s[g] += cluster.map_shared_rank(total, b)[g * CB + c];
      }
      if constexpr (SECOND) {
        reinterpret_cast<TO *>(p.out)[unit * p.cols + c0 + c] = TO(s[0]);
      } else {
        const int e = p.ids[place0];
        const float xs = p.x_scale ? p.x_scale[place0 / p.k] : 1.f;
#pragma unroll
        for (int g = 0; g < PARTS; ++g) {
          const int64_t at = (int64_t)e * p.w_cols + g * p.gated_at + c0 + c;
          if (p.w_scale) s[g] *= xs * p.w_scale[at];
          if (p.bias) s[g] += p.bias[at];
        }
        const float a = it_expert_act(s[0], p.act);
        p.hidden[place0 * p.cols + c0 + c] = GATED ? a * s[PARTS - 1] : a;
      }
    }
  }
  cluster.sync();   // nobody's totals go before they are read
}

template <typename TX, typename TW, bool SECOND, bool GATED, typename TO>
it_status launch_rows(RowsParams p, int sms, double bytes, double flops, cudaStream_t st) {
  constexpr int CB = ROWS_COL_LANES * WVec<TW>::N;
  p.chunks = (p.cols + CB - 1) / CB;
  // shares of about 128 rows, as long as the blocks still run side by side (eight of 256 threads an SM)
  const int64_t base = p.units * p.chunks, rows = (int64_t)p.K * (SECOND ? p.k : 1);
  int shares = 1;
  while (shares < 8 && rows > 128 * (int64_t)shares && base * shares * 2 <= (int64_t)sms * 8) shares *= 2;
  IT_REQUIRE(base * shares <= INT32_MAX, IT_ERR_UNSUPPORTED, "too many places for one launch");
  cudaLaunchAttribute attr[2] = {};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)shares; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(base * shares)); cfg.blockDim = dim3(ROWS_THREADS); cfg.stream = st; cfg.attrs = attr; cfg.numAttrs = 2;
  IT_LAUNCH(IT_K_EXPERT_ROWS, bytes, flops, st, IT_CUDA_TRY((cudaLaunchKernelEx(&cfg, expert_rows_kernel<TX, TW, SECOND, GATED, TO>, p))));
  return IT_OK;
}

// ----------------------------------------------------------------------------- the places of a vertex added up
// out[v] = sum_j weights[v, j] * y[position of place (v, j)], in the order of j.  y: fp32 rows, by place (position NULL) or where the
// product left them.  Bound by DRAM: a read of every fp32 row, a write of the result.
struct CombineParams {
  int64_t n;
  int k, n_experts, dim;
  const float *y;
  const int32_t *position;
  const int32_t *ids;
  const float *weights;
  void *out;
};
template <typename T>
__global__ void __launch_bounds__(256) expert_combine_kernel(const CombineParams p) {
  it_allow_next();
  it_wait_prior();
  constexpr int N = kVec<T>;
  const int per = p.dim / N;
  const int64_t total = p.n * per;
  for (int64_t i = blockIdx.x * (int64_t)blockDim.x + threadIdx.x; i < total; i += (int64_t)gridDim.x * blockDim.x) {
    const int64_t v = i / per;
    const int c = (int)(i - v * per) * N;
    float acc[N];
#pragma unroll
    for (int q = 0; q < N; ++q) acc[q] = 0.f;
    for (int j = 0; j < p.k; ++j) {
      const int64_t place = v * p.k + j;
      if ((unsigned)p.ids[place] >= (unsigned)p.n_experts) continue;
      const float w = p.weights[place];
      const float4 *row = reinterpret_cast<const float4 *>(p.y + (p.position ? (int64_t)p.position[place] : place) * p.dim + c);
#pragma unroll
      for (int q = 0; q < N / 4; ++q) {
        const float4 f = row[q];
        acc[4 * q] = fmaf(w, f.x, acc[4 * q]); acc[4 * q + 1] = fmaf(w, f.y, acc[4 * q + 1]);
        acc[4 * q + 2] = fmaf(w, f.z, acc[4 * q + 2]); acc[4 * q + 3] = fmaf(w, f.w, acc[4 * q + 3]);
      }
    }
    *reinterpret_cast<uint4 *>(reinterpret_cast<T *>(p.out) + v * p.dim + c) = f32_to_vec(acc);
  }
}

it_status launch_combine(const it_experts_args &a, const float *y, const int32_t *position, cudaStream_t st) {
  const CombineParams p{a.n, a.d.top_k, a.d.n_experts, a.d.out_dim, y, position, a.ids, a.weights, a.out};
  const bool f32 = a.d.feat_dtype == IT_F32;
  const int64_t threads = a.n * (a.d.out_dim / (f32 ? 4 : 8)), blocks = (threads + 255) / 256, most = (int64_t)a.sms * 32;
  const dim3 grid((unsigned)(blocks < most ? blocks : most));
  const double bytes = (double)a.n * a.d.out_dim * (4.0 * a.d.top_k + it_dtype_size(a.d.feat_dtype));
  if (f32) IT_LAUNCH(IT_K_EXPERT_COMBINE, bytes, 0, st, IT_CUDA_TRY(it_launch_pdl(expert_combine_kernel<float>, grid, dim3(256), 0, st, p)));
  else IT_LAUNCH(IT_K_EXPERT_COMBINE, bytes, 0, st, IT_CUDA_TRY(it_launch_pdl(expert_combine_kernel<__nv_bfloat16>, grid, dim3(256), 0, st, p)));
  return IT_OK;
}

it_status few_places(const it_experts_args &a, float *hidden, cudaStream_t st) {
  const it_experts_desc &d = a.d;
  const int64_t places = a.n * d.top_k;
  RowsParams p{};
  p.k = d.top_k; p.n_experts = d.n_experts; p.ids = a.ids; p.weights = a.weights; p.act = d.act; p.status = a.status;
  p.units = places; p.K = d.in_dim; p.cols = d.hidden_dim > 0 ? d.hidden_dim : d.out_dim; p.w_cols = a.n1; p.gated_at = d.gated ? d.hidden_dim : 0;
  p.x = a.x; p.x_scale = a.x_scale; p.W = d.W1; p.bias = d.b1; p.w_scale = d.w1_scale; p.hidden = hidden;
  const double f1 = 2.0 * places * d.in_dim * a.n1, f2 = 2.0 * places * d.hidden_dim * d.out_dim;
  const bool f32 = d.feat_dtype == IT_F32;
  if (d.in_dtype == IT_E4M3) {
    if (d.gated) IT_TRY((launch_rows<__nv_fp8_e4m3, __nv_fp8_e4m3, false, true, float>(p, a.sms, 0, f1, st)));
    else IT_TRY((launch_rows<__nv_fp8_e4m3, __nv_fp8_e4m3, false, false, float>(p, a.sms, 0, f1, st)));
  } else if (f32) {
    if (d.gated) IT_TRY((launch_rows<float, float, false, true, float>(p, a.sms, 0, f1, st)));
    else IT_TRY((launch_rows<float, float, false, false, float>(p, a.sms, 0, f1, st)));
  } else {
    if (d.gated) IT_TRY((launch_rows<__nv_bfloat16, __nv_bfloat16, false, true, float>(p, a.sms, 0, f1, st)));
    else IT_TRY((launch_rows<__nv_bfloat16, __nv_bfloat16, false, false, float>(p, a.sms, 0, f1, st)));
  }
  if (d.hidden_dim == 0) return launch_combine(a, hidden, nullptr, st);
  p.units = a.n; p.K = d.hidden_dim; p.cols = p.w_cols = d.out_dim; p.gated_at = 0;
  p.x = hidden; p.x_scale = nullptr; p.W = d.W2; p.bias = d.b2; p.w_scale = nullptr; p.out = a.out;
  if (f32) return launch_rows<float, float, true, false, float>(p, a.sms, 0, f2, st);
  return launch_rows<float, __nv_bfloat16, true, false, __nv_bfloat16>(p, a.sms, 0, f2, st);
}

// ----------------------------------------------------------------------------- checks and scratch
constexpr int kMaxDim = 1 << 16, kMaxExperts = 4096;

it_status check(const it_experts_desc *d, int64_t n) {
  IT_REQUIRE(d != nullptr, IT_ERR_INVALID_ARG, "description is NULL");
  IT_REQUIRE(d->feat_dtype == IT_F32 || d->feat_dtype == IT_BF16, IT_ERR_INVALID_ARG, "bad feat_dtype");
  IT_REQUIRE(d->in_dtype == d->feat_dtype || d->in_dtype == IT_E4M3, IT_ERR_INVALID_ARG, "in_dtype must be feat_dtype or IT_E4M3");
  IT_REQUIRE(d->in_dtype != IT_E4M3 || d->feat_dtype == IT_BF16, IT_ERR_UNSUPPORTED, "states of IT_E4M3 go with feat_dtype IT_BF16");
  IT_REQUIRE(d->act >= IT_ACT_NONE && d->act <= IT_ACT_SILU, IT_ERR_INVALID_ARG, "bad activation %d", (int)d->act);
  IT_REQUIRE(n >= 0 && d->n_experts >= 1 && d->top_k >= 1, IT_ERR_INVALID_ARG, "bad shape (%lld vertices, %d experts, top_k %d)", (long long)n, d->n_experts, d->top_k);
  IT_REQUIRE(d->in_dim > 0 && d->hidden_dim >= 0 && d->out_dim > 0, IT_ERR_INVALID_ARG, "dims must be positive");
  IT_REQUIRE(!d->gated || d->hidden_dim > 0, IT_ERR_INVALID_ARG, "a gate needs hidden_dim > 0");
  const int step1 = d->in_dtype == IT_E4M3 ? 16 : 8, first = d->hidden_dim > 0 ? d->hidden_dim : d->out_dim;
  IT_REQUIRE(d->in_dim % step1 == 0 && first % step1 == 0 && d->hidden_dim % 8 == 0 && d->out_dim % 8 == 0, IT_ERR_INVALID_ARG,
             "widths must be multiples of 8, rows of e4m3 of 16 (in %d, hidden %d, out %d)", d->in_dim, d->hidden_dim, d->out_dim);
  IT_REQUIRE(d->in_dim <= kMaxDim && d->hidden_dim <= kMaxDim && d->out_dim <= kMaxDim, IT_ERR_UNSUPPORTED, "more than %d columns", kMaxDim);
  IT_REQUIRE(d->n_experts <= kMaxExperts, IT_ERR_UNSUPPORTED, "%d experts, at most %d", d->n_experts, kMaxExperts);
  const int64_t places = INT32_MAX / (d->feat_dtype == IT_F32 ? 3 : 1) - 128 * (int64_t)d->n_experts;
  IT_REQUIRE(places > 0 && n <= places / d->top_k, IT_ERR_UNSUPPORTED, "%lld vertices with %d places each: too many rows for 32 bits", (long long)n, d->top_k);
  return IT_OK;
}

// Few places keep the form by place, whose time grows with the weights that its places read: up to so many.  By place against sorted, us (captured): bf16 64-256-64
// 64 places 8.6 / 10.5, 128 9.3 / 10.7; 256-256 64 6.2 / 9.7, 128 10.1 / 9.7; 128-512-128 (64 experts) 64 11.9 / 15.2, 128 18.6 / 15.5; 256-1024-256
// 64 21.5 / 24.0, 128 33.5 / 24.0; gated 768-1024-768 16 27.1 / 30.0, 32 41.6 / 32.1.  fp32, whose sorted form splits all weights first:
// 64-256-64 128 12.6 / 20.5, 192 19.7 / 20.6, 256 23.2 / 20.9, 448 32.3 / 21.8; 256-1024-256 192 72 / 76, 256 86 / 77; of many experts 512-64-512 (64) 256 23.3 / 47.1.
int64_t most_few(const it_experts_desc &d) {
  const bool f32 = d.feat_dtype == IT_F32;
  const int64_t first = d.hidden_dim > 0 ? (int64_t)d.hidden_dim * (d.gated ? 2 : 1) : d.out_dim;
  const int64_t bytes = (int64_t)d.in_dim * first * (f32 ? 4 : (d.in_dtype == IT_E4M3 ? 1 : 2)) + (int64_t)d.hidden_dim * d.out_dim * (f32 ? 4 : 2);
  const int64_t by_bytes = (f32 ? (int64_t)512 << 20 : (int64_t)80 << 20) / bytes, most = f32 ? 448 : 96;
  return by_bytes < most ? by_bytes : most;
}

// Products that are not fused and take their rows more than once, for several tiles of columns, have them put in order first: fetched by place, a
// k-block of 128 rows takes 1000 cycles, twice the product's (40k vertices, 4 of 32, 768-1024-768 gated, rows in order and both products 837 -> 794 us).
bool rows_in_order(const it_experts_desc &d) {
  if (it_experts_fused(d)) return false;
  const int cols = d.hidden_dim > 0 ? d.hidden_dim : d.out_dim;
  return d.feat_dtype == IT_F32 || cols > (d.gated ? 128 : 256);
}

struct ExpertsWs {
  bool few, sorted;
  size_t off_rows;                                   // few: fp32 rows by place
  size_t off_order, off_position, off_tiles, off_counts, off_hidden, off_sums, off_x, off_w1, off_w2;   // (tiles: the number of tiles, then their experts)
  int64_t tiles_max;
  size_t bytes;
};
constexpr size_t kStatusBytes = 256;

it_status plan(const it_experts_desc *d, int64_t n, ExpertsWs *w) {
  IT_TRY(check(d, n));
  *w = ExpertsWs{};
  const int64_t places = n * d->top_k;
  const size_t cols = (size_t)(d->hidden_dim > 0 ? d->hidden_dim : d->out_dim);
  size_t off = kStatusBytes;
  auto take = [&](size_t bytes) { const size_t o = off; off += it_align_up(bytes); return o; };
  const int64_t few = most_few(*d);
  w->few = places <= few;
  // Scratch for many vertices serves any fewer of them: a sorted call needs nearly none where its products are fused, a few places their hidden rows in fp32.
  w->off_rows = take((size_t)(places < few ? places : few) * cols * 4);
  w->bytes = off;
  if (!w->few) {
    off = kStatusBytes;
    const bool f32 = d->feat_dtype == IT_F32;
    w->tiles_max = it_experts_tiles_max(places, d->n_experts);
    const size_t rows = (size_t)w->tiles_max * 128, E = (size_t)d->n_experts, n1 = cols * (d->gated ? 2 : 1);
    w->off_order = take(rows * 4);
    w->off_position = take((size_t)places * 4);
    w->off_tiles = take(((size_t)w->tiles_max + 1) * 4);
    w->off_counts = take(it_experts_count_words(places, d->n_experts) * 4);
    w->off_hidden = take(d->hidden_dim > 0 && !it_experts_fused(*d) ? rows * cols * (f32 ? 6 : 2) : 0);
    w->off_sums = take(d->top_k > 1 ? rows * (size_t)d->out_dim * 4 : 0);
    w->sorted = rows_in_order(*d);
    w->off_x = take(w->sorted ? rows * (size_t)d->in_dim * (f32 ? 6 : (d->in_dtype == IT_E4M3 ? 1 : 2)) : 0);
    w->off_w1 = take(f32 ? E * d->in_dim * n1 * 6 : 0);
    w->off_w2 = take(f32 ? E * d->hidden_dim * d->out_dim * 6 : 0);
    w->bytes = off > w->bytes ? off : w->bytes;
  }
  return IT_OK;
}

// Many places: sorted by expert, one product (or two) over tiles of 128 places, the places of a vertex added up.
it_status many_places(const it_experts_args &a, const ExpertsWs &w, char *ws, uint32_t spin_limit, int no_loads, cudaStream_t st) {
  const it_experts_desc &d = a.d;
  const bool f32 = d.feat_dtype == IT_F32, two = d.hidden_dim > 0;
  it_experts_plan q{};
  q.order = (int32_t *)(ws + w.off_order); q.position = (int32_t *)(ws + w.off_position); q.n_tiles = (int32_t *)(ws + w.off_tiles);
  q.tile_expert = q.n_tiles + 1; q.counts = (int32_t *)(ws + w.off_counts); q.tiles_max = w.tiles_max;
  IT_TRY(it_launch_experts_plan(a, q, st));
  const void *x = a.x, *W1 = d.W1, *W2 = d.W2;
  if (f32) {
    it_experts_parts parts{};
    auto part = [&](const void *src, size_t off, int64_t elems) {
      parts.src[parts.count] = (const float *)src; parts.dst[parts.count] = (__nv_bfloat16 *)(ws + off); parts.elems[parts.count++] = elems;
      return (const void *)(ws + off);
    };
    x = ws + w.off_x;
    parts.x = (const float *)a.x; parts.x_parts = (__nv_bfloat16 *)(ws + w.off_x); parts.row = d.in_dim; parts.top_k = d.top_k;
    parts.order = q.order; parts.n_tiles = q.n_tiles; parts.tiles_max = q.tiles_max;
    W1 = part(d.W1, w.off_w1, (int64_t)d.n_experts * d.in_dim * a.n1);
    if (two) W2 = part(d.W2, w.off_w2, (int64_t)d.n_experts * d.hidden_dim * d.out_dim);
    IT_TRY(it_launch_experts_parts(parts, a.sms, st));
  } else if (w.sorted) {
    IT_TRY(it_launch_experts_rows(a, q, ws + w.off_x, st));
    x = ws + w.off_x;
  }
  const it_expert_store last = d.top_k > 1 ? IT_EXPERT_SUMS : (f32 ? IT_EXPERT_OUT_F32 : IT_EXPERT_OUT_BF16);
  void *result = d.top_k > 1 ? (void *)(ws + w.off_sums) : a.out;
  if (it_experts_fused(d)) {
    IT_TRY(it_launch_experts_fused(a, q, result, spin_limit, no_loads, st));
    return d.top_k > 1 ? launch_combine(a, (const float *)result, q.position, st) : IT_OK;
  }
  it_expert_gemm g{};
  g.parts = f32 ? 3 : 1; g.spin_limit = spin_limit; g.no_loads = no_loads;
  g.A = x; g.gather = !w.sorted; g.a_rows = w.sorted ? w.tiles_max * 128 : a.n; g.W = W1; g.K = d.in_dim; g.w_cols = a.n1; g.cols = two ? d.hidden_dim : d.out_dim;
  g.eight = d.in_dtype == IT_E4M3; g.act = d.act; g.gated = d.gated != 0; g.bias = d.b1; g.w_scale = d.w1_scale; g.x_scale = a.x_scale;
  g.store = two ? (f32 ? IT_EXPERT_PARTS : IT_EXPERT_HIDDEN) : last;
  g.dst = two ? (void *)(ws + w.off_hidden) : result;
  IT_TRY(it_launch_expert_gemm(a, q, g, st));
  if (two) {
    g.A = ws + w.off_hidden; g.gather = 0; g.a_rows = w.tiles_max * 128; g.W = W2; g.K = d.hidden_dim; g.w_cols = g.cols = d.out_dim;
    g.eight = 0; g.act = IT_ACT_NONE; g.gated = 0; g.bias = d.b2; g.w_scale = nullptr; g.x_scale = nullptr; g.store = last; g.dst = result;
    IT_TRY(it_launch_expert_gemm(a, q, g, st));
  }
  return d.top_k > 1 ? launch_combine(a, (const float *)(ws + w.off_sums), q.position, st) : IT_OK;
}

}  // namespace

extern "C" it_status it_experts_workspace_bytes(const it_experts_desc *d, int64_t n, size_t *out_bytes) {
  IT_REQUIRE(out_bytes != nullptr, IT_ERR_INVALID_ARG, "out_bytes is NULL");
  ExpertsWs w;
  IT_TRY(plan(d, n, &w));
  *out_bytes = w.bytes;
  return IT_OK;
}

namespace {
it_status forward(const it_experts_desc *d, int64_t n, const void *x, const float *x_scale, const int32_t *ids, const float *weights, void *out, void *workspace,
                  size_t workspace_bytes, uint32_t spin_limit, int no_loads, cudaStream_t st) {
  ExpertsWs w;
  IT_TRY(plan(d, n, &w));
  const bool eight = d->in_dtype == IT_E4M3;
  IT_REQUIRE(d->W1 != nullptr, IT_ERR_INVALID_ARG, "W1 is NULL");
  IT_REQUIRE((d->W2 != nullptr) == (d->hidden_dim > 0), IT_ERR_INVALID_ARG, "W2 goes with hidden_dim > 0, and only with it");
  IT_REQUIRE(d->hidden_dim > 0 || d->b2 == nullptr, IT_ERR_INVALID_ARG, "b2 goes with hidden_dim > 0");
  IT_REQUIRE(eight == (d->w1_scale != nullptr), IT_ERR_INVALID_ARG, "w1_scale goes with states of IT_E4M3, and only with them");
  IT_REQUIRE(it_aligned(d->W1, 16) && it_aligned(d->W2, 16) && it_aligned(d->b1, 16) && it_aligned(d->b2, 16) && it_aligned(d->w1_scale, 16), IT_ERR_INVALID_ARG,
             "the experts' arrays must be 16-byte aligned");
  IT_REQUIRE(workspace != nullptr && it_aligned(workspace, 256), IT_ERR_WORKSPACE, "workspace is NULL or not 256-byte aligned");
  IT_REQUIRE(workspace_bytes >= w.bytes, IT_ERR_WORKSPACE, "workspace has %zu bytes, it_experts_forward needs %zu", workspace_bytes, w.bytes);
  if (n == 0) {   // nothing to do, and nothing that could have given up
    IT_CUDA_TRY(cudaMemsetAsync(workspace, 0, sizeof(int), st));
    return IT_OK;
  }
  IT_REQUIRE(x != nullptr && ids != nullptr && weights != nullptr && out != nullptr, IT_ERR_INVALID_ARG, "x / ids / weights / out is NULL");
  IT_REQUIRE(eight == (x_scale != nullptr), IT_ERR_INVALID_ARG, "x_scale goes with states of IT_E4M3, and only with them");
  IT_REQUIRE(it_aligned(x, 16) && it_aligned(out, 16) && it_aligned(ids, 4) && it_aligned(weights, 4) && it_aligned(x_scale, 4), IT_ERR_INVALID_ARG,
             "x and out must be 16-byte aligned, ids, weights and x_scale 4-byte");
  const int s = it_dtype_size(d->feat_dtype), s1 = eight ? 1 : s;
  const int64_t n1 = d->hidden_dim > 0 ? (int64_t)d->hidden_dim * (d->gated ? 2 : 1) : d->out_dim;
  const size_t E = (size_t)d->n_experts, ob = (size_t)n * d->out_dim * s, pb = (size_t)n * d->top_k * 4;
  const struct { const void *p; size_t bytes; } in[] = {
      {x, (size_t)n * d->in_dim * s1}, {x_scale, (size_t)n * 4}, {ids, pb}, {weights, pb}, {d->W1, E * d->in_dim * n1 * s1}, {d->b1, E * n1 * 4},
      {d->W2, E * d->hidden_dim * d->out_dim * s}, {d->b2, E * d->out_dim * 4}, {d->w1_scale, E * n1 * 4}};
  for (const auto &i : in)
    IT_REQUIRE(!it_overlap(i.p, i.bytes, out, ob) && !it_overlap(i.p, i.bytes, workspace, workspace_bytes), IT_ERR_INVALID_ARG, "an input overlaps out or the workspace");
  IT_REQUIRE(!it_overlap(out, ob, workspace, workspace_bytes), IT_ERR_INVALID_ARG, "out overlaps the workspace");
  it_experts_args a{};
  a.d = *d; a.n = n; a.n1 = (int)n1; a.x = x; a.x_scale = x_scale; a.ids = ids; a.weights = weights; a.out = out;
  a.status = (int *)workspace; a.sms = it_current_sms();
  char *ws = (char *)workspace;
  return w.few ? few_places(a, (float *)(ws + w.off_rows), st) : many_places(a, w, ws, spin_limit, no_loads, st);
}
}  // namespace

extern "C" it_status it_experts_forward(const it_experts_desc *d, int64_t n, const void *x, const float *x_scale, const int32_t *ids,
                                        const float *weights, void *out, void *workspace, size_t workspace_bytes, void *stream) {
  return forward(d, n, x, x_scale, ids, weights, out, workspace, workspace_bytes, 0, 0, (cudaStream_t)stream);
}

extern "C" it_status it_debug_expire_wait_experts(const it_experts_desc *d, int64_t n, const void *x, const float *x_scale, const int32_t *ids,
                                                  const float *weights, void *out, void *workspace, size_t workspace_bytes, void *stream) {
  ExpertsWs w;
  IT_TRY(plan(d, n, &w));
  IT_REQUIRE(n > 0 && !w.few, IT_ERR_UNSUPPORTED, "the form for few places has no waits");
  return forward(d, n, x, x_scale, ids, weights, out, workspace, workspace_bytes, 4096, 1, (cudaStream_t)stream);
}

extern "C" it_status it_experts_check(void *workspace, void *stream) {
  IT_REQUIRE(workspace != nullptr && it_aligned(workspace, 256), IT_ERR_WORKSPACE, "workspace is NULL or not 256-byte aligned");
  int word = 0;
  cudaStream_t st = (cudaStream_t)stream;
  IT_CUDA_TRY(cudaMemcpyAsync(&word, workspace, sizeof(int), cudaMemcpyDeviceToHost, st));
  IT_CUDA_TRY(cudaStreamSynchronize(st));
  IT_REQUIRE(word == 0, IT_ERR_TIMEOUT, "a kernel of it_experts_forward gave up a bounded wait: its output is not valid");
  return IT_OK;
}
