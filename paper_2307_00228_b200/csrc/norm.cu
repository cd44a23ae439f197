// it_residual_norm: s = x + residual, y = s / sqrt(mean(s^2) + eps) * weight, one pass over the rows.
//
// Bound by DRAM bytes (a row is read once per operand and written once per output; about ten instructions an element).  A row lies in
// the registers of a group of lanes, so that the sum of squares and the scale of an 8-bit output are reduced by shuffles
// and nothing is read twice; only rows of more than 2 KB take a block each and are read again (out of the cache) for the output.
#include <cuda_fp8.h>

#include <type_traits>

#include "rows.cuh"

namespace {

struct NormParams {
  int64_t n;
  int dim;
  float eps;
  const void *x, *residual;
  const float *weight;
  void *sum_out, *out;
  float *scales;
};

constexpr int NORM_THREADS = 256;
constexpr float kE4m3Max = 448.f;
constexpr float kTiny = 1.17549435e-38f;   // 2^-126: the scale of a row of zeros, whose inverse is still finite

__device__ __forceinline__ float max_nan(float a, float b) {   // NaN if either is
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float row_scale(float amax) { return max_nan(amax / kE4m3Max, kTiny); }

template <int N> __device__ __forceinline__ void store_e4m3(void *to, const float (&y)[N]) {
  uint32_t w[N / 4];
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(y[4 * i], y[4 * i + 1]), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(y[4 * i + 2], y[4 * i + 3]), __NV_SATFINITE, __NV_E4M3);
    w[i] = lo | (hi << 16);
  }
  if constexpr (N == 8) *reinterpret_cast<uint2 *>(to) = make_uint2(w[0], w[1]);
  else *reinterpret_cast<uint32_t *>(to) = w[0];
}

// s of one 16-byte vector
template <typename T> __device__ __forceinline__ void load_sum(const NormParams &p, int64_t at, float (&v)[kVec<T>]) {
  const uint4 a = *reinterpret_cast<const uint4 *>(reinterpret_cast<const T *>(p.x) + at);
  vec_to_f32(a, v);
  if (p.residual) {
    const uint4 b = *reinterpret_cast<const uint4 *>(reinterpret_cast<const T *>(p.residual) + at);
    float r[kVec<T>];
    vec_to_f32(b, r);
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i) v[i] += r[i];
  }
}
template <int N> __device__ __forceinline__ void load_weight(const float *weight, int c, float (&g)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    const float4 q = weight ? *reinterpret_cast<const float4 *>(weight + c + i) : make_float4(1.f, 1.f, 1.f, 1.f);
    g[i] = q.x; g[i + 1] = q.y; g[i + 2] = q.z; g[i + 3] = q.w;
  }
}

// LPR lanes per row, V vectors per lane.
template <typename T, bool EIGHT, int LPR, int V>
__global__ void __launch_bounds__(NORM_THREADS) norm_rows_kernel(const NormParams p) {
  it_allow_next();
  it_wait_prior();
  constexpr int N = kVec<T>, ROWS = NORM_THREADS / LPR;
  const int gl = threadIdx.x % LPR, nv = p.dim / N;
  float g[V][N];
#pragma unroll
  for (int j = 0; j < V; ++j)
    if (j * LPR + gl < nv) load_weight(p.weight, (j * LPR + gl) * N, g[j]);
  const float inv_dim = 1.f / (float)p.dim;
  // (whole warps go round together: the shuffles name every lane)
  for (int64_t row0 = (int64_t)blockIdx.x * ROWS; row0 < p.n; row0 += (int64_t)gridDim.x * ROWS) {
    const int64_t row = row0 + threadIdx.x / LPR;
    const bool real = row < p.n;
    float v[V][N], ss = 0.f;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int q = j * LPR + gl;
      if (real && q < nv) {
        load_sum<T>(p, row * p.dim + q * N, v[j]);
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[j][i] = 0.f;
      }
    }
#pragma unroll
    for (int j = 0; j < V; ++j)
#pragma unroll
      for (int i = 0; i < N; ++i) ss = fmaf(v[j][i], v[j][i], ss);
#pragma unroll
    for (int o = LPR / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    const float r = rsqrtf(fmaf(ss, inv_dim, p.eps));
    float amax = 0.f;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int q = j * LPR + gl;
      if (!real || q >= nv) continue;
      const int64_t at = row * p.dim + q * N;
      if (p.sum_out) *reinterpret_cast<uint4 *>(reinterpret_cast<T *>(p.sum_out) + at) = f32_to_vec(v[j]);
#pragma unroll
      for (int i = 0; i < N; ++i) v[j][i] = v[j][i] * r * g[j][i];
      if constexpr (EIGHT) {
#pragma unroll
        for (int i = 0; i < N; ++i) amax = max_nan(amax, fabsf(v[j][i]));
      } else {
        *reinterpret_cast<uint4 *>(reinterpret_cast<T *>(p.out) + at) = f32_to_vec(v[j]);
      }
    }
    if constexpr (EIGHT) {
#pragma unroll
      for (int o = LPR / 2; o > 0; o >>= 1) amax = max_nan(amax, __shfl_xor_sync(0xffffffffu, amax, o));
      const float scale = row_scale(amax), inv = 1.f / scale;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int q = j * LPR + gl;
        if (!real || q >= nv) continue;
#pragma unroll
        for (int i = 0; i < N; ++i) v[j][i] *= inv;
        store_e4m3(reinterpret_cast<unsigned char *>(p.out) + row * p.dim + q * N, v[j]);
      }
      if (real && gl == 0) p.scales[row] = scale;
    }
  }
}

// Rows of more than 32 lanes x 4 vectors: a block each, read again for the output.  A thread writes only what it alone reads, and
// reads all of a vector before it writes any of it, so that sum_out and out may lie over the operands: the output pass comes last.
template <typename T, bool EIGHT>
__global__ void __launch_bounds__(NORM_THREADS) norm_long_rows_kernel(const NormParams p) {
  it_allow_next();
  it_wait_prior();
  constexpr int N = kVec<T>, WARPS = NORM_THREADS / 32;
  __shared__ float part[2][WARPS];
  const int nv = p.dim / N, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int64_t row = blockIdx.x; row < p.n; row += gridDim.x) {
    float ss = 0.f;
    for (int q = threadIdx.x; q < nv; q += NORM_THREADS) {
      float v[N];
      load_sum<T>(p, row * p.dim + q * N, v);
#pragma unroll
      for (int i = 0; i < N; ++i) ss = fmaf(v[i], v[i], ss);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    if (lane == 0) part[0][warp] = ss;
    __syncthreads();
    ss = 0.f;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) ss += part[0][w];
    const float r = rsqrtf(ss / (float)p.dim + p.eps);
    float inv = 1.f;
    if constexpr (EIGHT) {
      float amax = 0.f;
      for (int q = threadIdx.x; q < nv; q += NORM_THREADS) {
        float v[N], g[N];
        load_sum<T>(p, row * p.dim + q * N, v);
        load_weight(p.weight, q * N, g);
#pragma unroll
        for (int i = 0; i < N; ++i) amax = max_nan(amax, fabsf(v[i] * r * g[i]));
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) amax = max_nan(amax, __shfl_xor_sync(0xffffffffu, amax, o));
      if (lane == 0) part[1][warp] = amax;
      __syncthreads();
      amax = 0.f;
#pragma unroll
      for (int w = 0; w < WARPS; ++w) amax = max_nan(amax, part[1][w]);
      const float scale = row_scale(amax);
      inv = 1.f / scale;
      if (threadIdx.x == 0) p.scales[row] = scale;
    }
    for (int q = threadIdx.x; q < nv; q += NORM_THREADS) {
      const int64_t at = row * p.dim + q * N;
      float v[N], g[N];
      load_sum<T>(p, at, v);
      load_weight(p.weight, q * N, g);
      if (p.sum_out) *reinterpret_cast<uint4 *>(reinterpret_cast<T *>(p.sum_out) + at) = f32_to_vec(v);
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = v[i] * r * g[i];
      if constexpr (EIGHT) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] *= inv;
        store_e4m3(reinterpret_cast<unsigned char *>(p.out) + at, v);
      } else {
        *reinterpret_cast<uint4 *>(reinterpret_cast<T *>(p.out) + at) = f32_to_vec(v);
      }
    }
    __syncthreads();   // the partial sums are read before the next row's
  }
}

template <typename T, bool EIGHT>
it_status launch(const NormParams &p, double bytes, double flops, cudaStream_t st) {
  const int nv = p.dim / kVec<T>, sms = it_current_sms();
  auto rows = [&](auto lpr, auto v) -> it_status {
    constexpr int LPR = decltype(lpr)::value, V = decltype(v)::value;
    const int64_t blocks = (p.n + NORM_THREADS / LPR - 1) / (NORM_THREADS / LPR), most = (int64_t)sms * 32;
    IT_LAUNCH(IT_K_NORM, bytes, flops, st,
              IT_CUDA_TRY(it_launch_pdl(norm_rows_kernel<T, EIGHT, LPR, V>, dim3((unsigned)(blocks < most ? blocks : most)), dim3(NORM_THREADS), 0, st, p)));
    return IT_OK;
  };
#define IT_NORM_CASE(LPR, V) return rows(std::integral_constant<int, LPR>{}, std::integral_constant<int, V>{})
  if (nv <= 1) IT_NORM_CASE(1, 1);
  if (nv <= 2) IT_NORM_CASE(2, 1);
  if (nv <= 4) IT_NORM_CASE(4, 1);
  if (nv <= 8) IT_NORM_CASE(8, 1);
  if (nv <= 16) IT_NORM_CASE(16, 1);
  if (nv <= 32) IT_NORM_CASE(32, 1);
  if (nv <= 64) IT_NORM_CASE(32, 2);
  if (nv <= 96) IT_NORM_CASE(32, 3);
  if (nv <= 128) IT_NORM_CASE(32, 4);
#undef IT_NORM_CASE
  const int64_t most = (int64_t)sms * 8;
  IT_LAUNCH(IT_K_NORM, bytes, flops, st,
            IT_CUDA_TRY(it_launch_pdl(norm_long_rows_kernel<T, EIGHT>, dim3((unsigned)(p.n < most ? p.n : most)), dim3(NORM_THREADS), 0, st, p)));
  return IT_OK;
}

}  // namespace

extern "C" it_status it_residual_norm(const it_norm_desc *d, int64_t n, const void *x, const void *residual, void *sum_out, void *out,
                                      float *scales, void *stream) {
  IT_REQUIRE(d != nullptr, IT_ERR_INVALID_ARG, "description is NULL");
  IT_REQUIRE(d->feat_dtype == IT_F32 || d->feat_dtype == IT_BF16, IT_ERR_INVALID_ARG, "bad feat_dtype");
  IT_REQUIRE(d->out_dtype == d->feat_dtype || d->out_dtype == IT_E4M3, IT_ERR_INVALID_ARG, "out_dtype must be feat_dtype or IT_E4M3");
  const int s = it_dtype_size(d->feat_dtype);
  const bool eight = d->out_dtype == IT_E4M3;
  IT_REQUIRE(n >= 0 && d->dim > 0, IT_ERR_INVALID_ARG, "bad shape (%lld rows of %d)", (long long)n, d->dim);
  IT_REQUIRE((int64_t)d->dim * s % 16 == 0 && (!eight || d->dim % 16 == 0), IT_ERR_INVALID_ARG, "rows must be a multiple of 16 bytes (dim %d)", d->dim);
  IT_REQUIRE(n <= INT64_MAX / 16 / d->dim, IT_ERR_INVALID_ARG, "bad shape (%lld rows of %d)", (long long)n, d->dim);
  IT_REQUIRE(d->eps >= 0.f && d->eps <= 3e38f, IT_ERR_INVALID_ARG, "eps must be finite and not negative");
  IT_REQUIRE(it_aligned(d->weight, 16), IT_ERR_INVALID_ARG, "weight must be 16-byte aligned");
  IT_REQUIRE(eight == (scales != nullptr) || n == 0, IT_ERR_INVALID_ARG, "scales go with an output of IT_E4M3, and only with it");
  if (n == 0) return IT_OK;
  IT_REQUIRE(x != nullptr && out != nullptr, IT_ERR_INVALID_ARG, "x / out is NULL");
  IT_REQUIRE(it_aligned(x, 16) && it_aligned(residual, 16) && it_aligned(sum_out, 16) && it_aligned(out, 16) && it_aligned(scales, 4), IT_ERR_INVALID_ARG,
             "matrices must be 16-byte aligned");
  const size_t rows = (size_t)n * d->dim * s, out_rows = eight ? (size_t)n * d->dim : rows, wb = (size_t)d->dim * 4, sb = (size_t)n * 4;
  auto clash = [&](const void *o, size_t ob, bool may) {   // an output against what is read: the same matrix, or apart
    return (it_overlap(o, ob, x, rows) && !(may && o == x)) || (it_overlap(o, ob, residual, rows) && !(may && o == residual)) || it_overlap(o, ob, d->weight, wb);
  };
  IT_REQUIRE(!clash(sum_out, rows, true) && !clash(out, out_rows, !eight) && !clash(scales, sb, false), IT_ERR_INVALID_ARG,
             "an output overlaps an input without being the same matrix");
  IT_REQUIRE(!it_overlap(sum_out, rows, out, out_rows) && !it_overlap(scales, sb, out, out_rows) && !it_overlap(scales, sb, sum_out, rows), IT_ERR_INVALID_ARG,
             "the outputs overlap");
  const NormParams p{n, d->dim, d->eps, x, residual, d->weight, sum_out, out, scales};
  const double bytes = (double)rows * (1 + (residual != nullptr) + (sum_out != nullptr)) + (double)out_rows + (eight ? (double)sb : 0.0);
  const double flops = 5.0 * (double)n * d->dim;
  cudaStream_t st = (cudaStream_t)stream;
  if (d->feat_dtype == IT_F32) return eight ? launch<float, true>(p, bytes, flops, st) : launch<float, false>(p, bytes, flops, st);
  return eight ? launch<__nv_bfloat16, true>(p, bytes, flops, st) : launch<__nv_bfloat16, false>(p, bytes, flops, st);
}
