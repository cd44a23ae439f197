// it_route: per vertex, the top_k of n_experts by score (+ a bias for balance, + groups), and the weights of the chosen.
//
// The choice has to be that of exact arithmetic, which 32 bits cannot promise next to a border.  Without a bias the order of the scores
// is the order of the logits, and nothing is rounded.  With one (or where a group is worth a sum) the fast kernel works in fp32 and
// looks at the gap between every two neighbours of the choice: where it is within the rounding of the two (route_near), the whole warp
// takes the row again in 64 bits.
//
// A row lies in the registers of 1 to 32 lanes (8 experts a lane, 16 and 32 beyond 256 experts); a choice is a maximum over a lane's
// keys and a few shuffles.  Bound by issue slots: the row's bytes are few.
#include <float.h>
#include <math.h>
#include <type_traits>

#include "rows.cuh"

namespace {

constexpr int ROUTE_THREADS = 128, ROUTE_WARPS = ROUTE_THREADS / 32;
constexpr int ROUTE_MAX_EXPERTS = 1024, ROUTE_MAX_K = 32;

struct RouteParams {
  int64_t n;
  int experts, k, n_groups, group_size, group_k, group_best;
  int sigmoid, renorm, need_sum;   // need_sum: the softmax is taken over the whole row
  float scale;
  const float *bias;
  const void *logits;
  int32_t *ids;
  float *weights;
  uint32_t group_magic;            // e / group_size = (e * group_magic) >> 22 for e < 1024
};

constexpr float kClosed = -INFINITY;
// A logit as it counts: NaN closes the expert, +inf is the largest finite value.
__device__ __forceinline__ float open_logit(float l) { return l != l ? kClosed : fminf(l, FLT_MAX); }
__device__ __forceinline__ float open_key(float k) { return k != k ? kClosed : k; }
__device__ __forceinline__ double open_key(double k) { return k != k ? (double)kClosed : k; }

// ----------------------------------------------------------------------------- 64 bits, a warp per row
// key: [experts] doubles of shared memory, then [n_groups] of the groups' worths.
__device__ void route_row_exact(const RouteParams &p, const void *logits, bool bf16, int64_t row, double *key, int lane) {
  const unsigned full = 0xffffffffu;
  double *worth = key + p.experts;
  auto logit = [&](int e) {
    const int64_t at = row * p.experts + e;
    return open_logit(bf16 ? __bfloat162float(reinterpret_cast<const __nv_bfloat16 *>(logits)[at]) : reinterpret_cast<const float *>(logits)[at]);
  };
  float top = kClosed;
  for (int e = lane; e < p.experts; e += 32) top = fmaxf(top, logit(e));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(full, top, o));
  double total = 0.0;
  if (!p.sigmoid) {
    for (int e = lane; e < p.experts; e += 32) {
      const float l = logit(e);
      if (l > kClosed) total += exp((double)l - (double)top);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(full, total, o);
  }
  auto score = [&](float l) -> double {
    if (!(l > kClosed)) return 0.0;
    return p.sigmoid ? 1.0 / (1.0 + exp(-(double)l)) : exp((double)l - (double)top) / total;
  };
  __syncwarp();   // (the previous row's keys have been read)
  for (int e = lane; e < p.experts; e += 32) {
    const float l = logit(e);
    double k = (double)l;
    if (p.bias && l > kClosed) k = open_key(score(l) + (double)p.bias[e]);
    key[e] = k;
  }
  __syncwarp();
  if (p.n_groups > 1) {
    for (int g = lane; g < p.n_groups; g += 32) {
      double a = (double)kClosed, b = (double)kClosed;
      for (int i = 0; i < p.group_size; ++i) {
        const double k = key[g * p.group_size + i];
        if (k > a) { b = a; a = k; }
        else if (k > b) b = k;
      }
      if (p.group_best == 2 && a > (double)kClosed) {
        if (!p.bias) { a = score((float)a); b = b > (double)kClosed ? score((float)b) : 0.0; }
        else if (!(b > (double)kClosed)) b = 0.0;
        a += b;
      }
      worth[g] = a;
    }
    __syncwarp();
    for (int g = lane; g < p.n_groups; g += 32) {
      int rank = 0;
      for (int o = 0; o < p.n_groups; ++o) rank += worth[o] > worth[g] || (worth[o] == worth[g] && o < g);
      if (rank >= p.group_k)
        for (int i = 0; i < p.group_size; ++i) key[g * p.group_size + i] = (double)kClosed;
    }
    __syncwarp();
  }
  int my_id = -1;
  double my_w = 0.0;
  for (int j = 0; j < p.k; ++j) {
    double best = (double)kClosed;
    int at = ROUTE_MAX_EXPERTS;
    for (int e = lane; e < p.experts; e += 32)
      if (key[e] > best) { best = key[e]; at = e; }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const double b = __shfl_xor_sync(full, best, o);
      const int a = __shfl_xor_sync(full, at, o);
      if (b > best || (b == best && a < at)) { best = b; at = a; }
    }
    if (at == ROUTE_MAX_EXPERTS) break;   // (the same for all lanes)
    if (lane == j) { my_id = at; my_w = score(logit(at)); }
    if (lane == 0) key[at] = (double)kClosed;
    __syncwarp();
  }
  double sum = my_w;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(full, sum, o);
  if (p.renorm) my_w = sum > 0.0 ? my_w / sum : 0.0;
  if (lane < p.k) {
    p.ids[row * p.k + lane] = my_id;
    p.weights[row * p.k + lane] = (float)(my_w * (double)p.scale);
  }
}

// ----------------------------------------------------------------------------- the fast kernel
// Whether fp32 leaves open which of two keys (or sums of keys) a >= b is larger.  pa, pb: the scores in them, each off by at most 5 ulp
// (expf 2, the sum of a row 1, the division 1, their product 1); adding a bias rounds once more, by half an ulp of the key.
// In a softmax the difference from the row's largest logit is rounded too, by |difference| * 2^-24: pa and pb come with that share
// (route_slack), which below 1e-30 would no longer be represented.
__device__ __forceinline__ bool route_near(float a, float b, float pa, float pb) {
  return a - b <= 1e-6f * (pa + pb) + 2.5e-7f * (fabsf(a) + fabsf(b)) + 1e-30f;
}
__device__ __forceinline__ float route_slack(float score, float below_top) { return score * fmaf(fabsf(below_top), 0.125f, 1.f); }

// L lanes per row, C experts per lane.
template <typename T, int L, int C>
__global__ void __launch_bounds__(ROUTE_THREADS) route_kernel(const RouteParams p) {
  it_allow_next();
  it_wait_prior();
  constexpr int R = 32 / L;                       // rows of a warp
  constexpr int N = kVec<T> < C ? kVec<T> : C;    // consecutive experts of a lane
  constexpr unsigned full = 0xffffffffu;
  extern __shared__ double route_smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gl = lane % L, r = lane / L;
  // per warp: ids and weights of its rows [R][k] each, the fp32 keys and worths of its rows (groups), or the 64-bit ones of one row
  const int E = p.experts, per_warp = E + p.n_groups;
  double *mine64 = route_smem + (size_t)warp * per_warp;
  const int row_words = E + E / 32 + 1 + p.n_groups;   // a pad word after every 32 keys
  float *after = reinterpret_cast<float *>(route_smem + (size_t)ROUTE_WARPS * per_warp);
  const int warp_words = R * 2 * p.k + (p.n_groups > 1 ? R * row_words : 0);
  int32_t *out_ids = reinterpret_cast<int32_t *>(after + (size_t)warp * warp_words);
  float *out_w = reinterpret_cast<float *>(out_ids + R * p.k);
  float *keys = out_w + R * p.k + (size_t)r * row_words, *worth = keys + E + E / 32 + 1;
  auto expert = [&](int c) { return ((c / N) * L + gl) * N + c % N; };
  const bool vec = (E * (int)sizeof(T)) % 16 == 0 && N == kVec<T> && ((uintptr_t)p.logits & 15) == 0;

  for (int64_t row0 = ((int64_t)blockIdx.x * ROUTE_WARPS + warp) * R; row0 < p.n; row0 += (int64_t)gridDim.x * ROUTE_WARPS * R) {
    const int64_t row = row0 + r < p.n ? row0 + r : p.n - 1;   // lanes past the last row repeat it, and store nothing
    const T *from = reinterpret_cast<const T *>(p.logits) + row * E;
    float logit[C], key[C];
#pragma unroll
    for (int c0 = 0; c0 < C; c0 += N) {
      const int e0 = expert(c0);
      if constexpr (N == kVec<T>) {
        if (vec) {
          float v[N];
          if (e0 < E) vec_to_f32(*reinterpret_cast<const uint4 *>(from + e0), v);
#pragma unroll
          for (int i = 0; i < N; ++i) logit[c0 + i] = e0 < E ? open_logit(v[i]) : kClosed;
          continue;
        }
      }
#pragma unroll
      for (int i = 0; i < N; ++i) logit[c0 + i] = e0 + i < E ? open_logit(to_f32(from[e0 + i])) : kClosed;
    }
    float top = 0.f, inv = 1.f;
    if (!p.sigmoid) {
      top = logit[0];
#pragma unroll
      for (int c = 1; c < C; ++c) top = fmaxf(top, logit[c]);
#pragma unroll
      for (int o = L / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(full, top, o));
      if (!(top > kClosed)) top = 0.f;   // nothing is open
    }
    auto raw = [&](float l) { return p.sigmoid ? 1.f / (1.f + expf(-l)) : expf(l - top); };   // (a closed logit: 0)
    bool near = false;
    if (p.bias) {
      float sum = 0.f;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        key[c] = raw(logit[c]);
        sum += key[c];
      }
      if (!p.sigmoid) {
#pragma unroll
        for (int o = L / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(full, sum, o);
        inv = sum > 0.f ? 1.f / sum : 0.f;
      }
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int e = expert(c);
        key[c] = logit[c] > kClosed ? open_key(fmaf(key[c], inv, __ldg(p.bias + e))) : kClosed;
      }
    } else {
#pragma unroll
      for (int c = 0; c < C; ++c) key[c] = logit[c];
      if (p.need_sum) {
        float sum = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c) sum += raw(logit[c]);
#pragma unroll
        for (int o = L / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(full, sum, o);
        inv = sum > 0.f ? 1.f / sum : 0.f;
      }
    }
    if (p.n_groups > 1) {
      __syncwarp();
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int e = expert(c);
        if (e < E) keys[e + (e >> 5)] = key[c];
      }
      __syncwarp();
      for (int g = gl; g < p.n_groups; g += L) {
        float a = kClosed, b = kClosed;
        for (int i = 0, e = g * p.group_size; i < p.group_size; ++i, ++e) {
          const float k = keys[e + (e >> 5)];
          b = fmaxf(b, fminf(a, k));
          a = fmaxf(a, k);
        }
        if (p.group_best == 2 && a > kClosed) {
          const float second = b > kClosed ? (p.bias ? b : raw(b)) : 0.f;
          a = (p.bias ? a : raw(a)) + second;
        }
        worth[g] = a;
      }
      __syncwarp();
      // every lane ranks all groups whose experts it holds by way of one flag per group, kept in place of the keys
      const bool exact = !p.bias && p.group_best == 1;
      for (int g = gl; g < p.n_groups; g += L) {
        const float w = worth[g];
        int rank = 0;
        for (int o = 0; o < p.n_groups; ++o) {
          const float v = worth[o];
          rank += v > w || (v == w && o < g);
          // a worth with a bias: two scores of at most inv each, whose slack (x e^-x / 8) is below 5 %; without: sums of e^-x with x < 104
          if (!exact && o != g && v > kClosed && w > kClosed) near |= v >= w && route_near(v, w, p.bias ? 2.2f * inv : 14.f * v, p.bias ? 2.2f * inv : 14.f * w);
        }
        keys[g] = rank < p.group_k ? 1.f : 0.f;
      }
      __syncwarp();
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int e = expert(c);
        if (e < E && keys[(e * p.group_magic) >> 22] == 0.f) key[c] = kClosed;
      }
    }
    // the choice, one more than asked for where its border has to be looked at
    float before = INFINITY, p_before = 0.f, sum = 0.f;
    const int rounds = p.k + (p.bias && p.k < E ? 1 : 0);
    for (int j = 0; j < rounds; ++j) {
      float best = kClosed, l = kClosed;
      int at = ROUTE_MAX_EXPERTS;
#pragma unroll
      for (int c = 0; c < C; ++c)
        if (key[c] > best) { best = key[c]; at = expert(c); l = logit[c]; }
#pragma unroll
      for (int o = L / 2; o > 0; o >>= 1) {
        const float b = __shfl_xor_sync(full, best, o), bl = __shfl_xor_sync(full, l, o);
        const int a = __shfl_xor_sync(full, at, o);
        if (b > best || (b == best && a < at)) { best = b; at = a; l = bl; }
      }
#pragma unroll
      for (int c = 0; c < C; ++c)
        if (expert(c) == at) key[c] = kClosed;
      const bool some = best > kClosed;
      const float w = some ? raw(l) * (p.bias || p.need_sum ? inv : 1.f) : 0.f;
      const float slack = p.sigmoid ? w : route_slack(w, some ? l - top : 0.f);
      if (p.bias && some && j > 0) near |= route_near(before, best, p_before, slack);
      before = best;
      p_before = slack;
      if (j < p.k) {
        sum += w;
        if (gl == 0) { out_ids[r * p.k + j] = some ? at : -1; out_w[r * p.k + j] = w; }
      }
    }
    const float f = p.renorm ? (sum > 0.f ? p.scale / sum : 0.f) : p.scale;
    __syncwarp();
    if (gl == 0)
      for (int j = 0; j < p.k; ++j) out_w[r * p.k + j] *= f;
    __syncwarp();
    const int real = p.n - row0 < R ? (int)(p.n - row0) : R;
    for (int i = lane; i < real * p.k; i += 32) {
      p.ids[row0 * p.k + i] = out_ids[i];
      p.weights[row0 * p.k + i] = out_w[i];
    }
    __syncwarp();
    unsigned again = __ballot_sync(full, near);
    while (again) {
      const int which = (__ffs(again) - 1) / L;
      route_row_exact(p, p.logits, sizeof(T) == 2, row0 + which < p.n ? row0 + which : p.n - 1, mine64, lane);
      again &= ~((full >> (32 - L)) << (which * L));
      __syncwarp();
    }
  }
}

template <typename T, int L, int C>
it_status launch(const RouteParams &p, double bytes, double flops, cudaStream_t st) {
  constexpr int R = 32 / L;
  const size_t warp64 = (size_t)(p.experts + p.n_groups) * 8;
  const size_t warp32 = ((size_t)R * 2 * p.k + (p.n_groups > 1 ? (size_t)R * (p.experts + p.experts / 32 + 1 + p.n_groups) : 0)) * 4;
  const size_t smem = ROUTE_WARPS * (warp64 + warp32);
  if (smem > 48 * 1024) IT_CUDA_TRY(cudaFuncSetAttribute(route_kernel<T, L, C>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
  const int64_t blocks = (p.n + ROUTE_WARPS * R - 1) / (ROUTE_WARPS * R), most = (int64_t)it_current_sms() * 16;
  IT_LAUNCH(IT_K_ROUTE, bytes, flops, st,
            IT_CUDA_TRY(it_launch_pdl(route_kernel<T, L, C>, dim3((unsigned)(blocks < most ? blocks : most)), dim3(ROUTE_THREADS), smem, st, p)));
  return IT_OK;
}

template <typename T>
it_status dispatch(const RouteParams &p, double bytes, double flops, cudaStream_t st) {
  const int e = p.experts;
  if (e <= 8) return launch<T, 1, 8>(p, bytes, flops, st);
  if (e <= 16) return launch<T, 2, 8>(p, bytes, flops, st);
  if (e <= 32) return launch<T, 4, 8>(p, bytes, flops, st);
  if (e <= 64) return launch<T, 8, 8>(p, bytes, flops, st);
  if (e <= 128) return launch<T, 16, 8>(p, bytes, flops, st);
  if (e <= 256) return launch<T, 32, 8>(p, bytes, flops, st);
  if (e <= 512) return launch<T, 32, 16>(p, bytes, flops, st);
  return launch<T, 32, 32>(p, bytes, flops, st);
}

}  // namespace

extern "C" it_status it_route(const it_route_desc *d, int64_t n, const void *logits, int32_t *ids, float *weights, void *stream) {
  IT_REQUIRE(d != nullptr, IT_ERR_INVALID_ARG, "description is NULL");
  IT_REQUIRE(d->logit_dtype == IT_F32 || d->logit_dtype == IT_BF16, IT_ERR_INVALID_ARG, "bad logit_dtype");
  IT_REQUIRE(d->score == IT_SCORE_SOFTMAX || d->score == IT_SCORE_SIGMOID, IT_ERR_INVALID_ARG, "bad score %d", (int)d->score);
  const int E = d->n_experts, k = d->top_k;
  IT_REQUIRE(n >= 0 && E >= 1, IT_ERR_INVALID_ARG, "bad shape (%lld rows of %d)", (long long)n, E);
  IT_REQUIRE(E <= ROUTE_MAX_EXPERTS, IT_ERR_UNSUPPORTED, "%d experts, at most %d", E, ROUTE_MAX_EXPERTS);
  IT_REQUIRE(k >= 1 && k <= E, IT_ERR_INVALID_ARG, "top_k %d of %d experts", k, E);
  IT_REQUIRE(k <= ROUTE_MAX_K, IT_ERR_UNSUPPORTED, "top_k %d, at most %d", k, ROUTE_MAX_K);
  IT_REQUIRE(d->n_groups >= 1 && E % d->n_groups == 0, IT_ERR_INVALID_ARG, "%d groups do not divide %d experts", d->n_groups, E);
  IT_REQUIRE(d->group_k >= 1 && d->group_k <= d->n_groups, IT_ERR_INVALID_ARG, "group_k %d of %d groups", d->group_k, d->n_groups);
  IT_REQUIRE(d->group_best == 1 || d->group_best == 2, IT_ERR_INVALID_ARG, "group_best %d is neither 1 nor 2", d->group_best);
  IT_REQUIRE(isfinite(d->weight_scale), IT_ERR_INVALID_ARG, "weight_scale is not finite");
  IT_REQUIRE(n <= INT64_MAX / 8 / E, IT_ERR_INVALID_ARG, "bad shape (%lld rows of %d)", (long long)n, E);
  if (n == 0) return IT_OK;
  IT_REQUIRE(logits != nullptr && ids != nullptr && weights != nullptr, IT_ERR_INVALID_ARG, "logits / ids / weights is NULL");
  const int s = it_dtype_size(d->logit_dtype);
  IT_REQUIRE(it_aligned(logits, s) && it_aligned(ids, 4) && it_aligned(weights, 4) && it_aligned(d->balance_bias, 4), IT_ERR_INVALID_ARG,
             "a pointer is not aligned to its elements");
  const size_t in = (size_t)n * E * s, out = (size_t)n * k * 4, bb = (size_t)E * 4;
  IT_REQUIRE(!it_overlap(ids, out, weights, out) && !it_overlap(ids, out, logits, in) && !it_overlap(weights, out, logits, in) &&
                 !it_overlap(ids, out, d->balance_bias, bb) && !it_overlap(weights, out, d->balance_bias, bb),
             IT_ERR_INVALID_ARG, "ids / weights overlap each other or an input");
  RouteParams p{};
  p.n = n; p.experts = E; p.k = k; p.n_groups = d->n_groups; p.group_size = E / d->n_groups; p.group_k = d->group_k; p.group_best = d->group_best;
  p.sigmoid = d->score == IT_SCORE_SIGMOID; p.renorm = d->renormalise != 0; p.scale = d->weight_scale;
  p.need_sum = !p.sigmoid && !p.renorm;
  p.bias = d->balance_bias; p.logits = logits; p.ids = ids; p.weights = weights;
  p.group_magic = ((1u << 22) + p.group_size - 1) / p.group_size;
  const double bytes = (double)in + 2.0 * out, flops = (double)n * E * (4.0 + k);
  return d->logit_dtype == IT_F32 ? dispatch<float>(p, bytes, flops, (cudaStream_t)stream) : dispatch<__nv_bfloat16>(p, bytes, flops, (cudaStream_t)stream);
}
