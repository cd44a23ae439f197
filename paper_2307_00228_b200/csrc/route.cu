// it_route: per vertex, the top_k of n_experts by score (+ a bias for balance, + groups), and the weights of the chosen.
//
// The choice has to be that of exact arithmetic, which 32 bits cannot promise next to a border.  Without a bias the order of the scores
// is the order of the logits, and nothing is rounded.  With one (or where a group is worth a sum) the fast kernel works in fp32 and
// looks at the gap between every two neighbours of the choice, and between its last key and the best one left out: where it is within the
// rounding of the two (route_near), the whole warp takes the row again in 64 bits.  Behind the best one left out may be keys that are less
// exact than it (a large score with a large negative bias), so that gap is held against the largest rounding that a key of the row can have.
//
// A row lies in the registers of 1 to 32 lanes (8 experts a lane, 16 and 32 beyond 256 experts), or of one thread where experts and
// places are few.  Bound by issue slots: the row's bytes are few.
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

// Scores end at what 64 bits hold: a softmax's at a logit 745.13 below the row's largest, a sigmoid's at -709.78, where e^-l has no double.
__device__ __forceinline__ bool route_scored(bool sigmoid, float l, float top) { return sigmoid ? l > -709.7827f : l - top >= -745.13f; }
// The score of a chosen logit next to those chosen with it, of which `most` is the largest: divided by e^most (softmax) or by e^min(most, 0) (sigmoid), so that
// the scores of a row's chosen add up to between 1/2 and their number however small they are.
__device__ __forceinline__ double route_share(bool sigmoid, float l, float top, float most) {
  if (!(l > kClosed) || !route_scored(sigmoid, l, top)) return 0.0;
  if (!sigmoid) return exp((double)l - (double)most);
  return l < 0.f ? exp((double)l - (double)fminf(most, 0.f)) / (1.0 + exp((double)l)) : 1.0 / (1.0 + exp(-(double)l));
}
// Whether a chosen score is too small for 32 bits to be divided by the sum of the chosen: the row is then taken again in 64.  (Where the sum is
// 1 or more, so is what becomes of it.)
__device__ __forceinline__ bool route_tiny(bool sigmoid, float score, float sum, float l, float top) {
  return score < 1.2e-37f && sum < 1.f && route_scored(sigmoid, l, top);
}

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
  float my_l = kClosed;
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
    if (lane == j) { my_id = at; my_l = logit(at); }
    if (lane == 0) key[at] = (double)kClosed;
    __syncwarp();
  }
  double my_w;
  if (p.renorm) {
    float most = my_l;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(full, most, o));
    my_w = route_share(p.sigmoid, my_l, top, most);
    double sum = my_w;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(full, sum, o);
    my_w = sum > 0.0 ? my_w / sum : 0.0;
  } else {
    my_w = score(my_l);
  }
  if (lane < p.k) {
    p.ids[row * p.k + lane] = my_id;
    p.weights[row * p.k + lane] = (float)(my_w * (double)p.scale);
  }
}

// ----------------------------------------------------------------------------- the fast kernel
// Whether fp32 leaves open which of two keys (or sums of keys) a >= b is larger.  pa, pb: the scores in them, as far as their rounding goes
// (route_slack); adding a bias rounds once more, by half an ulp of the key.  A score is off by at most `rel` of itself.  A sigmoid, 1e-6: the hardware
// exponential 2^-22, a sum 2^-24, a reciprocal 2^-23.  A softmax, 4e-6: the exponential 2^-22, that of the row's sum 2^-22, the exponents in that sum
// ln(1024) times 2.3 * 2^-24, its up to 36 additions and the division 2^-24 each.  The exponent is rounded too (the difference, the factor log2(e), the
// product: 2.3 * 2^-24 of it): that share, 0.15 rel, is in pa and pb, which below 1e-30 would no longer be represented.
__device__ __forceinline__ bool route_near(float a, float b, float pa, float pb, float rel) {
  return a - b <= rel * (pa + pb) + 2.5e-7f * (fabsf(a) + fabsf(b)) + 1e-30f;
}
// (p (1 + 0.15 |x|) of a score p = e^-|x| is largest at x = 0: no score of a row has more slack than 1, or than the softmax's largest score)
__device__ __forceinline__ float route_slack(float score, float below_top) { return score * fmaf(fminf(fabsf(below_top), 1e30f), 0.15f, 1.f); }

__device__ __forceinline__ float route_rcp(float x) {   // of 1 to infinity
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// A float as an unsigned number of the same order (neither operand is NaN; -0 counts as 0).
__device__ __forceinline__ unsigned route_order(float k) {
  const unsigned u = __float_as_uint(k + 0.f);
  return u ^ ((unsigned)((int)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float route_unorder(unsigned o) { return __uint_as_float(o ^ ((o >> 31) ? 0x80000000u : 0xffffffffu)); }

// L lanes per row, C experts per lane; a round of the choice is a maximum over a lane's keys and over the lanes.  The scores of the chosen
// are taken afterwards, a lane each.
// (eight blocks an SM: 200k rows of 256 experts in groups 758 us with the 138 registers that it would take, 385 with 64 and some spills; 1M rows of 64 366 and 262,
// with six blocks 278, with seven 271)
template <typename T, int L, int C>
__global__ void __launch_bounds__(ROUTE_THREADS, C == 8 ? 8 : 1) route_kernel(const RouteParams p) {
  it_allow_next();
  it_wait_prior();
  constexpr int R = 32 / L;                       // rows of a warp
  constexpr int N = kVec<T> < C ? kVec<T> : C;    // consecutive experts of a lane
  constexpr unsigned full = 0xffffffffu;
  extern __shared__ double route_smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gl = lane % L, r = lane / L;
  // per warp: expert, key and score of its rows' choices [R][rounds] each, the fp32 keys, worths and their slacks of its rows (groups); the 64-bit ones of one row
  const int E = p.experts, per_warp = E + p.n_groups, rounds = p.k + (p.bias && p.k < E ? 1 : 0);
  double *mine64 = route_smem + (size_t)warp * per_warp;
  const int row_words = E + E / 32 + 1 + 2 * p.n_groups;   // a pad word after every 32 keys
  float *after = reinterpret_cast<float *>(route_smem + (size_t)ROUTE_WARPS * per_warp);
  const int warp_words = R * 3 * rounds + (L == 32 ? 64 : 0) + (p.n_groups > 1 ? R * row_words : 0);
  int32_t *at_s = reinterpret_cast<int32_t *>(after + (size_t)warp * warp_words);
  unsigned *order_s = reinterpret_cast<unsigned *>(at_s + R * rounds + 32);   // (one row a warp: 32 candidates, their experts behind the choices)
  float *key_s = reinterpret_cast<float *>(at_s + R * rounds + (L == 32 ? 64 : 0)), *score_s = key_s + R * rounds;
  float *keys = score_s + R * rounds + (size_t)r * row_words, *worth = keys + E + E / 32 + 1, *slack = worth + p.n_groups;
  auto expert = [&](int c) { return ((c / N) * L + gl) * N + c % N; };
  const bool vec = (E * (int)sizeof(T)) % 16 == 0 && N == kVec<T> && ((uintptr_t)p.logits & 15) == 0;
  float bias[C];
#pragma unroll
  for (int c = 0; c < C; ++c) bias[c] = p.bias && expert(c) < E ? open_key(p.bias[expert(c)]) : 0.f;   // (NaN closes: minus infinity)
  // groups: whether they are runs of lanes, and of how many; else lanes that scan one group together
  const int segment = p.group_size / N;
  const bool segments = p.n_groups > 1 && p.n_groups <= 64 && p.group_size % N == 0 && segment <= L && (segment & (segment - 1)) == 0;
  int per_group = 1;
  while (per_group * 2 * p.n_groups <= L && p.group_size % (per_group * 2) == 0) per_group *= 2;

  for (int64_t row0 = ((int64_t)blockIdx.x * ROUTE_WARPS + warp) * R; row0 < p.n; row0 += (int64_t)gridDim.x * ROUTE_WARPS * R) {
    const int64_t row = row0 + r < p.n ? row0 + r : p.n - 1;   // lanes past the last row repeat it, and store nothing
    const T *from = reinterpret_cast<const T *>(p.logits) + row * E;
    float key[C];   // logits first
#pragma unroll
    for (int c0 = 0; c0 < C; c0 += N) {
      const int e0 = expert(c0);
      if constexpr (N == kVec<T>) {
        if (vec) {
          float v[N];
          if (e0 < E) vec_to_f32(*reinterpret_cast<const uint4 *>(from + e0), v);
#pragma unroll
          for (int i = 0; i < N; ++i) key[c0 + i] = e0 < E ? open_logit(v[i]) : kClosed;
          continue;
        }
      }
#pragma unroll
      for (int i = 0; i < N; ++i) key[c0 + i] = e0 + i < E ? open_logit(to_f32(from[e0 + i])) : kClosed;
    }
    float top = 0.f, inv = 1.f;
    if (!p.sigmoid) {
      top = key[0];
#pragma unroll
      for (int c = 1; c < C; ++c) top = fmaxf(top, key[c]);
#pragma unroll
      for (int o = L / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(full, top, o));
      if (!(top > kClosed)) top = 0.f;   // nothing is open
    }
    auto raw = [&](float l, float top_of) { return p.sigmoid ? 1.f / (1.f + expf(-l)) : expf(l - top_of); };   // (a closed logit: 0)
    auto rough = [&](float l) { return p.sigmoid ? route_rcp(1.f + it_exp(-l)) : it_exp(l - top); };         // what keys are made of
    bool near = false;
    if (p.bias || p.need_sum) {
      float sum = 0.f, s[C];
#pragma unroll
      for (int c = 0; c < C; ++c) {
        s[c] = p.bias ? rough(key[c]) : raw(key[c], top);
        sum += s[c];
      }
      if (!p.sigmoid) {
#pragma unroll
        for (int o = L / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(full, sum, o);
        inv = sum > 0.f ? 1.f / sum : 0.f;
      }
      if (p.bias) {
#pragma unroll
        for (int c = 0; c < C; ++c) key[c] = key[c] > kClosed ? fmaf(s[c], inv, bias[c]) : kClosed;
      }
    }
    const float rel = p.sigmoid ? 1e-6f : 4e-6f;
    const bool exact_worth = !p.bias && p.group_best == 1;
    // What a group's worth may be off by, from its two largest keys.  With a bias: two scores of at most inv each, whose slack is at most that, and two keys and
    // their sum rounded by half an ulp each (large biases of opposite sign leave a small sum).  Without: a sum of e^-x, x < 104, each off by 2^-22 and x 2^-24.
    // (the borders worth - slack and worth + slack are rounded too: 2.5e-7 is four halves of an ulp)
    auto worth_slack = [&](float a, float b, float w) {
      if (!p.bias) return 1.6e-5f * w + 1e-30f;
      return 2.2f * rel * inv + 2.5e-7f * (fabsf(a) + (p.group_best == 2 && b > kClosed ? fabsf(b) : 0.f)) + 1e-30f;
    };
    auto worth_of = [&](float a, float b) {   // a group's two largest keys
      if (p.group_best == 1 || !(a > kClosed)) return a;
      const float second = b > kClosed ? (p.bias ? b : raw(b, top)) : 0.f;
      return (p.bias ? a : raw(a, top)) + second;
    };
    if (p.n_groups > 1 && segments) {
      // groups are runs of lanes in every chunk of N consecutive experts a lane: nothing leaves the registers
      constexpr int CH = C / N;
      // worth of this lane's group in every chunk, and what it may be off by; the least that a kept one may be worth, the most that one may that is not
      float w[CH], off[CH], keep = INFINITY, drop = kClosed;
      int rank[CH];
#pragma unroll
      for (int j = 0; j < CH; ++j) {
        float a = kClosed, b = kClosed;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          b = fmaxf(b, fminf(a, key[j * N + i]));
          a = fmaxf(a, key[j * N + i]);
        }
        for (int o = 1; o < segment; o <<= 1) {
          const float a2 = __shfl_xor_sync(full, a, o), b2 = __shfl_xor_sync(full, b, o);
          b = fmaxf(fmaxf(b, b2), fminf(a, a2));
          a = fmaxf(a, a2);
        }
        w[j] = worth_of(a, b);
        off[j] = worth_slack(a, b, w[j]);
        rank[j] = 0;
      }
      const int per_chunk = L / segment, mine = gl / segment;
#pragma unroll
      for (int jo = 0; jo < CH; ++jo)
        for (int o = 0; o < per_chunk; ++o) {
          if (jo * per_chunk + o >= p.n_groups) break;
          const float v = __shfl_sync(full, w[jo], r * L + o * segment);
#pragma unroll
          for (int j = 0; j < CH; ++j) rank[j] += v > w[j] || (v == w[j] && jo * per_chunk + o < j * per_chunk + mine);
        }
#pragma unroll
      for (int j = 0; j < CH; ++j) {
        if (!(w[j] > kClosed)) continue;   // (no open expert, or no group at all)
        if (rank[j] < p.group_k) keep = fminf(keep, w[j] - off[j]);
        else drop = fmaxf(drop, w[j] + off[j]);
      }
#pragma unroll
      for (int o = L / 2; o > 0; o >>= 1) {
        keep = fminf(keep, __shfl_xor_sync(full, keep, o));
        drop = fmaxf(drop, __shfl_xor_sync(full, drop, o));
      }
      near = !exact_worth && drop >= keep;
#pragma unroll
      for (int j = 0; j < CH; ++j)
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (rank[j] >= p.group_k) key[j * N + i] = kClosed;
    } else if (p.n_groups > 1) {
      __syncwarp();
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int e = expert(c);
        if (e < E) keys[e + (e >> 5)] = key[c];
      }
      __syncwarp();
      const int share = p.group_size / per_group, at_once = L / per_group;
      for (int g0 = 0; g0 < p.n_groups; g0 += at_once) {   // (whole warps: the lanes of a group compare notes)
        const int g = g0 + gl / per_group;
        float a = kClosed, b = kClosed;
        if (g < p.n_groups) {
          int e = g * p.group_size + (gl % per_group) * share;
          for (int i = 0; i < share; ++i, ++e) {
            const float k = keys[e + (e >> 5)];
            b = fmaxf(b, fminf(a, k));
            a = fmaxf(a, k);
          }
        }
        for (int o = 1; o < per_group; o <<= 1) {
          const float a2 = __shfl_xor_sync(full, a, o), b2 = __shfl_xor_sync(full, b, o);
          b = fmaxf(fmaxf(b, b2), fminf(a, a2));
          a = fmaxf(a, a2);
        }
        if (g < p.n_groups && gl % per_group == 0) {
          const float w = worth_of(a, b);
          worth[g] = w;
          slack[g] = worth_slack(a, b, w);
        }
      }
      __syncwarp();
      // one flag per group, in place of the keys
      float keep = INFINITY, drop = kClosed;
      for (int g = gl; g < p.n_groups; g += L) {
        const float w = worth[g];
        int rank = 0;
        for (int o = 0; o < p.n_groups; ++o) {
          const float v = worth[o];
          rank += v > w || (v == w && o < g);
        }
        keys[g] = rank < p.group_k ? 1.f : 0.f;
        if (!(w > kClosed)) continue;
        if (rank < p.group_k) keep = fminf(keep, w - slack[g]);
        else drop = fmaxf(drop, w + slack[g]);
      }
      __syncwarp();
#pragma unroll
      for (int o = L / 2; o > 0; o >>= 1) {
        keep = fminf(keep, __shfl_xor_sync(full, keep, o));
        drop = fmaxf(drop, __shfl_xor_sync(full, drop, o));
      }
      near = !exact_worth && drop >= keep;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int e = expert(c);
        if (e < E && keys[(e * p.group_magic) >> 22] == 0.f) key[c] = kClosed;
      }
    }
    __syncwarp();   // the last row's choices have been read
    // the choice, one more than asked for where its border has to be looked at
    if constexpr (L == 32) {
      // Keys as numbers, so that a warp's maximum is one instruction.  The `rounds` largest of the lanes' own largest keys bound the choice from
      // below; the keys from there on, few more than asked for, are ranked against one another, a lane each.
      unsigned k[C], best = 0;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        k[c] = key[c] > kClosed ? route_order(key[c]) : 0u;
        best = best > k[c] ? best : k[c];
      }
      unsigned least = 0, m = best;
      for (int j = 0; j < rounds;) {
        const unsigned top_m = __reduce_max_sync(full, m);
        if (top_m == 0) break;
        least = top_m;
        j += __popc(__ballot_sync(full, m == top_m));
        if (m == top_m) m = 0;
        if (j < rounds) least = 1;   // (fewer lanes with an open key than rounds: every open key)
      }
      int total = 0;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const bool in = k[c] >= least && k[c] != 0;
        const unsigned who = __ballot_sync(full, in);
        const int pos = total + __popc(who & ((1u << lane) - 1u));
        if (in && pos < 32) { at_s[rounds + pos] = expert(c); order_s[pos] = k[c]; }
        total += __popc(who);
      }
      __syncwarp();
      if (total <= 32) {
        const unsigned mine = lane < total ? order_s[lane] : 0u;
        const int e = lane < total ? at_s[rounds + lane] : 0;
        int rank = 0;
        for (int q = 0; q < total; ++q) {
          const unsigned o = order_s[q];
          rank += o > mine || (o == mine && at_s[rounds + q] < e);
        }
        if (lane < total && rank < rounds) { at_s[rank] = e; key_s[rank] = route_unorder(mine); }
        if (lane >= total && lane < rounds) { at_s[lane] = -1; key_s[lane] = kClosed; }
        if (lane + 32 < rounds) { at_s[lane + 32] = -1; key_s[lane + 32] = kClosed; }
        __syncwarp();
      } else {   // many equal keys: one after the other
        for (int j = 0; j < rounds; ++j) {
          unsigned most = 0;
          int at = ROUTE_MAX_EXPERTS;
#pragma unroll
          for (int c = 0; c < C; ++c)
            if (k[c] > most) { most = k[c]; at = expert(c); }
          const unsigned of_all = __reduce_max_sync(full, most);
          const int e = (int)__reduce_min_sync(full, most == of_all ? (unsigned)at : (unsigned)ROUTE_MAX_EXPERTS);
          if (lane == 0) { at_s[j] = of_all ? e : -1; key_s[j] = of_all ? route_unorder(of_all) : kClosed; }
#pragma unroll
          for (int c = 0; c < C; ++c)
            if (expert(c) == e) k[c] = 0u;
          __syncwarp();
        }
      }
    } else {
      for (int j = 0; j < rounds; ++j) {
        float best = kClosed;
        int at = ROUTE_MAX_EXPERTS;
#pragma unroll
        for (int c = 0; c < C; ++c)
          if (key[c] > best) { best = key[c]; at = expert(c); }
#pragma unroll
        for (int o = L / 2; o > 0; o >>= 1) {
          const float b = __shfl_xor_sync(full, best, o);
          const int a = __shfl_xor_sync(full, at, o);
          if (b > best || (b == best && a < at)) { best = b; at = a; }
        }
#pragma unroll
        for (int c = 0; c < C; ++c)
          if (expert(c) == at) key[c] = kClosed;
        if (gl == 0) { at_s[r * rounds + j] = best > kClosed ? at : -1; key_s[r * rounds + j] = best; }
      }
      __syncwarp();
    }
    // scores of the chosen, a lane each: unbiased, and divided by the row's sum where the keys are
    for (int i0 = 0; i0 < R * rounds; i0 += 32) {
      const int i = i0 + lane, rr = R == 1 ? 0 : (i < R * rounds ? i / rounds : 0);
      const float t = __shfl_sync(full, top, rr * L), f = __shfl_sync(full, inv, rr * L);
      if (i < R * rounds) {
        const int e = at_s[i];
        float w = 0.f;
        if (e >= 0) {
          const int64_t row_i = row0 + rr < p.n ? row0 + rr : p.n - 1;
          w = raw(p.bias ? open_logit(to_f32(reinterpret_cast<const T *>(p.logits)[row_i * E + e])) : key_s[i], t) * f;
        }
        score_s[i] = w;
      }
    }
    __syncwarp();
    unsigned again = 0;   // rows that are taken again, a bit each
    const bool may_again = p.bias || p.sigmoid || p.n_groups > 1;   // (a softmax's largest score is else among the chosen)
    for (int i0 = 0; i0 < R * rounds; i0 += 32) {
      const int i = i0 + lane, rr = R == 1 ? 0 : (i < R * rounds ? i / rounds : 0), j = i - rr * rounds;
      const float t = __shfl_sync(full, top, rr * L), most = __shfl_sync(full, inv, rr * L);   // most: the largest score that there can be (a sigmoid: 1)
      bool close = false;
      if (i < R * rounds) {
        float sum = 0.f;
        if (p.renorm)
          for (int q = 0; q < p.k; ++q) sum += score_s[rr * rounds + q];
        const float w = score_s[i], key_i = key_s[i];
        if (p.bias && j > 0 && at_s[i] >= 0) {
          // (-ln of a score is at least its exponent: a softmax divides by 1 or more, a sigmoid by 1 + e^-x)
          const float before = score_s[i - 1];
          close = route_near(key_s[i - 1], key_i, route_slack(before, __logf(fmaxf(before, 1e-38f))),
                             j == p.k ? most : route_slack(w, __logf(fmaxf(w, 1e-38f))), rel);
        }
        if (j < p.k && row0 + rr < p.n) {
          const int64_t to = (row0 + rr) * p.k + j;
          const int e = at_s[i];
          p.ids[to] = e;
          p.weights[to] = (p.renorm ? (sum > 0.f ? w / sum : 0.f) : w) * p.scale;
          if (p.renorm && e >= 0 && w < 1.2e-37f)
            close |= route_tiny(p.sigmoid, w, sum, open_logit(to_f32(reinterpret_cast<const T *>(p.logits)[(row0 + rr) * E + e])), t);
        }
      }
      if (may_again) again |= __reduce_or_sync(full, close ? 1u << rr : 0u);
    }
    if (p.n_groups > 1) again |= __reduce_or_sync(full, near ? 1u << r : 0u);
    while (again) {
      const int which = __ffs(again) - 1;
      again &= again - 1;
      if (row0 + which < p.n) route_row_exact(p, p.logits, sizeof(T) == 2, row0 + which, mine64, lane);
      __syncwarp();
    }
  }
}

// Few experts, few places, no groups: a thread per row, its best keys kept in order as the experts go by.  KL: keys kept (with a bias
// one more than top_k, whose border is looked at).
template <typename T, int C, int KL>
__global__ void __launch_bounds__(ROUTE_THREADS) route_thread_kernel(const RouteParams p) {
  it_allow_next();
  it_wait_prior();
  constexpr int N = kVec<T>;
  constexpr unsigned full = 0xffffffffu;
  extern __shared__ double route_smem[];
  const int E = p.experts, lane = threadIdx.x & 31;
  double *mine64 = route_smem + (size_t)(threadIdx.x >> 5) * (E + p.n_groups);
  const bool vec = (E * (int)sizeof(T)) % 16 == 0 && ((uintptr_t)p.logits & 15) == 0;
  for (int64_t row0 = (int64_t)blockIdx.x * ROUTE_THREADS; row0 < p.n; row0 += (int64_t)gridDim.x * ROUTE_THREADS) {
    const bool real = row0 + threadIdx.x < p.n;
    const int64_t row = real ? row0 + threadIdx.x : p.n - 1;
    const T *from = reinterpret_cast<const T *>(p.logits) + row * E;
    float key[C];
    if (vec) {
#pragma unroll
      for (int c0 = 0; c0 < C; c0 += N) {
        float v[N];
        if (c0 < E) vec_to_f32(*reinterpret_cast<const uint4 *>(from + c0), v);
#pragma unroll
        for (int i = 0; i < N; ++i) key[c0 + i] = c0 < E ? open_logit(v[i]) : kClosed;
      }
    } else {
#pragma unroll
      for (int c = 0; c < C; ++c) key[c] = c < E ? open_logit(to_f32(from[c])) : kClosed;
    }
    float top = key[0], inv = 1.f;
#pragma unroll
    for (int c = 1; c < C; ++c) top = fmaxf(top, key[c]);
    if (!(top > kClosed)) top = 0.f;
    auto raw = [&](float l) { return p.sigmoid ? 1.f / (1.f + expf(-l)) : expf(l - top); };
    auto rough = [&](float l) { return p.sigmoid ? route_rcp(1.f + it_exp(-l)) : it_exp(l - top); };   // what keys are made of
    if (p.bias || p.need_sum) {
      float sum = 0.f;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        sum += p.bias ? rough(key[c]) : raw(key[c]);
      }
      if (!p.sigmoid) inv = sum > 0.f ? 1.f / sum : 0.f;
      if (p.bias) {
#pragma unroll
        for (int c = 0; c < C; ++c)
          if (c < E) key[c] = key[c] > kClosed ? open_key(fmaf(rough(key[c]), inv, p.bias[c])) : kClosed;
      }
    }
    float best[KL];
    int at[KL];
#pragma unroll
    for (int j = 0; j < KL; ++j) { best[j] = kClosed; at[j] = -1; }
#pragma unroll
    for (int c = 0; c < C; ++c) {   // (an equal key that comes later stays behind)
#pragma unroll
      for (int j = KL - 1; j > 0; --j) {
        const bool past = key[c] > best[j - 1], here = key[c] > best[j];
        at[j] = past ? at[j - 1] : (here ? c : at[j]);
        best[j] = past ? best[j - 1] : (here ? key[c] : best[j]);
      }
      if (key[c] > best[0]) { best[0] = key[c]; at[0] = c; }
    }
    float w[KL], sum = 0.f;
    bool near = false;
#pragma unroll
    for (int j = 0; j < KL; ++j) {
      w[j] = 0.f;
      float slack = 0.f;
      if (at[j] >= 0) {
        const float l = p.bias ? open_logit(to_f32(from[at[j]])) : best[j];
        w[j] = raw(l) * inv;
        slack = route_slack(w[j], p.sigmoid ? fminf(l, 0.f) : l - top);
      }
      if (j < p.k) sum += w[j];
      if (p.bias && j > 0 && j <= p.k && at[j] >= 0) {
        const float l = open_logit(to_f32(from[at[j - 1]]));
        near |= route_near(best[j - 1], best[j], route_slack(w[j - 1], p.sigmoid ? fminf(l, 0.f) : l - top), j == p.k ? inv : slack, p.sigmoid ? 1e-6f : 4e-6f);
      }
    }
    if (p.renorm && (p.bias || p.sigmoid)) {   // (a softmax's largest score is else among the chosen)
#pragma unroll
      for (int j = 0; j < KL; ++j)
        if (j < p.k && at[j] >= 0 && w[j] < 1.2e-37f) near |= route_tiny(p.sigmoid, w[j], sum, open_logit(to_f32(from[at[j]])), top);
    }
#pragma unroll
    for (int j = 0; j < KL; ++j) w[j] = (p.renorm ? (sum > 0.f ? w[j] / sum : 0.f) : w[j]) * p.scale;
    if (real) {
      int32_t *ids = p.ids + row * p.k;
      float *ws = p.weights + row * p.k;
      if (p.k == 2 && (((uintptr_t)p.ids | (uintptr_t)p.weights) & 7) == 0) {
        *reinterpret_cast<int2 *>(ids) = make_int2(at[0], at[1]);
        *reinterpret_cast<float2 *>(ws) = make_float2(w[0], w[1]);
      } else {
#pragma unroll
        for (int j = 0; j < KL; ++j)
          if (j < p.k) { ids[j] = at[j]; ws[j] = w[j]; }
      }
    }
    unsigned again = p.bias || p.sigmoid ? __ballot_sync(full, near && real) : 0u;
    while (again) {
      const int which = __ffs(again) - 1;
      again &= again - 1;
      route_row_exact(p, p.logits, sizeof(T) == 2, row0 + (threadIdx.x & ~31) + which, mine64, lane);
      __syncwarp();
    }
  }
}

it_status launch_route(void (*kernel)(const RouteParams), const RouteParams &p, int rows_per_block, size_t smem, double bytes, double flops, cudaStream_t st) {
  if (smem > 48 * 1024) IT_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
  const int64_t blocks = (p.n + rows_per_block - 1) / rows_per_block, most = (int64_t)it_current_sms() * 16;
  IT_LAUNCH(IT_K_ROUTE, bytes, flops, st,
            IT_CUDA_TRY(it_launch_pdl(kernel, dim3((unsigned)(blocks < most ? blocks : most)), dim3(ROUTE_THREADS), smem, st, p)));
  return IT_OK;
}

template <typename T, int L, int C>
it_status launch(const RouteParams &p, double bytes, double flops, cudaStream_t st) {
  constexpr int R = 32 / L;
  const size_t warp64 = (size_t)(p.experts + p.n_groups) * 8;
  const size_t warp32 = ((size_t)R * 3 * (p.k + 1) + (L == 32 ? 64 : 0) + (p.n_groups > 1 ? (size_t)R * (p.experts + p.experts / 32 + 1 + 2 * p.n_groups) : 0)) * 4;
  return launch_route(route_kernel<T, L, C>, p, ROUTE_WARPS * R, ROUTE_WARPS * (warp64 + warp32), bytes, flops, st);
}

template <typename T, int C>
it_status launch_thread(const RouteParams &p, double bytes, double flops, cudaStream_t st) {
  const int kl = p.k + (p.bias ? 1 : 0);
  const size_t smem = (size_t)ROUTE_WARPS * (p.experts + p.n_groups) * 8;
  if (kl <= 2) return launch_route(route_thread_kernel<T, C, 2>, p, ROUTE_THREADS, smem, bytes, flops, st);
  if (kl <= 3) return launch_route(route_thread_kernel<T, C, 3>, p, ROUTE_THREADS, smem, bytes, flops, st);
  return launch_route(route_thread_kernel<T, C, 5>, p, ROUTE_THREADS, smem, bytes, flops, st);
}

template <typename T>
it_status dispatch(const RouteParams &p, double bytes, double flops, cudaStream_t st) {
  const int e = p.experts;
  if (e <= 32 && p.k <= 4 && p.n_groups == 1) {
    if (e <= 8) return launch_thread<T, 8>(p, bytes, flops, st);
    if (e <= 16) return launch_thread<T, 16>(p, bytes, flops, st);
    return launch_thread<T, 32>(p, bytes, flops, st);
  }
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
