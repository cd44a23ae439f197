// Declarations shared by the files of it_experts_forward.
#pragma once

#include "rows.cuh"

struct it_experts_args {
  it_experts_desc d;
  int64_t n;
  int n1;                  // columns of W1
  const void *x;
  const float *x_scale;
  const int32_t *ids;
  const float *weights;
  void *out;
  int *status;             // device word: 0, or 1 after a wait that gave up
  int sms;
};

// ----------------------------------------------------------------------------- experts_plan.cu
// Places sorted by expert: every expert's places fill whole tiles of 128 positions, the last one padded with -1.
struct it_experts_plan {
  int32_t *order;          // [tiles_max * 128] the place at a position, or -1
  int32_t *position;       // [places] where a place went (places of no expert: undefined)
  int32_t *tile_expert;    // [tiles_max]
  int32_t *n_tiles;        // device word
  int32_t *counts;         // [blocks][n_experts] scratch
  int64_t tiles_max;
};
int64_t it_experts_tiles_max(int64_t places, int n_experts);
size_t it_experts_count_words(int64_t places, int n_experts);
// Also zeroes a.status and, where a vertex has one place only, the rows of `out` whose id is no expert.
it_status it_launch_experts_plan(const it_experts_args &a, const it_experts_plan &q, cudaStream_t st);
// fp32 values as three bf16 parts each (24 bits: 8 a part, cut off, so that the parts add up exactly): dst[i] is [3, elems[i]], x_parts [3, positions, row]
// with the rows of x in the order of the positions.
struct it_experts_parts {
  const float *src[2]; __nv_bfloat16 *dst[2]; int64_t elems[2]; int count;
  const float *x; __nv_bfloat16 *x_parts; int row, top_k; const int32_t *order, *n_tiles; int64_t tiles_max;
};
it_status it_launch_experts_parts(const it_experts_parts &q, int sms, cudaStream_t st);
// Rows of x in the order of the positions.
it_status it_launch_experts_rows(const it_experts_args &a, const it_experts_plan &q, void *to, cudaStream_t st);

// ----------------------------------------------------------------------------- experts_tc.cu
enum it_expert_store {
  IT_EXPERT_HIDDEN = 0,    // row `position` of a bf16 matrix
  IT_EXPERT_PARTS = 1,     // row `position` of three bf16 matrices, tiles_max * 128 rows apart
  IT_EXPERT_SUMS = 2,      // row `position` of an fp32 matrix
  IT_EXPERT_OUT_BF16 = 3,  // row `place` (top_k = 1) of the output, times the place's weight
  IT_EXPERT_OUT_F32 = 4
};
// One product of every tile with its expert's weights.
struct it_expert_gemm {
  const void *A;           // rows of K elements: of x, found by place / top_k (gather = 1), or by position
  int gather;
  int64_t a_rows;          // of one part
  const void *W;           // [parts][n_experts][K, w_cols]
  int K, w_cols, cols;     // cols: of the result (gated: half of w_cols)
  int parts;               // 3: fp32 operands as bf16 parts
  int eight;               // operands in e4m3
  int act, gated;
  const float *bias, *w_scale, *x_scale;
  it_expert_store store;
  void *dst;
  uint32_t spin_limit;     // polls after which a wait gives up (0: the default)
  int no_loads;            // test hook: issue no operand copies
};
it_status it_launch_expert_gemm(const it_experts_args &a, const it_experts_plan &q, const it_expert_gemm &g, cudaStream_t st);

// ----------------------------------------------------------------------------- experts_fused.cu
// Both products in one kernel, the hidden row never in memory; dst: fp32 rows by position (top_k > 1), or the output.
bool it_experts_fused(const it_experts_desc &d);
it_status it_launch_experts_fused(const it_experts_args &a, const it_experts_plan &q, void *dst, uint32_t spin_limit, int no_loads, cudaStream_t st);

// ----------------------------------------------------------------------------- experts.cu
// Activations of the experts, in fp32.
#ifdef __CUDACC__
__device__ __forceinline__ float it_max_nan(float a, float b) {   // NaN if either is
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float it_expert_act(float v, int act) {
  if (act == IT_ACT_RELU) return it_max_nan(v, 0.f);
  if (act == IT_ACT_ELU) return it_elu(v);
  if (act == IT_ACT_SILU) return __fdividef(v, 1.f + it_exp(-v));   // (off by a few ulp; 0 where the divisor passes 2^126)
  return v;
}
#endif
