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

// ----------------------------------------------------------------------------- experts.cu
// Activations of the experts, in fp32.
#ifdef __CUDACC__
__device__ __forceinline__ float it_expert_act(float v, int act) {
  if (act == IT_ACT_RELU) return fmaxf(v, 0.f);
  if (act == IT_ACT_ELU) return it_elu(v);
  if (act == IT_ACT_SILU) return v / (1.f + it_exp(-v));
  return v;
}
#endif
