// Device helpers of the softmax operators: base-2 exponentials, and which rows a call
// ignores.
#pragma once

#include "rows.cuh"
#include "softmax.h"

namespace esspt {

__device__ __forceinline__ float exp2_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// Whether row t takes part: a target inside the catalogue, or a list with a share.
__device__ __forceinline__ bool row_kept(const TargetArgs& a, int64_t t) {
  return a.logits ? a.self[t] != kIgnored : (uint32_t)a.ids[t] < (uint32_t)a.V;
}

__device__ __forceinline__ float warp_max(float x) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, off));
  return x;
}

// A running maximum and the sum of 2^(s - maximum): another such pair is added.
// While the maximum is -infinity the sum is zero, and NaN sums stay NaN.
__device__ __forceinline__ void merge_stat(float& m, float& l, float m2, float l2) {
  const float top = fmaxf(m, m2), at = top == -INFINITY ? 0.f : top;
  l = l * exp2_fast(m - at) + l2 * exp2_fast(m2 - at);
  m = top;
}

}  // namespace esspt
