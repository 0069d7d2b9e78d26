// Device helpers of the softmax operators: 16-bit types, vector loads of rows,
// base-2 exponentials, and which rows a call ignores.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "softmax.h"

namespace esspt {

__device__ __forceinline__ float exp2_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
template <typename T>
__device__ __forceinline__ T from_float(float x);
template <>
__device__ __forceinline__ float from_float<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <>
__device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }

// VEC values of type T at p (VEC * sizeof(T) bytes, aligned to that), as fp32.
template <typename T, int VEC>
__device__ __forceinline__ void load_vec(const T* p, float (&x)[VEC]) {
  struct alignas(VEC * sizeof(T)) Pack {
    T v[VEC];
  };
  const Pack k = *reinterpret_cast<const Pack*>(p);
#pragma unroll
  for (int i = 0; i < VEC; ++i) x[i] = to_float(k.v[i]);
}
template <typename T, int VEC>
__device__ __forceinline__ void store_vec(T* p, const float (&x)[VEC]) {
  struct alignas(VEC * sizeof(T)) Pack {
    T v[VEC];
  } k;
#pragma unroll
  for (int i = 0; i < VEC; ++i) k.v[i] = from_float<T>(x[i]);
  *reinterpret_cast<Pack*>(p) = k;
}

// Whether row t takes part: a target inside the catalogue, or a list with a share.
__device__ __forceinline__ bool row_kept(const TargetArgs& a, int64_t t) {
  return a.logits ? a.self[t] != kIgnored : (uint32_t)a.ids[t] < (uint32_t)a.V;
}

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
  return x;
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
