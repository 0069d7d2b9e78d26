// Layer norm, forward and backward: the C-ABI, and the kernel that adds the blocks' sums for the weights.  The others are in
// norm.cuh.
#include <cmath>
#include <new>
#include <type_traits>

#include "chained.cuh"
#include "norm.h"
#include "operator.h"
#include "ptx.cuh"
#include "rows.cuh"

using namespace esspt;

struct esspt_norm {
  esspt_norm_config cfg{};
  cudaStream_t st = nullptr;
  char* base = nullptr;
  int sms = 0;
  Errors err;
};

namespace {

thread_local Errors g_create;

constexpr int kMaxSms = 256;  // what the workspace is sized for

// dw and db from the blocks' sums: 32 columns to a block, whose warps take every 32nd block's.
constexpr int kWeightWarps = 32;
template <typename W>
__global__ void __launch_bounds__(32 * kWeightWarps) norm_weights_kernel(const float* part, int blocks, int D, W* dw, W* db) {
  __shared__ float sums[kWeightWarps][33];
  const int c = blockIdx.x * 32 + (threadIdx.x & 31), warp = threadIdx.x / 32;
  float s = 0.f;
  await_previous_kernel();
  if (c < 2 * D)
    for (int k0 = warp; k0 < blocks; k0 += 8 * kWeightWarps) {
      float x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) x[u] = k0 + u * kWeightWarps < blocks ? part[(int64_t)(k0 + u * kWeightWarps) * 2 * D + c] : 0.f;
#pragma unroll
      for (int u = 0; u < 8; ++u) s += x[u];
    }
  sums[warp][threadIdx.x & 31] = s;
  __syncthreads();
  if (warp || c >= 2 * D) return;
  s = 0.f;
#pragma unroll
  for (int k = 0; k < kWeightWarps; ++k) s += sums[k][threadIdx.x];
  W* to = c < D ? dw : db;
  if (to) to[c < D ? c : c - D] = from_float<W>(s);
}

const char* config_fault(const esspt_norm_config* c) {
  if (!c) return "null config";
  if (c->max_rows < 1 || c->max_rows >= ((int64_t)1 << 31)) return "max_rows must be in [1, 2^31 - 1]";
  static_assert(kNormWidth == 8192, "the text below");
  if (c->width < 1 || c->width > kNormWidth) return "width must be in [1, 8192]";
  if (c->dtype < ESSPT_F32 || c->dtype > ESSPT_F16) return "unknown dtype";
  if (c->weight_dtype != ESSPT_F32 && c->weight_dtype != c->dtype) return "weight_dtype must be fp32 or the rows'";
  if (!(c->eps > 0.f) || !std::isfinite(c->eps)) return "eps must be positive and finite";
  return nullptr;
}

size_t workspace(const esspt_norm_config& c) {
  if (!c.backward) return 256;
  const Spread a = spread(c.width, 16 / (int)size_of(c.dtype), true), b = spread(c.width, 1, true);
  const size_t blocks = (size_t)kMaxSms * (a.resident > b.resident ? a.resident : b.resident);
  return 256 + up256(blocks * 2 * c.width * sizeof(float));
}

cudaError_t launch(const esspt_norm_config& c, Norm& a, bool back, int bytes, int sms, unsigned* blocks, cudaStream_t st) {
  a.weight_f32 = c.weight_dtype == ESSPT_F32;
  if (c.dtype == ESSPT_F32) return launch_norm<float>(a, back, bytes, sms, blocks, st);
  if (c.dtype == ESSPT_BF16) return launch_norm<__nv_bfloat16>(a, back, bytes, sms, blocks, st);
  return launch_norm<__half>(a, back, bytes, sms, blocks, st);
}

}  // namespace

extern "C" {

size_t esspt_norm_workspace_bytes(const esspt_norm_config* cfg) { return config_fault(cfg) ? 0 : workspace(*cfg); }

esspt_status esspt_norm_create(const esspt_norm_config* cfg, void* d_workspace, size_t bytes, esspt_norm** out) {
  g_create.text[0] = 0;
  if (const char* why = config_fault(cfg)) return g_create.fail(ESSPT_EINVAL, why);
  if (!out || !d_workspace || misaligned(d_workspace, 256)) return g_create.fail(ESSPT_EINVAL, "null or misaligned pointer");
  if (bytes < workspace(*cfg)) return g_create.fail(ESSPT_ENOSPC, "workspace too small");
  int dev = 0, sms = 0;
  ESSPT_CUDA(g_create, cudaGetDevice(&dev));
  ESSPT_CUDA(g_create, cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  esspt_norm* nm = new (std::nothrow) esspt_norm;
  if (!nm) return g_create.fail(ESSPT_ENOSPC, "out of host memory");
  nm->cfg = *cfg;
  nm->st = static_cast<cudaStream_t>(cfg->stream);
  nm->base = static_cast<char*>(d_workspace);
  nm->sms = sms < kMaxSms ? sms : kMaxSms;
  *out = nm;
  return ESSPT_OK;
}

esspt_status esspt_norm_destroy(esspt_norm* nm) {
  if (!nm) return ESSPT_OK;
  const cudaError_t e = cudaStreamSynchronize(nm->st);
  delete nm;
  return e == cudaSuccess ? ESSPT_OK : g_create.cuda(e, "esspt_norm_destroy");
}

esspt_status esspt_norm_forward(esspt_norm* nm, const void* d_x, int64_t x_stride, int64_t n, const void* d_weight,
                                const void* d_bias, void* d_y, float* d_mean, float* d_rstd) {
  if (!nm) return ESSPT_EINVAL;
  nm->err.text[0] = 0;
  const esspt_norm_config& c = nm->cfg;
  const size_t size = size_of(c.dtype), wsize = size_of(c.weight_dtype);
  if (n < 0 || n > c.max_rows) return nm->err.fail(ESSPT_EINVAL, "n must be in [0, max_rows]");
  if (!d_mean != !d_rstd) return nm->err.fail(ESSPT_EINVAL, "both statistics or neither");
  if (n == 0) return ESSPT_OK;
  if (!d_x || !d_y) return nm->err.fail(ESSPT_EINVAL, "null pointer");
  if (x_stride < c.width) return nm->err.fail(ESSPT_EINVAL, "a row stride is below the width");
  if (misaligned(d_x, size) || misaligned(d_y, size) || misaligned(d_weight, wsize) || misaligned(d_bias, wsize) ||
      misaligned(d_mean, 4) || misaligned(d_rstd, 4))
    return nm->err.fail(ESSPT_EINVAL, "a pointer is not aligned to its type");
  Norm a{};
  a.x = d_x, a.x_stride = x_stride, a.n = n, a.D = c.width, a.inv_D = 1.f / c.width, a.eps = c.eps;
  a.weight = d_weight, a.bias = d_bias, a.y = d_y, a.mean = d_mean, a.rstd = d_rstd;
  unsigned blocks = 0;
  const int bytes = vector_bytes(c.width, size, (uintptr_t)d_x | (uintptr_t)d_y | (uintptr_t)x_stride * size);
  ESSPT_CUDA(nm->err, launch(c, a, false, bytes, nm->sms, &blocks, nm->st));
  return ESSPT_OK;
}

esspt_status esspt_norm_backward(esspt_norm* nm, const void* d_dy, int64_t dy_stride, const void* d_x,
                                 int64_t x_stride, int64_t n, const void* d_weight, const float* d_mean,
                                 const float* d_rstd, void* d_dx, void* d_dweight, void* d_dbias) {
  if (!nm) return ESSPT_EINVAL;
  nm->err.text[0] = 0;
  const esspt_norm_config& c = nm->cfg;
  const size_t size = size_of(c.dtype), wsize = size_of(c.weight_dtype);
  if (!c.backward) return nm->err.fail(ESSPT_EINVAL, "the handle was made without backward");
  if (n < 0 || n > c.max_rows) return nm->err.fail(ESSPT_EINVAL, "n must be in [0, max_rows]");
  if (n > 0 && (!d_dy || !d_x || !d_mean || !d_rstd)) return nm->err.fail(ESSPT_EINVAL, "null pointer");
  if (n > 0 && (x_stride < c.width || dy_stride < c.width))
    return nm->err.fail(ESSPT_EINVAL, "a row stride is below the width");
  if (misaligned(d_x, size) || misaligned(d_dy, size) || misaligned(d_dx, size) || misaligned(d_weight, wsize) ||
      misaligned(d_dweight, wsize) || misaligned(d_dbias, wsize) || misaligned(d_mean, 4) || misaligned(d_rstd, 4))
    return nm->err.fail(ESSPT_EINVAL, "a pointer is not aligned to its type");
  if (n == 0) {
    if (d_dweight) ESSPT_CUDA(nm->err, cudaMemsetAsync(d_dweight, 0, c.width * wsize, nm->st));
    if (d_dbias) ESSPT_CUDA(nm->err, cudaMemsetAsync(d_dbias, 0, c.width * wsize, nm->st));
    return ESSPT_OK;
  }
  Norm a{};
  a.x = d_x, a.x_stride = x_stride, a.dy = d_dy, a.dy_stride = dy_stride, a.n = n, a.D = c.width;
  a.inv_D = 1.f / c.width, a.weight = d_weight, a.y = d_dx;
  a.mean = const_cast<float*>(d_mean), a.rstd = const_cast<float*>(d_rstd);
  a.part = reinterpret_cast<float*>(nm->base + 256), a.want_w = d_dweight || d_dbias;
  if (!a.want_w && !d_dx) return ESSPT_OK;
  unsigned blocks = 0;
  const int bytes = vector_bytes(c.width, size, (uintptr_t)d_x | (uintptr_t)d_dy | (uintptr_t)d_dx |
                                                    (uintptr_t)x_stride * size | (uintptr_t)dy_stride * size);
  ESSPT_CUDA(nm->err, launch(c, a, true, bytes, nm->sms, &blocks, nm->st));
  if (!a.want_w) return ESSPT_OK;
  const unsigned columns = (2 * c.width + 31) / 32;
  auto weights = [&](auto* type) {
    using W = std::remove_pointer_t<decltype(type)>;
    return launch_chained(norm_weights_kernel<W>, columns, 32 * kWeightWarps, nm->st, true, (const float*)a.part, (int)blocks, c.width,
                          (W*)d_dweight, (W*)d_dbias);
  };
  const cudaError_t e = c.weight_dtype == ESSPT_F32    ? weights((float*)nullptr)
                        : c.weight_dtype == ESSPT_BF16 ? weights((__nv_bfloat16*)nullptr)
                                                       : weights((__half*)nullptr);
  ESSPT_CUDA(nm->err, e);
  return ESSPT_OK;
}

const char* esspt_norm_last_error(const esspt_norm* nm) { return nm ? nm->err.text : g_create.text; }

}  // extern "C"
