// Layer norm, forward and backward: kernels and C-ABI.
//
// A group of `threads` lanes holds a row in registers (a part of a warp, a warp, or a whole
// block for wide rows), N vectors of VEC values a thread, so that a row is read once: the mean first,
// then the variance from differences to it.  All arithmetic in fp32.
#include <cmath>
#include <new>
#include <type_traits>

#include "operator.h"
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

constexpr int kMaxSms = 256;   // what the workspace is sized for
constexpr int kBlocksPerSm = 4;  // of the backward pass, whose blocks keep partial sums

struct Norm {
  const void *x, *dy;
  int64_t x_stride, dy_stride, n;
  int32_t D;
  int32_t lanes;  // threads of a row: a power of two up to 32, or the block
  float inv_D, eps;
  const void *weight, *bias;
  void* y;        // dx in the backward pass
  float *mean, *rstd;
  float* part;    // [blocks][2][D] sums for dw and db
  int want_w;     // whether they are asked for
};

// The sum over a row's group of threads; `shared` has a float2 for each warp.
template <bool WIDE>
__device__ __forceinline__ float2 group_sum(float2 v, int lanes, float2* shared) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) {
    if (!WIDE && off >= lanes) continue;
    v.x += __shfl_xor_sync(0xffffffffu, v.x, off);
    v.y += __shfl_xor_sync(0xffffffffu, v.y, off);
  }
  if (WIDE) {
    const int warp = threadIdx.x / 32, warps = blockDim.x / 32;
    if ((threadIdx.x & 31) == 0) shared[warp] = v;
    __syncthreads();
    v = make_float2(0.f, 0.f);
    for (int i = 0; i < warps; ++i) v.x += shared[i].x, v.y += shared[i].y;
    __syncthreads();
  }
  return v;
}

template <typename T, int VEC, int N>
__device__ __forceinline__ void load_row(const T* row, int D, int lane, int lanes, bool live, float (&x)[N][VEC]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int c = (lane + i * lanes) * VEC;
#pragma unroll
    for (int j = 0; j < VEC; ++j) x[i][j] = 0.f;
    if (live && c < D) load_vec<T, VEC>(row + c, x[i]);
  }
}

// Weights by single values: they may stand anywhere, and come from the caches.
template <typename W, int VEC, int N>
__device__ __forceinline__ void load_weights(const void* from, float otherwise, int D, int lane, int lanes, float (&x)[N][VEC]) {
  const W* w = static_cast<const W*>(from);
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      const int c = (lane + i * lanes) * VEC + j;
      x[i][j] = w && c < D ? to_float(w[c]) : otherwise;
    }
}

template <typename T, typename W, int VEC, int N, bool WIDE>
__global__ void __launch_bounds__(WIDE ? 1024 : 256) norm_forward_kernel(Norm a) {
  __shared__ float2 shared[32];
  const int lanes = WIDE ? blockDim.x : a.lanes, lane = threadIdx.x & (WIDE ? ~0 : lanes - 1);
  const int64_t t = WIDE ? blockIdx.x : (int64_t)blockIdx.x * (blockDim.x / lanes) + threadIdx.x / lanes;
  const bool live = t < a.n;
  float x[N][VEC], w[N][VEC], b[N][VEC];
  load_row<T, VEC, N>(static_cast<const T*>(a.x) + t * a.x_stride, a.D, lane, lanes, live, x);
  load_weights<W, VEC, N>(a.weight, 1.f, a.D, lane, lanes, w);
  load_weights<W, VEC, N>(a.bias, 0.f, a.D, lane, lanes, b);
  float2 s = make_float2(0.f, 0.f);
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int j = 0; j < VEC; ++j) s.x += x[i][j];
  const float mean = group_sum<WIDE>(s, lanes, shared).x * a.inv_D;
  s.x = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      x[i][j] -= mean;
      if ((lane + i * lanes) * VEC + j < a.D) s.x += x[i][j] * x[i][j];
    }
  const float rstd = 1.f / sqrtf(group_sum<WIDE>(s, lanes, shared).x * a.inv_D + a.eps);
  if (!live) return;
  T* y = static_cast<T*>(a.y) + t * a.D;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int c = (lane + i * lanes) * VEC;
#pragma unroll
    for (int j = 0; j < VEC; ++j) x[i][j] = x[i][j] * rstd * w[i][j] + b[i][j];
    if (c < a.D) store_vec<T, VEC>(y + c, x[i]);
  }
  if (lane == 0 && a.mean) a.mean[t] = mean, a.rstd[t] = rstd;
}

// Blocks stay and go through rows; a thread's columns are the same in all of them, and it keeps their sums for dw
// and db.  At the end the groups of a block add theirs, one behind the other.
template <typename T, typename W, int VEC, int N, bool WIDE>
__global__ void __launch_bounds__(WIDE ? 1024 : 256) norm_backward_kernel(Norm a) {
  extern __shared__ float sums[];  // [2][D]
  __shared__ float2 shared[32];
  const int lanes = WIDE ? blockDim.x : a.lanes, lane = threadIdx.x & (WIDE ? ~0 : lanes - 1);
  const int groups = blockDim.x / lanes, group = threadIdx.x / lanes;
  float w[N][VEC], dw[N][VEC] = {}, db[N][VEC] = {};
  load_weights<W, VEC, N>(a.weight, 1.f, a.D, lane, lanes, w);
  for (int64_t t0 = (int64_t)blockIdx.x * groups; t0 < a.n; t0 += (int64_t)gridDim.x * groups) {
    const int64_t t = t0 + group;
    const bool live = t < a.n;
    float x[N][VEC], dy[N][VEC];
    load_row<T, VEC, N>(static_cast<const T*>(a.x) + t * a.x_stride, a.D, lane, lanes, live, x);
    load_row<T, VEC, N>(static_cast<const T*>(a.dy) + t * a.dy_stride, a.D, lane, lanes, live, dy);
    const float mean = live ? a.mean[t] : 0.f, rstd = live ? a.rstd[t] : 0.f;
    float2 s = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        x[i][j] = (x[i][j] - mean) * rstd;
        dw[i][j] += dy[i][j] * x[i][j];
        db[i][j] += dy[i][j];
        dy[i][j] *= w[i][j];
        if ((lane + i * lanes) * VEC + j < a.D) s.x += dy[i][j], s.y += dy[i][j] * x[i][j];
      }
    s = group_sum<WIDE>(s, lanes, shared);
    s.x *= a.inv_D, s.y *= a.inv_D;
    if (!live || !a.y) continue;
    T* dx = static_cast<T*>(a.y) + t * a.D;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = (lane + i * lanes) * VEC;
#pragma unroll
      for (int j = 0; j < VEC; ++j) x[i][j] = rstd * (dy[i][j] - s.x - x[i][j] * s.y);
      if (c < a.D) store_vec<T, VEC>(dx + c, x[i]);
    }
  }
  if (!a.want_w) return;
  for (int k = 0; k < groups; ++k) {
    if (group == k) {
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          const int c = (lane + i * lanes) * VEC + j;
          if (c < a.D) {
            sums[c] = (k ? sums[c] : 0.f) + dw[i][j];
            sums[a.D + c] = (k ? sums[a.D + c] : 0.f) + db[i][j];
          }
        }
    }
    __syncthreads();
  }
  for (int c = threadIdx.x; c < 2 * a.D; c += blockDim.x) a.part[(int64_t)blockIdx.x * 2 * a.D + c] = sums[c];
}

// dw and db from the blocks' sums: 32 columns to a block, a warp for every eighth block's.
template <typename W>
__global__ void __launch_bounds__(256) norm_weights_kernel(const float* part, int blocks, int D, W* dw, W* db) {
  __shared__ float sums[8][33];
  const int c = blockIdx.x * 32 + (threadIdx.x & 31), warp = threadIdx.x / 32;
  float s = 0.f;
  if (c < 2 * D)
    for (int k = warp; k < blocks; k += 8) s += part[(int64_t)k * 2 * D + c];
  sums[warp][threadIdx.x & 31] = s;
  __syncthreads();
  if (warp || c >= 2 * D) return;
  s = 0.f;
#pragma unroll
  for (int k = 0; k < 8; ++k) s += sums[k][threadIdx.x];
  W* to = c < D ? dw : db;
  if (to) to[c < D ? c : c - D] = from_float<W>(s);
}

const char* config_fault(const esspt_norm_config* c) {
  if (!c) return "null config";
  if (c->max_rows < 1 || c->max_rows >= ((int64_t)1 << 31)) return "max_rows must be in [1, 2^31 - 1]";
  if (c->width < 1 || c->width > 8192) return "width must be in [1, 8192]";
  if (c->dtype < ESSPT_F32 || c->dtype > ESSPT_F16) return "unknown dtype";
  if (c->weight_dtype != ESSPT_F32 && c->weight_dtype != c->dtype) return "weight_dtype must be fp32 or the rows'";
  if (!(c->eps > 0.f) || !std::isfinite(c->eps)) return "eps must be positive and finite";
  return nullptr;
}

size_t workspace(const esspt_norm_config& c) {
  return 256 + (c.backward ? up256((size_t)kMaxSms * kBlocksPerSm * 2 * c.width * sizeof(float)) : 0);
}

// How a row is spread over threads: the threads of a block and of a row, and N.
struct Spread {
  int threads, lanes, n;
  bool wide;
};
Spread spread(int vectors, int most) {
  Spread s{256, 32, 1, false};
  if (vectors <= 32) {
    while (s.lanes / 2 >= vectors && s.lanes > 1) s.lanes /= 2;
  } else if (vectors <= 64 && most >= 2) {
    s.n = 2;
  } else {
    s.wide = true;
    s.n = most;
    while (s.n > 1 && (vectors + s.n / 2 - 1) / (s.n / 2) <= 256) s.n /= 2;
    s.threads = s.lanes = ((vectors + s.n - 1) / s.n + 31) / 32 * 32;
  }
  return s;
}

template <bool BACK, typename T, typename W, int VEC, int N>
cudaError_t launch(const Spread& s, const Norm& a, unsigned blocks, cudaStream_t st) {
  const size_t shared = BACK ? 2 * a.D * sizeof(float) : 0;
  if (s.wide) {
    auto* kernel = BACK ? norm_backward_kernel<T, W, VEC, N, true> : norm_forward_kernel<T, W, VEC, N, true>;
    if (BACK) {
      cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 2 * 8192 * 4);
      if (e != cudaSuccess) return e;
    }
    kernel<<<blocks, s.threads, shared, st>>>(a);
  } else {
    auto* kernel = BACK ? norm_backward_kernel<T, W, VEC, N, false> : norm_forward_kernel<T, W, VEC, N, false>;
    kernel<<<blocks, s.threads, shared, st>>>(a);
  }
  return cudaGetLastError();
}

template <bool BACK, typename T, typename W, int VEC>
cudaError_t launch_by_size(Norm& a, int sms, unsigned* blocks, cudaStream_t st) {
  const Spread s = spread((a.D + VEC - 1) / VEC, VEC == 1 ? 8 : VEC == 4 ? 4 : 2);
  a.lanes = s.lanes;
  const int64_t groups = (a.n + s.threads / s.lanes - 1) / (s.threads / s.lanes);
  *blocks = (unsigned)(BACK && groups > sms * kBlocksPerSm ? sms * kBlocksPerSm : groups);
  switch (s.n) {
    case 1: return launch<BACK, T, W, VEC, 1>(s, a, *blocks, st);
    case 2: return launch<BACK, T, W, VEC, 2>(s, a, *blocks, st);
    case 4:
      if constexpr (VEC <= 4) return launch<BACK, T, W, VEC, 4>(s, a, *blocks, st);
    default:
      if constexpr (VEC == 1) return launch<BACK, T, W, VEC, 8>(s, a, *blocks, st);
  }
  return cudaErrorInvalidConfiguration;
}

template <bool BACK, typename T, typename W>
cudaError_t launch_by_width(Norm& a, int bytes, int sms, unsigned* blocks, cudaStream_t st) {
  if (bytes >= 16) return launch_by_size<BACK, T, W, 16 / sizeof(T)>(a, sms, blocks, st);
  return launch_by_size<BACK, T, W, 1>(a, sms, blocks, st);
}

template <bool BACK>
cudaError_t launch_norm(const esspt_norm_config& c, Norm& a, int bytes, int sms, unsigned* blocks, cudaStream_t st) {
  const bool f32 = c.weight_dtype == ESSPT_F32;
  if (c.dtype == ESSPT_F32) return launch_by_width<BACK, float, float>(a, bytes, sms, blocks, st);
  if (c.dtype == ESSPT_BF16)
    return f32 ? launch_by_width<BACK, __nv_bfloat16, float>(a, bytes, sms, blocks, st)
               : launch_by_width<BACK, __nv_bfloat16, __nv_bfloat16>(a, bytes, sms, blocks, st);
  return f32 ? launch_by_width<BACK, __half, float>(a, bytes, sms, blocks, st)
             : launch_by_width<BACK, __half, __half>(a, bytes, sms, blocks, st);
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
  ESSPT_CUDA(nm->err, launch_norm<false>(c, a, bytes, nm->sms, &blocks, nm->st));
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
  ESSPT_CUDA(nm->err, launch_norm<true>(c, a, bytes, nm->sms, &blocks, nm->st));
  if (!a.want_w) return ESSPT_OK;
  const unsigned columns = (2 * c.width + 31) / 32;
  if (c.weight_dtype == ESSPT_F32)
    norm_weights_kernel<<<columns, 256, 0, nm->st>>>(a.part, (int)blocks, c.width, (float*)d_dweight, (float*)d_dbias);
  else if (c.weight_dtype == ESSPT_BF16)
    norm_weights_kernel<<<columns, 256, 0, nm->st>>>(a.part, (int)blocks, c.width, (__nv_bfloat16*)d_dweight,
                                                     (__nv_bfloat16*)d_dbias);
  else
    norm_weights_kernel<<<columns, 256, 0, nm->st>>>(a.part, (int)blocks, c.width, (__half*)d_dweight, (__half*)d_dbias);
  ESSPT_CUDA(nm->err, cudaGetLastError());
  return ESSPT_OK;
}

const char* esspt_norm_last_error(const esspt_norm* nm) { return nm ? nm->err.text : g_create.text; }

}  // extern "C"
