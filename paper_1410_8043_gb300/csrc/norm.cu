// Layer norm, forward and backward: kernels and C-ABI.
//
// A group of lanes (a part of a warp, a warp, or for wide rows a block) holds a row in registers, N vectors of
// VEC values a lane, so that a row is read once.  Groups stay and go through rows: their weights stay in registers, and the
// next row's loads are under way while this one is summed.  All arithmetic is fp32.
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

constexpr int kMaxSms = 256;  // what the workspace is sized for
// Threads of a wide row's block, at most: 256 with up to eight values each, 512 with more.
constexpr int most_wide(int values) { return values <= 8 ? 256 : 512; }
constexpr int kMostWarps = 16;

// Threads that an SM holds: with eight values each 64 registers do forward, 80 backward; with more 128.
constexpr int resident(bool back, int values) { return values > 8 ? 512 : back ? 768 : 1024; }

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

template <typename T, int VEC, int N>
struct Row {
  struct alignas(VEC * sizeof(T)) Pack {
    T v[VEC];
  };
  Pack p[N];

  __device__ __forceinline__ void load(const T* row, int D, int lane, int lanes, bool live) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = (lane + i * lanes) * VEC;
      if (live && c < D) {
        p[i] = *reinterpret_cast<const Pack*>(row + c);
      } else {
#pragma unroll
        for (int j = 0; j < VEC; ++j) p[i].v[j] = from_float<T>(0.f);
      }
    }
  }
  __device__ __forceinline__ void get(float (&x)[N][VEC]) const {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int j = 0; j < VEC; ++j) x[i][j] = to_float(p[i].v[j]);
  }
};

// Weights by single values: they may stand anywhere, and are read once.
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

// The sum over the lanes of a warp that hold one row.
__device__ __forceinline__ float lanes_sum(float v, int lanes) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) {
    const float other = __shfl_xor_sync(0xffffffffu, v, off);
    if (off < lanes) v += other;
  }
  return v;
}


template <typename T, typename W, int VEC, int N, bool WIDE>
__global__ void __launch_bounds__(WIDE ? most_wide(VEC * N) : 256, resident(false, VEC * N) / (WIDE ? most_wide(VEC * N) : 256)) norm_forward_kernel(Norm a) {
  __shared__ float2 shared[2][kMostWarps];
  const int lanes = WIDE ? blockDim.x : a.lanes, lane = threadIdx.x & (WIDE ? ~0 : lanes - 1);
  const int groups = blockDim.x / lanes, group = WIDE ? 0 : threadIdx.x / lanes;
  const T* rows = static_cast<const T*>(a.x);
  Row<T, VEC, N> next;
  int64_t t = (int64_t)blockIdx.x * groups + group;
  const int64_t step = (int64_t)gridDim.x * groups;
  next.load(rows + t * a.x_stride, a.D, lane, lanes, t < a.n);
  float w[N][VEC], b[N][VEC];
  load_weights<W, VEC, N>(a.weight, 1.f, a.D, lane, lanes, w);
  load_weights<W, VEC, N>(a.bias, 0.f, a.D, lane, lanes, b);
  auto count = [&](int warp) {  // values of a warp
    int c = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int left = a.D - (warp * 32 + i * lanes) * VEC;
      c += left < 0 ? 0 : left < 32 * VEC ? left : 32 * VEC;
    }
    return (float)c;
  };
  const int warp = threadIdx.x / 32, other = threadIdx.x & 31;
  const float inv_own = WIDE ? 1.f / fmaxf(count(warp), 1.f) : a.inv_D, count_other = WIDE && other < blockDim.x / 32 ? count(other) : 0.f;
  for (int64_t t0 = (int64_t)blockIdx.x * groups, turn = 0; t0 < a.n; t0 += step, t += step, turn ^= 1) {
    float x[N][VEC];
    next.get(x);
    next.load(rows + (t + step) * a.x_stride, a.D, lane, lanes, t + step < a.n);
    // Mean and squares of differences to it, of the lanes of a warp.
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int j = 0; j < VEC; ++j) s += x[i][j];
    s = lanes_sum(s, WIDE ? 32 : lanes);
    float mean = s * inv_own, m2 = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const float d = x[i][j] - mean;
        if ((lane + i * lanes) * VEC + j < a.D) m2 += d * d;
      }
    m2 = lanes_sum(m2, WIDE ? 32 : lanes);
    if (WIDE) {
      // Of the warps: squares about the row's mean are those about a warp's and their distance's.
      if (other == 0) shared[turn][warp] = make_float2(mean, m2);
      __syncthreads();  // (the next row's go to the other half)
      const float2 v = count_other > 0.f ? shared[turn][other] : make_float2(0.f, 0.f);
      mean = lanes_sum(count_other * v.x, 32) * a.inv_D;
      m2 = lanes_sum(v.y + count_other * (v.x - mean) * (v.x - mean), 32);
    }
    const float rstd = 1.f / sqrtf(m2 * a.inv_D + a.eps);
    if (t >= a.n) continue;
    T* y = static_cast<T*>(a.y) + t * a.D;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = (lane + i * lanes) * VEC;
#pragma unroll
      for (int j = 0; j < VEC; ++j) x[i][j] = (x[i][j] - mean) * rstd * w[i][j] + b[i][j];
      if (c < a.D) store_vec<T, VEC>(y + c, x[i]);
    }
    if (lane == 0 && a.mean) a.mean[t] = mean, a.rstd[t] = rstd;
  }
}

// A thread's columns are the same in all rows, and it keeps their sums for dw and db; at the end those of a
// block are added, the groups of a warp by shuffles, then warp behind warp.
template <typename T, typename W, int VEC, int N, bool WIDE>
__global__ void __launch_bounds__(WIDE ? most_wide(VEC * N) : 256, resident(true, VEC * N) / (WIDE ? most_wide(VEC * N) : 256)) norm_backward_kernel(Norm a) {
  extern __shared__ float sums[];  // [2][D]
  __shared__ float2 shared[2][kMostWarps];
  const int lanes = WIDE ? blockDim.x : a.lanes, lane = threadIdx.x & (WIDE ? ~0 : lanes - 1);
  const int groups = blockDim.x / lanes, group = WIDE ? 0 : threadIdx.x / lanes;
  Row<T, VEC, N> next_x, next_dy;
  int64_t t = (int64_t)blockIdx.x * groups + group;
  const int64_t step = (int64_t)gridDim.x * groups;
  float next_mean = 0.f, next_rstd = 0.f;
  auto load = [&](int64_t at) {
    const bool live = at < a.n;
    next_x.load(static_cast<const T*>(a.x) + at * a.x_stride, a.D, lane, lanes, live);
    next_dy.load(static_cast<const T*>(a.dy) + at * a.dy_stride, a.D, lane, lanes, live);
    next_mean = live ? a.mean[at] : 0.f, next_rstd = live ? a.rstd[at] : 0.f;
  };
  load(t);
  float w[N][VEC], dw[N][VEC] = {}, db[N][VEC] = {};
  load_weights<W, VEC, N>(a.weight, 1.f, a.D, lane, lanes, w);
  for (int64_t t0 = (int64_t)blockIdx.x * groups, turn = 0; t0 < a.n; t0 += step, t += step, turn ^= 1) {
    float x[N][VEC], dy[N][VEC];
    next_x.get(x), next_dy.get(dy);
    const float mean = next_mean, rstd = next_rstd;
    load(t + step);
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
    if (!a.y) continue;
    s = make_float2(lanes_sum(s.x, WIDE ? 32 : lanes), lanes_sum(s.y, WIDE ? 32 : lanes));
    if (WIDE) {
      if ((threadIdx.x & 31) == 0) shared[turn][threadIdx.x / 32] = s;
      __syncthreads();  // (the next row's go to the other half)
      s = make_float2(0.f, 0.f);
      for (int k = 0; k < (int)blockDim.x / 32; ++k) s.x += shared[turn][k].x, s.y += shared[turn][k].y;
    }
    s.x *= a.inv_D, s.y *= a.inv_D;
    if (t >= a.n) continue;
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
  if (!WIDE) {
    for (int off = 16; off >= lanes; off >>= 1)
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          dw[i][j] += __shfl_xor_sync(0xffffffffu, dw[i][j], off);
          db[i][j] += __shfl_xor_sync(0xffffffffu, db[i][j], off);
        }
  }
  float* part = a.part + (int64_t)blockIdx.x * 2 * a.D;
  const int warp = WIDE ? 0 : threadIdx.x / 32, warps = WIDE ? 1 : blockDim.x / 32;
  for (int k = 0; k < warps; ++k) {
    if (warp == k && (WIDE || (threadIdx.x & 31) < lanes)) {
      float* to = k == warps - 1 ? part : sums;
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          const int c = (lane + i * lanes) * VEC + j;
          if (c < a.D) {
            to[c] = (k ? sums[c] : 0.f) + dw[i][j];
            to[a.D + c] = (k ? sums[a.D + c] : 0.f) + db[i][j];
          }
        }
    }
    if (k < warps - 1) __syncthreads();
  }
}

// dw and db from the blocks' sums: 32 columns to a block, whose warps take every 16th block's.
constexpr int kWeightWarps = 16;
template <typename W>
__global__ void __launch_bounds__(32 * kWeightWarps) norm_weights_kernel(const float* part, int blocks, int D, W* dw, W* db) {
  __shared__ float sums[kWeightWarps][33];
  const int c = blockIdx.x * 32 + (threadIdx.x & 31), warp = threadIdx.x / 32;
  float s = 0.f;
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
  if (c->width < 1 || c->width > 8192) return "width must be in [1, 8192]";
  if (c->dtype < ESSPT_F32 || c->dtype > ESSPT_F16) return "unknown dtype";
  if (c->weight_dtype != ESSPT_F32 && c->weight_dtype != c->dtype) return "weight_dtype must be fp32 or the rows'";
  if (!(c->eps > 0.f) || !std::isfinite(c->eps)) return "eps must be positive and finite";
  return nullptr;
}

// How rows of D values are spread over threads: those of a block and of a row, vectors of a thread (N), and
// blocks of an SM.
struct Spread {
  int threads, lanes, n, resident;
  bool wide;
};
Spread spread(int D, int vec, bool back) {
  const int vectors = (D + vec - 1) / vec;
  Spread s{256, 32, 1, 0, false};
  if (vectors <= 32) {
    while (s.lanes / 2 >= vectors && s.lanes > 1) s.lanes /= 2;
  } else if (vectors <= 64) {
    s.n = 2;
  } else {
    s.wide = true;
    while ((vectors + s.n - 1) / s.n > most_wide(s.n * vec)) s.n *= 2;
    s.threads = s.lanes = ((vectors + s.n - 1) / s.n + 31) / 32 * 32;
  }
  s.resident = resident(back, s.n * vec) / s.threads;
  return s;
}

size_t workspace(const esspt_norm_config& c) {
  if (!c.backward) return 256;
  const Spread a = spread(c.width, 16 / (int)size_of(c.dtype), true), b = spread(c.width, 1, true);
  const size_t blocks = (size_t)kMaxSms * (a.resident > b.resident ? a.resident : b.resident);
  return 256 + up256(blocks * 2 * c.width * sizeof(float));
}

template <bool BACK, typename T, typename W, int VEC, int N, bool WIDE>
cudaError_t launch(const Spread& s, const Norm& a, unsigned blocks, cudaStream_t st) {
  if (!BACK) {
    norm_forward_kernel<T, W, VEC, N, WIDE><<<blocks, s.threads, 0, st>>>(a);
    return cudaGetLastError();
  }
  auto* kernel = norm_backward_kernel<T, W, VEC, N, WIDE>;
  kernel<<<blocks, s.threads, WIDE ? 0 : 2 * a.D * sizeof(float), st>>>(a);  // (rows of one warp: at most 4 KB)
  return cudaGetLastError();
}

template <bool BACK, typename T, typename W, int VEC>
cudaError_t launch_by_size(Norm& a, int sms, unsigned* blocks, cudaStream_t st) {
  const Spread s = spread(a.D, VEC, BACK);
  a.lanes = s.lanes;
  const int64_t groups = (a.n + s.threads / s.lanes - 1) / (s.threads / s.lanes);
  *blocks = (unsigned)(groups > sms * s.resident ? sms * s.resident : groups);
  if (!s.wide)
    return s.n == 1 ? launch<BACK, T, W, VEC, 1, false>(s, a, *blocks, st) : launch<BACK, T, W, VEC, 2, false>(s, a, *blocks, st);
  switch (s.n) {
    case 1: return launch<BACK, T, W, VEC, 1, true>(s, a, *blocks, st);
    case 2: return launch<BACK, T, W, VEC, 2, true>(s, a, *blocks, st);
    case 4:
      if constexpr (VEC <= 4) return launch<BACK, T, W, VEC, 4, true>(s, a, *blocks, st);
    case 8:
      if constexpr (VEC == 1) return launch<BACK, T, W, VEC, 8, true>(s, a, *blocks, st);
    case 16:
      if constexpr (VEC == 1) return launch<BACK, T, W, VEC, 16, true>(s, a, *blocks, st);
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
    norm_weights_kernel<<<columns, 32 * kWeightWarps, 0, nm->st>>>(a.part, (int)blocks, c.width, (float*)d_dweight, (float*)d_dbias);
  else if (c.weight_dtype == ESSPT_BF16)
    norm_weights_kernel<<<columns, 32 * kWeightWarps, 0, nm->st>>>(a.part, (int)blocks, c.width, (__nv_bfloat16*)d_dweight,
                                                     (__nv_bfloat16*)d_dbias);
  else
    norm_weights_kernel<<<columns, 32 * kWeightWarps, 0, nm->st>>>(a.part, (int)blocks, c.width, (__half*)d_dweight, (__half*)d_dbias);
  ESSPT_CUDA(nm->err, cudaGetLastError());
  return ESSPT_OK;
}

const char* esspt_norm_last_error(const esspt_norm* nm) { return nm ? nm->err.text : g_create.text; }

}  // extern "C"
