// Embedding lookup with scaling, and its gradient by sorted tokens: kernels and C-ABI.
#include <cub/device/device_radix_sort.cuh>
#include <cmath>
#include <new>

#include "operator.h"
#include "rows.cuh"

using namespace esspt;

struct esspt_embed {
  esspt_embed_config cfg{};
  cudaStream_t st = nullptr;
  char* base = nullptr;
  int sms = 0;
  Errors err;
};

namespace {

constexpr uint32_t kErrId = 1u;
constexpr int kThreads = 256, kDeep = 4;

thread_local Errors g_create;

struct Lookup {
  const void* w;
  int64_t w_stride;
  const int32_t* ids;
  int64_t n;
  int32_t V, D, per_row;  // per_row: vectors of a row
  float scale;
  void* out;
  uint32_t* status;
};

// A block takes kThreads * kDeep vectors of the result, one behind the other; a thread
// has kDeep loads under way.
template <typename T, int VEC>
__global__ void __launch_bounds__(kThreads) lookup_kernel(Lookup a) {
  const int64_t first = (int64_t)blockIdx.x * (kThreads * kDeep), all = a.n * a.per_row;
  const int64_t row0 = first / a.per_row;
  const uint32_t rest = (uint32_t)(first - row0 * a.per_row);
  const T* w = static_cast<const T*>(a.w);
  T* out = static_cast<T*>(a.out);
  float x[kDeep][VEC];
#pragma unroll
  for (int k = 0; k < kDeep; ++k) {
    const uint32_t at = rest + k * kThreads + threadIdx.x, row = at / (uint32_t)a.per_row, col = at - row * a.per_row;
#pragma unroll
    for (int i = 0; i < VEC; ++i) x[k][i] = 0.f;
    if (first + k * kThreads + threadIdx.x < all) {
      const int32_t id = a.ids[row0 + row];
      if (id >= a.V) atomicOr(a.status, kErrId);
      if ((uint32_t)id < (uint32_t)a.V) load_vec<T, VEC>(w + id * a.w_stride + col * VEC, x[k]);
    }
  }
#pragma unroll
  for (int k = 0; k < kDeep; ++k) {
    const int64_t at = first + k * kThreads + threadIdx.x;
    if (at >= all) break;
#pragma unroll
    for (int i = 0; i < VEC; ++i) x[k][i] *= a.scale;
    store_vec<T, VEC>(out + at * VEC, x[k]);
  }
}

// Padding sorts behind all rows.
__global__ void keys_kernel(const int32_t* ids, int64_t n, int32_t V, uint32_t* key, uint32_t* val, uint32_t* status) {
  const int64_t t = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (t >= n) return;
  const int32_t id = ids[t];
  if (id >= V) atomicOr(status, kErrId);
  key[t] = (uint32_t)id < (uint32_t)V ? id : V;
  val[t] = (uint32_t)t;
}

struct Gradient {
  const void* grad;
  int64_t grad_stride;
  const uint32_t *key, *val;  // sorted
  int64_t n;
  int32_t V, D, per_row;
  float scale;
  int accumulate;
  void* out;
};

__device__ __forceinline__ int64_t lower_bound(const uint32_t* key, int64_t n, uint32_t v) {
  int64_t lo = 0;
  while (n > 0) {
    const int64_t half = n / 2;
    if (key[lo + half] < v) {
      lo += half + 1;
      n -= half + 1;
    } else {
      n = half;
    }
  }
  return lo;
}

// A warp per row of the result.
template <typename T, int VEC>
__global__ void __launch_bounds__(kThreads) gradient_kernel(Gradient a) {
  const int lane = threadIdx.x & 31;
  const int64_t v = (int64_t)blockIdx.x * (kThreads / 32) + threadIdx.x / 32;
  if (v >= a.V) return;
  const int64_t begin = lower_bound(a.key, a.n, (uint32_t)v);
  int64_t end = begin;
  while (end < a.n && a.key[end] == v) ++end;
  if (begin == end && a.accumulate) return;
  const T* grad = static_cast<const T*>(a.grad);
  T* out = static_cast<T*>(a.out) + v * a.D;
  for (int c = lane; c < a.per_row; c += 32) {
    float sum[VEC] = {}, x[VEC];
    for (int64_t i = begin; i < end; ++i) {
      load_vec<T, VEC>(grad + a.val[i] * a.grad_stride + c * VEC, x);
#pragma unroll
      for (int j = 0; j < VEC; ++j) sum[j] += x[j];
    }
    if (a.accumulate) load_vec<T, VEC>(out + c * VEC, x);
#pragma unroll
    for (int j = 0; j < VEC; ++j) sum[j] = a.accumulate ? fmaf(sum[j], a.scale, x[j]) : sum[j] * a.scale;
    store_vec<T, VEC>(out + c * VEC, sum);
  }
}

const char* config_fault(const esspt_embed_config* c) {
  if (!c) return "null config";
  if (c->max_tokens < 1 || c->max_tokens > (1 << 30)) return "max_tokens must be in [1, 2^30]";
  if (c->n_rows < 1 || c->n_rows > (1 << 30)) return "n_rows must be in [1, 2^30]";
  if (c->width < 1 || c->width > 8192) return "width must be in [1, 8192]";
  if (c->dtype < ESSPT_F32 || c->dtype > ESSPT_F16) return "unknown dtype";
  return nullptr;
}

int bits_of(uint32_t most) {
  int b = 1;
  while (b < 32 && (most >> b) != 0) ++b;
  return b;
}

struct Carve {
  size_t status, key[2], val[2], sort, sort_bytes, total;
};

Carve carve(const esspt_embed_config& c) {
  Carve k{};
  size_t o = 0;
  auto take = [&o](size_t bytes) {
    const size_t at = o;
    o += up256(bytes);
    return at;
  };
  k.status = take(sizeof(uint32_t));
  if (c.backward) {
    for (int i = 0; i < 2; ++i) k.key[i] = take(c.max_tokens * 4), k.val[i] = take(c.max_tokens * 4);
    cub::DoubleBuffer<uint32_t> none(nullptr, nullptr);
    cub::DeviceRadixSort::SortPairs(nullptr, k.sort_bytes, none, none, (int)c.max_tokens, 0, bits_of((uint32_t)c.n_rows));
    k.sort = take(k.sort_bytes);
  }
  k.total = o;
  return k;
}

// `f` as a kernel of this type and vector width, with the arguments that call() takes.
template <typename F>
cudaError_t by_type(int dtype, int bytes, F f) {
  if (dtype == ESSPT_F32) {
    if (bytes >= 16) return f((float*)nullptr, std::integral_constant<int, 4>{});
    return f((float*)nullptr, std::integral_constant<int, 1>{});
  }
  if (dtype == ESSPT_BF16) {
    if (bytes >= 16) return f((__nv_bfloat16*)nullptr, std::integral_constant<int, 8>{});
    if (bytes >= 4) return f((__nv_bfloat16*)nullptr, std::integral_constant<int, 2>{});
    return f((__nv_bfloat16*)nullptr, std::integral_constant<int, 1>{});
  }
  if (bytes >= 16) return f((__half*)nullptr, std::integral_constant<int, 8>{});
  if (bytes >= 4) return f((__half*)nullptr, std::integral_constant<int, 2>{});
  return f((__half*)nullptr, std::integral_constant<int, 1>{});
}

}  // namespace

extern "C" {

size_t esspt_embed_workspace_bytes(const esspt_embed_config* cfg) { return config_fault(cfg) ? 0 : carve(*cfg).total; }

esspt_status esspt_embed_create(const esspt_embed_config* cfg, void* d_workspace, size_t bytes, esspt_embed** out) {
  g_create.text[0] = 0;
  if (const char* why = config_fault(cfg)) return g_create.fail(ESSPT_EINVAL, why);
  if (!out || !d_workspace || misaligned(d_workspace, 256)) return g_create.fail(ESSPT_EINVAL, "null or misaligned pointer");
  if (bytes < carve(*cfg).total) return g_create.fail(ESSPT_ENOSPC, "workspace too small");
  int dev = 0, sms = 0;
  ESSPT_CUDA(g_create, cudaGetDevice(&dev));
  ESSPT_CUDA(g_create, cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  ESSPT_CUDA(g_create, cudaMemsetAsync(d_workspace, 0, 256, static_cast<cudaStream_t>(cfg->stream)));
  esspt_embed* em = new (std::nothrow) esspt_embed;
  if (!em) return g_create.fail(ESSPT_ENOSPC, "out of host memory");
  em->cfg = *cfg;
  em->st = static_cast<cudaStream_t>(cfg->stream);
  em->base = static_cast<char*>(d_workspace);
  em->sms = sms;
  *out = em;
  return ESSPT_OK;
}

esspt_status esspt_embed_destroy(esspt_embed* em) {
  if (!em) return ESSPT_OK;
  const cudaError_t e = cudaStreamSynchronize(em->st);
  delete em;
  return e == cudaSuccess ? ESSPT_OK : g_create.cuda(e, "esspt_embed_destroy");
}

esspt_status esspt_embed_lookup(esspt_embed* em, const void* d_w, int64_t w_stride, const int32_t* d_ids, int64_t n,
                                float scale, void* d_out) {
  if (!em) return ESSPT_EINVAL;
  em->err.text[0] = 0;
  const esspt_embed_config& c = em->cfg;
  const size_t size = size_of(c.dtype);
  if (n < 0 || n > c.max_tokens) return em->err.fail(ESSPT_EINVAL, "n must be in [0, max_tokens]");
  if (!std::isfinite(scale)) return em->err.fail(ESSPT_EINVAL, "scale must be finite");
  if (n == 0) return ESSPT_OK;
  if (!d_w || !d_ids || !d_out) return em->err.fail(ESSPT_EINVAL, "null pointer");
  if (w_stride < c.width) return em->err.fail(ESSPT_EINVAL, "a row stride is below the width");
  if (misaligned(d_w, size) || misaligned(d_out, size) || misaligned(d_ids, 4))
    return em->err.fail(ESSPT_EINVAL, "a pointer is not aligned to its type");
  Lookup a{d_w, w_stride, d_ids, n, (int32_t)c.n_rows, c.width, 0, scale, d_out, reinterpret_cast<uint32_t*>(em->base)};
  const int bytes = vector_bytes(c.width, size, (uintptr_t)d_w | (uintptr_t)d_out | (uintptr_t)w_stride * size);
  const cudaError_t launched = by_type(c.dtype, bytes, [&](auto* type, auto vec) {
    using T = std::remove_pointer_t<decltype(type)>;
    a.per_row = c.width / vec;
    const int64_t blocks = (n * a.per_row + kThreads * kDeep - 1) / (kThreads * kDeep);
    lookup_kernel<T, vec><<<(unsigned)blocks, kThreads, 0, em->st>>>(a);
    return cudaGetLastError();
  });
  ESSPT_CUDA(em->err, launched);
  return ESSPT_OK;
}

esspt_status esspt_embed_gradient(esspt_embed* em, const int32_t* d_ids, const void* d_grad, int64_t grad_stride,
                                  int64_t n, float scale, int32_t accumulate, void* d_grad_w) {
  if (!em) return ESSPT_EINVAL;
  em->err.text[0] = 0;
  const esspt_embed_config& c = em->cfg;
  const size_t size = size_of(c.dtype);
  if (!c.backward) return em->err.fail(ESSPT_EINVAL, "the handle was made without backward");
  if (n < 0 || n > c.max_tokens) return em->err.fail(ESSPT_EINVAL, "n must be in [0, max_tokens]");
  if (!std::isfinite(scale)) return em->err.fail(ESSPT_EINVAL, "scale must be finite");
  if (!d_grad_w || (n > 0 && (!d_ids || !d_grad))) return em->err.fail(ESSPT_EINVAL, "null pointer");
  if (n > 0 && grad_stride < c.width) return em->err.fail(ESSPT_EINVAL, "a row stride is below the width");
  if (misaligned(d_grad, size) || misaligned(d_grad_w, size) || misaligned(d_ids, 4))
    return em->err.fail(ESSPT_EINVAL, "a pointer is not aligned to its type");
  if (n == 0) {
    if (!accumulate) ESSPT_CUDA(em->err, cudaMemsetAsync(d_grad_w, 0, (size_t)c.n_rows * c.width * size, em->st));
    return ESSPT_OK;
  }
  const Carve k = carve(c);
  auto at = [&](size_t o) { return reinterpret_cast<uint32_t*>(em->base + o); };
  cub::DoubleBuffer<uint32_t> key(at(k.key[0]), at(k.key[1])), val(at(k.val[0]), at(k.val[1]));
  keys_kernel<<<(unsigned)((n + kThreads - 1) / kThreads), kThreads, 0, em->st>>>(d_ids, n, (int32_t)c.n_rows, key.Current(),
                                                                                  val.Current(), at(k.status));
  ESSPT_CUDA(em->err, cudaGetLastError());
  size_t bytes = k.sort_bytes;
  ESSPT_CUDA(em->err, cub::DeviceRadixSort::SortPairs(em->base + k.sort, bytes, key, val, (int)n, 0,
                                                      bits_of((uint32_t)c.n_rows), em->st));
  Gradient a{d_grad, grad_stride, key.Current(), val.Current(), n, (int32_t)c.n_rows, c.width, 0, scale, accumulate, d_grad_w};
  const int vb = vector_bytes(c.width, size, (uintptr_t)d_grad | (uintptr_t)d_grad_w | (uintptr_t)grad_stride * size);
  const cudaError_t launched = by_type(c.dtype, vb, [&](auto* type, auto vec) {
    using T = std::remove_pointer_t<decltype(type)>;
    a.per_row = c.width / vec;
    gradient_kernel<T, vec><<<(unsigned)((c.n_rows + 7) / 8), kThreads, 0, em->st>>>(a);
    return cudaGetLastError();
  });
  ESSPT_CUDA(em->err, launched);
  return ESSPT_OK;
}

esspt_status esspt_embed_poll(esspt_embed* em) {
  if (!em) return ESSPT_EINVAL;
  em->err.text[0] = 0;
  uint32_t bits = 0;
  ESSPT_CUDA(em->err, cudaMemcpyAsync(&bits, em->base, sizeof(bits), cudaMemcpyDeviceToHost, em->st));
  ESSPT_CUDA(em->err, cudaStreamSynchronize(em->st));
  if (!bits) return ESSPT_OK;
  ESSPT_CUDA(em->err, cudaMemsetAsync(em->base, 0, sizeof(bits), em->st));
  return em->err.fail(ESSPT_EINVAL, "an id is outside the table");
}

const char* esspt_embed_last_error(const esspt_embed* em) { return em ? em->err.text : g_create.text; }

}  // extern "C"
