// AdamW over many tensors at once, moments in 32 or in 8 bits: kernels and C-ABI.
//
// The tensors are cut into tiles of 4096 values, a block takes a tile, a warp a block of 128 values of it at a time,
// four values a thread.
#include <cmath>
#include <cstring>
#include <limits>
#include <new>
#include <vector>

#include "operator.h"
#include "rows.cuh"

using namespace esspt;

namespace {

constexpr int kBlock = 128;     // values with an exponent of their own (8 bits)
constexpr int kTile = 4096;     // values a block takes
constexpr int kThreads = 256;
constexpr int kGroup = 440;     // tensors of a launch: their gradients' addresses are among its parameters
constexpr uint32_t kNoNumber = 255;  // exponent of a block that is NaN

struct Tensor {
  float* p;
  void* copy;
  int64_t count, at;  // at: its place in the flat order
  float decay;
  uint32_t vector;    // whether p and copy are aligned to four values
};

// A tile: values [index * kTile, ...) of a tensor.
struct Tile {
  uint32_t tensor, index;
};

// Steps taken, and b1, b2 to that power.
struct State {
  int64_t steps;
  double b1t, b2t;
  uint32_t done;  // blocks of a step that have ended; 0 between steps
};

struct Moments {
  float *m, *v;             // 32 bits
  uint8_t *mc, *uc, *me, *ue;  // 8 bits: codes and exponents
};

struct Step {
  const Tensor* tensors;
  const Tile* tiles;
  State* state;
  Moments held;
  uint32_t n_tiles, first_tensor;
  int tick;  // the launch that ends a step counts it
  float lr, b1, b2, one_b1, one_b2, eps;
  double b1d, b2d;
  const float *d_lr, *grad_scale;
  uint32_t seed_lo, seed_hi;
  const void* grads[kGroup];
};

__host__ __device__ __forceinline__ uint32_t mix(uint32_t x) {
  x = (x ^ (x >> 16)) * 0x5851F42Du;
  x = (x ^ (x >> 15)) * 0x2545F491u;
  return x ^ (x >> 16);
}
__device__ __forceinline__ uint32_t place_hash(int64_t i, uint32_t key) {
  return mix(((uint32_t)i * 0x9E3779B1u + (uint32_t)(i >> 32) * 0x85EBCA77u) ^ key);
}

// 8-bit magnitudes are fp32's bits without the low 23 - FRACTION ones, above an exponent: a floor of x is a
// shift of its bits, and so is floor(x / d + rho) with rho's bits added below.
template <int FRACTION>
__device__ __forceinline__ uint32_t block_exponent(float largest_of_four) {
  const uint32_t top = __reduce_max_sync(0xffffffffu, __float_as_uint(largest_of_four) & 0x7fffffffu);
  const uint32_t e = (top + ((1u << (23 - FRACTION)) - 1)) >> 23;
  return e < 16 ? 16 : e > kNoNumber ? kNoNumber : e;
}
template <int FRACTION, bool KEEP>  // KEEP: what is below the least code is held as it, not as it or zero
__device__ __forceinline__ uint32_t hold(float x, uint32_t e, uint32_t r) {
  constexpr int kDrop = 23 - FRACTION;
  const uint32_t zero = (e - 15) << 23, least = zero + (1u << kDrop), b = __float_as_uint(x);
  if (b >= least) return (b - zero + (r << (kDrop - 16))) >> kDrop & (16u << FRACTION) - 1;  // (the mask: of NaN alone)
  if (KEEP) return x > 0.f;
  return x >= (float)(65536u - r) * (__uint_as_float(least) * (1.f / 65536.f));
}
template <int FRACTION>
__device__ __forceinline__ float held(uint32_t code, uint32_t e) {
  if (e == kNoNumber) return __uint_as_float(0x7fffffffu);
  return code ? __uint_as_float((code << (23 - FRACTION)) + ((e - 15) << 23)) : 0.f;
}
__device__ __forceinline__ float held_m(uint32_t code, uint32_t e) {
  const float x = held<3>(code & 127u, e);
  return code & 128u ? -x : x;
}
__device__ __forceinline__ uint32_t hold_m(float x, uint32_t e, uint32_t r) {
  const uint32_t code = hold<3, false>(fabsf(x), e, r);
  return code && x < 0.f ? code | 128u : code;
}

// Four values of a block: one behind the other, or 32 apart where they are not aligned.
template <typename T>
__device__ __forceinline__ void get4(const T* from, bool vector, int lane, int64_t left, float (&x)[4]) {
  if (vector) return load_vec<T, 4>(from + lane * 4, x);
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] = lane + 32 * j < left ? to_float(from[lane + 32 * j]) : 0.f;
}
template <typename T>
__device__ __forceinline__ void put4(T* to, bool vector, int lane, int64_t left, const float (&x)[4]) {
  if (vector) return store_vec<T, 4>(to + lane * 4, x);
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (lane + 32 * j < left) to[lane + 32 * j] = from_float<T>(x[j]);
}
__device__ __forceinline__ void get_codes(const uint8_t* from, bool vector, int lane, uint32_t (&c)[4]) {
  const uint32_t w = vector ? reinterpret_cast<const uint32_t*>(from)[lane] : 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) c[j] = vector ? (w >> (8 * j)) & 255u : from[lane + 32 * j];
}
__device__ __forceinline__ void put_codes(uint8_t* to, bool vector, int lane, const uint32_t (&c)[4]) {
  if (vector) {
    reinterpret_cast<uint32_t*>(to)[lane] = c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24;
    return;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) to[lane + 32 * j] = (uint8_t)c[j];
}
__device__ __forceinline__ float largest(const float (&x)[4]) {  // of magnitudes; NaN if one is
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) top = max(top, __float_as_uint(x[j]) & 0x7fffffffu);
  return __uint_as_float(top);
}

template <int BITS, typename H>
__global__ void __launch_bounds__(kThreads) adamw_kernel(__grid_constant__ const Step a) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
  const State s = *a.state;
  const float lr = a.d_lr ? *a.d_lr : a.lr, scale = a.grad_scale ? *a.grad_scale : 1.f;
  const float rate = lr / (float)(1.0 - s.b1t * a.b1d), root = sqrtf((float)(1.0 - s.b2t * a.b2d));
  const uint32_t key = mix(a.seed_lo ^ mix(a.seed_hi ^ mix((uint32_t)(s.steps + 1))));
  for (uint32_t k = blockIdx.x; k < a.n_tiles; k += gridDim.x) {
    const Tile tile = a.tiles[k];
    const Tensor t = a.tensors[tile.tensor];
    const void* grad = a.grads[tile.tensor - a.first_tensor];
    if (!grad) continue;
    const float keep = 1.f - lr * t.decay;
    const bool aligned = t.vector && (uintptr_t)grad % (t.copy ? 8 : 16) == 0;
    for (int b = warp; b < kTile / kBlock; b += kThreads / 32) {
      const int64_t i = (int64_t)tile.index * kTile + b * kBlock, left = t.count - i;
      if (left <= 0) break;
      const int64_t at = t.at + i;
      const bool vector = aligned && left >= kBlock;
      float p[4], g[4], m[4], v[4];
      get4(t.p + i, vector, lane, left, p);
      if (t.copy)
        get4(static_cast<const H*>(grad) + i, vector, lane, left, g);
      else
        get4(static_cast<const float*>(grad) + i, vector, lane, left, g);
      if (BITS == 32) {
        get4(a.held.m + at, vector, lane, left, m);
        get4(a.held.v + at, vector, lane, left, v);
      } else {
        uint32_t mc[4], uc[4];
        get_codes(a.held.mc + at, vector, lane, mc);
        get_codes(a.held.uc + at, vector, lane, uc);
        const uint32_t me = a.held.me[at / kBlock], ue = a.held.ue[at / kBlock];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float u = held<4>(uc[j], ue);
          m[j] = held_m(mc[j], me), v[j] = __fmul_rn(u, u);
        }
      }
      float u[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (!vector && lane + 32 * j >= left) m[j] = v[j] = 0.f;  // between tensors
        const float gs = __fmul_rn(g[j], scale);
        m[j] = __fadd_rn(__fmul_rn(m[j], a.b1), __fmul_rn(gs, a.one_b1));
        v[j] = __fadd_rn(__fmul_rn(v[j], a.b2), __fmul_rn(__fmul_rn(gs, gs), a.one_b2));
        u[j] = __fsqrt_rn(v[j]);
        p[j] = p[j] * keep - rate * m[j] / (u[j] / root + a.eps);
      }
      put4(t.p + i, vector, lane, left, p);
      if (t.copy) put4(static_cast<H*>(t.copy) + i, vector, lane, left, p);
      if (BITS == 32) {
        put4(a.held.m + at, vector, lane, left, m);
        put4(a.held.v + at, vector, lane, left, v);
      } else {
        const uint32_t me = block_exponent<3>(largest(m)), ue = block_exponent<4>(largest(u));
        uint32_t mc[4], uc[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t h = place_hash(at + (vector ? lane * 4 + j : lane + 32 * j), key);
          mc[j] = hold_m(m[j], me, h >> 16), uc[j] = hold<4, true>(u[j], ue, h & 0xffffu);
        }
        put_codes(a.held.mc + at, vector, lane, mc);
        put_codes(a.held.uc + at, vector, lane, uc);
        if (lane == 0) a.held.me[at / kBlock] = (uint8_t)me, a.held.ue[at / kBlock] = (uint8_t)ue;
      }
    }
  }
  if (!a.tick) return;
  // Every block has read the state before it counts itself here; the last one counts the step.
  __syncthreads();
  if (threadIdx.x != 0) return;
  __threadfence();
  if (atomicAdd(&a.state->done, 1u) == gridDim.x - 1)
    *a.state = State{s.steps + 1, s.b1t * a.b1d, s.b2t * a.b2d, 0u};
}

// Eight-bit moments as bf16, which holds all of a code's bits; and moments taken from outside (8 bits: to the
// nearest code).
__global__ void __launch_bounds__(kThreads) moments_kernel(Moments held_at, int64_t blocks, __nv_bfloat16* m, __nv_bfloat16* u) {
  const int lane = threadIdx.x & 31;
  const int64_t b = (int64_t)blockIdx.x * (kThreads / 32) + threadIdx.x / 32;
  if (b >= blocks) return;
  const int64_t at = b * kBlock;
  uint32_t mc[4], uc[4];
  float x[4], y[4];
  get_codes(held_at.mc + at, true, lane, mc);
  get_codes(held_at.uc + at, true, lane, uc);
  const uint32_t me = held_at.me[b], ue = held_at.ue[b];
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] = held_m(mc[j], me), y[j] = held<4>(uc[j], ue);
  put4(m + at, true, lane, kBlock, x);
  put4(u + at, true, lane, kBlock, y);
}
template <int BITS>
__global__ void __launch_bounds__(kThreads) load_kernel(const Tensor* tensors, const Tile* tiles, Moments to, const void* m, const void* second) {
  const int lane = threadIdx.x & 31;
  const Tile tile = tiles[blockIdx.x];
  const Tensor t = tensors[tile.tensor];
  for (int b = threadIdx.x / 32; b < kTile / kBlock; b += kThreads / 32) {
    const int64_t i = (int64_t)tile.index * kTile + b * kBlock, left = t.count - i, at = t.at + i;
    if (left <= 0) break;
    float x[4], y[4];
    if (BITS == 32) {
      get4(static_cast<const float*>(m) + at, false, lane, left, x);
      get4(static_cast<const float*>(second) + at, false, lane, left, y);
    } else {
      get4(static_cast<const __nv_bfloat16*>(m) + at, false, lane, left, x);
      get4(static_cast<const __nv_bfloat16*>(second) + at, false, lane, left, y);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = y[j] < 0.f ? 0.f : y[j];
    if (BITS == 32) {
      put4(to.m + at, false, lane, left, x);
      put4(to.v + at, false, lane, left, y);
      continue;
    }
    const uint32_t me = block_exponent<3>(largest(x)), ue = block_exponent<4>(largest(y));
    uint32_t mc[4], uc[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) mc[j] = hold_m(x[j], me, 0x8000u), uc[j] = hold<4, true>(y[j], ue, 0x8000u);
    put_codes(to.mc + at, false, lane, mc);
    put_codes(to.uc + at, false, lane, uc);
    if (lane == 0) to.me[at / kBlock] = (uint8_t)me, to.ue[at / kBlock] = (uint8_t)ue;
  }
}
__global__ void state_kernel(State* to, State s) { *to = s; }

thread_local Errors g_create;

// The values' and tiles' numbers of a list; `why` says what is wrong with it.
struct Sizes {
  int64_t values = 0, tiles = 0;
  const char* why = nullptr;
};

Sizes measure(const esspt_adamw_config* c, const esspt_adamw_tensor* t) {
  Sizes z;
  auto no = [&z](const char* why) {
    z.why = why;
    return z;
  };
  if (!c || !t) return no("null config or list");
  if (c->n_tensors < 1 || c->n_tensors > (1 << 20)) return no("n_tensors must be in [1, 2^20]");
  if (c->state_bits != 32 && c->state_bits != 8) return no("state_bits must be 32 or 8");
  if (c->copy_dtype != ESSPT_BF16 && c->copy_dtype != ESSPT_F16) return no("copy_dtype must be bf16 or fp16");
  if (c->reserved != 0) return no("reserved must be 0");
  if (!(c->beta1 >= 0.0 && c->beta1 < 1.0 && c->beta2 >= 0.0 && c->beta2 < 1.0)) return no("betas must be in [0, 1)");
  if (!((float)c->eps > 0.f) || !std::isfinite((float)c->eps)) return no("eps must be positive and finite in fp32");
  for (int k = 0; k < c->n_tensors; ++k) {
    if (t[k].count < 0 || t[k].count > (int64_t)1 << 40) return no("a count must be in [0, 2^40]");
    if (!(t[k].weight_decay >= 0.f) || !std::isfinite(t[k].weight_decay))
      return no("a weight_decay must be finite and not negative");
    z.values += (t[k].count + kBlock - 1) / kBlock * kBlock;
    z.tiles += (t[k].count + kTile - 1) / kTile;
  }
  if (z.tiles >= (int64_t)1 << 31) return no("the tensors must have fewer than 2^43 values");
  return z;
}

struct Carve {
  size_t first, second, exp_first, exp_second, state, tensors, tiles, total;
};

Carve carve(const esspt_adamw_config& c, const Sizes& z) {
  Carve k{};
  size_t o = 0;
  auto take = [&o](size_t bytes, bool whole = true) {
    const size_t at = o;
    o += whole ? up256(bytes) : bytes;
    return at;
  };
  const size_t size = c.state_bits / 8;
  k.first = take(z.values * size, false);  // (v directly behind m)
  k.second = take(z.values * size);
  if (c.state_bits == 8) k.exp_first = take(z.values / kBlock), k.exp_second = take(z.values / kBlock);
  k.state = take(sizeof(State));
  k.tensors = take(c.n_tensors * sizeof(Tensor));
  k.tiles = take(z.tiles * sizeof(Tile));
  k.total = o;
  return k;
}

}  // namespace

struct esspt_adamw {
  esspt_adamw_config cfg{};
  cudaStream_t st = nullptr;
  char* base = nullptr;
  Carve k{};
  int64_t values = 0;
  int sms = 0;
  std::vector<uint32_t> first_tile;  // of every kGroup-th tensor, and their number
  std::vector<size_t> sizes;         // of a tensor's gradients, or 0 where it has no values
  Errors err;

  Moments moments() const {
    if (cfg.state_bits == 32)
      return Moments{reinterpret_cast<float*>(base + k.first), reinterpret_cast<float*>(base + k.second), nullptr, nullptr, nullptr,
                     nullptr};
    auto at = [this](size_t o) { return reinterpret_cast<uint8_t*>(base + o); };
    return Moments{nullptr, nullptr, at(k.first), at(k.second), at(k.exp_first), at(k.exp_second)};
  }
};

namespace {

esspt_status fill(esspt_adamw* aw, const esspt_adamw_tensor* tensors) {
  const esspt_adamw_config& c = aw->cfg;
  std::vector<Tensor> recs;
  std::vector<Tile> tiles;
  int64_t at = 0;
  for (int k = 0; k < c.n_tensors; ++k) {
    const esspt_adamw_tensor& t = tensors[k];
    const bool vector = !misaligned(t.d_param, 16) && !misaligned(t.d_copy, 8);
    recs.push_back(Tensor{t.d_param, t.d_copy, t.count, at, t.weight_decay, vector});
    aw->sizes.push_back(t.count == 0 ? 0 : t.d_copy ? 2 : 4);
    if (k % kGroup == 0) aw->first_tile.push_back((uint32_t)tiles.size());
    for (int64_t i = 0; i * kTile < t.count; ++i) tiles.push_back(Tile{(uint32_t)k, (uint32_t)i});
    at += (t.count + kBlock - 1) / kBlock * kBlock;
  }
  aw->first_tile.push_back((uint32_t)tiles.size());
  ESSPT_CUDA(g_create, cudaMemsetAsync(aw->base, 0, aw->k.state, aw->st));
  ESSPT_CUDA(g_create, cudaMemcpyAsync(aw->base + aw->k.tensors, recs.data(), recs.size() * sizeof(Tensor), cudaMemcpyHostToDevice, aw->st));
  ESSPT_CUDA(g_create, cudaMemcpyAsync(aw->base + aw->k.tiles, tiles.data(), tiles.size() * sizeof(Tile), cudaMemcpyHostToDevice, aw->st));
  state_kernel<<<1, 1, 0, aw->st>>>(reinterpret_cast<State*>(aw->base + aw->k.state), State{0, 1.0, 1.0, 0u});
  ESSPT_CUDA(g_create, cudaGetLastError());
  ESSPT_CUDA(g_create, cudaStreamSynchronize(aw->st));
  return ESSPT_OK;
}

template <int BITS>
void launch(const esspt_adamw_config& c, unsigned blocks, cudaStream_t st, const Step& a) {
  if (c.copy_dtype == ESSPT_BF16)
    adamw_kernel<BITS, __nv_bfloat16><<<blocks, kThreads, 0, st>>>(a);
  else
    adamw_kernel<BITS, __half><<<blocks, kThreads, 0, st>>>(a);
}

unsigned warps_for(int64_t blocks) { return (unsigned)((blocks + kThreads / 32 - 1) / (kThreads / 32)); }

}  // namespace

extern "C" {

int64_t esspt_adamw_moment_values(const esspt_adamw_config* cfg, const esspt_adamw_tensor* tensors) {
  const Sizes z = measure(cfg, tensors);
  return z.why ? 0 : z.values;
}

size_t esspt_adamw_workspace_bytes(const esspt_adamw_config* cfg, const esspt_adamw_tensor* tensors) {
  const Sizes z = measure(cfg, tensors);
  return z.why ? 0 : carve(*cfg, z).total;
}

esspt_status esspt_adamw_create(const esspt_adamw_config* cfg, const esspt_adamw_tensor* tensors, void* d_workspace,
                                size_t bytes, esspt_adamw** out) {
  g_create.text[0] = 0;
  const Sizes z = measure(cfg, tensors);
  if (z.why) return g_create.fail(ESSPT_EINVAL, z.why);
  for (int k = 0; k < cfg->n_tensors; ++k) {
    if (tensors[k].count > 0 && !tensors[k].d_param) return g_create.fail(ESSPT_EINVAL, "null pointer");
    if (misaligned(tensors[k].d_param, 4) || misaligned(tensors[k].d_copy, 2))
      return g_create.fail(ESSPT_EINVAL, "a pointer is not aligned to its type");
  }
  if (!out || !d_workspace || misaligned(d_workspace, 256)) return g_create.fail(ESSPT_EINVAL, "null or misaligned pointer");
  if (bytes < carve(*cfg, z).total) return g_create.fail(ESSPT_ENOSPC, "workspace too small");
  int dev = 0, sms = 0;
  ESSPT_CUDA(g_create, cudaGetDevice(&dev));
  ESSPT_CUDA(g_create, cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  esspt_adamw* aw = new (std::nothrow) esspt_adamw;
  if (!aw) return g_create.fail(ESSPT_ENOSPC, "out of host memory");
  aw->cfg = *cfg;
  aw->st = static_cast<cudaStream_t>(cfg->stream);
  aw->base = static_cast<char*>(d_workspace);
  aw->k = carve(*cfg, z);
  aw->values = z.values;
  aw->sms = sms;
  esspt_status st;
  try {
    st = fill(aw, tensors);
  } catch (const std::bad_alloc&) {
    st = g_create.fail(ESSPT_ENOSPC, "out of host memory");
  }
  if (st != ESSPT_OK) {
    delete aw;
    return st;
  }
  *out = aw;
  return ESSPT_OK;
}

esspt_status esspt_adamw_destroy(esspt_adamw* aw) {
  if (!aw) return ESSPT_OK;
  const cudaError_t e = cudaStreamSynchronize(aw->st);
  delete aw;
  return e == cudaSuccess ? ESSPT_OK : g_create.cuda(e, "esspt_adamw_destroy");
}

esspt_status esspt_adamw_step(esspt_adamw* aw, const void* const* h_grads, float lr, const float* d_lr,
                              const float* d_grad_scale) {
  if (!aw) return ESSPT_EINVAL;
  aw->err.text[0] = 0;
  const esspt_adamw_config& c = aw->cfg;
  if (!h_grads) return aw->err.fail(ESSPT_EINVAL, "null pointer");
  if (!d_lr && !std::isfinite(lr)) return aw->err.fail(ESSPT_EINVAL, "lr must be finite");
  if (misaligned(d_lr, 4) || misaligned(d_grad_scale, 4)) return aw->err.fail(ESSPT_EINVAL, "a pointer is not aligned to its type");
  for (int k = 0; k < c.n_tensors; ++k)
    if (aw->sizes[k] && misaligned(h_grads[k], aw->sizes[k]))
      return aw->err.fail(ESSPT_EINVAL, "a pointer is not aligned to its type");
  Step a{};
  a.tensors = reinterpret_cast<const Tensor*>(aw->base + aw->k.tensors);
  a.state = reinterpret_cast<State*>(aw->base + aw->k.state);
  a.held = aw->moments();
  a.lr = lr, a.b1 = (float)c.beta1, a.b2 = (float)c.beta2;
  a.one_b1 = (float)(1.0 - c.beta1), a.one_b2 = (float)(1.0 - c.beta2), a.eps = (float)c.eps;
  a.b1d = c.beta1, a.b2d = c.beta2;
  a.d_lr = d_lr, a.grad_scale = d_grad_scale;
  a.seed_lo = (uint32_t)c.seed, a.seed_hi = (uint32_t)(c.seed >> 32);
  for (int k = 0, group = 0; k < c.n_tensors; k += kGroup, ++group) {
    const int here = c.n_tensors - k < kGroup ? c.n_tensors - k : kGroup;
    a.first_tensor = (uint32_t)k;
    a.tiles = reinterpret_cast<const Tile*>(aw->base + aw->k.tiles) + aw->first_tile[group];
    a.n_tiles = aw->first_tile[group + 1] - aw->first_tile[group];
    a.tick = k + here == c.n_tensors;
    memcpy(a.grads, h_grads + k, here * sizeof(void*));
    if (a.n_tiles == 0 && !a.tick) continue;
    const unsigned blocks = a.n_tiles ? a.n_tiles : 1;
    if (c.state_bits == 32)
      launch<32>(c, blocks, aw->st, a);
    else
      launch<8>(c, blocks, aw->st, a);
    ESSPT_CUDA(aw->err, cudaGetLastError());
  }
  return ESSPT_OK;
}

esspt_status esspt_adamw_moments(esspt_adamw* aw, void* d_m, void* d_second) {
  if (!aw) return ESSPT_EINVAL;
  aw->err.text[0] = 0;
  if (aw->values == 0) return ESSPT_OK;
  if (!d_m || !d_second) return aw->err.fail(ESSPT_EINVAL, "null pointer");
  if (misaligned(d_m, 16) || misaligned(d_second, 16)) return aw->err.fail(ESSPT_EINVAL, "a pointer is not aligned to 16 bytes");
  if (aw->cfg.state_bits == 32) {
    const size_t bytes = aw->values * sizeof(float);
    ESSPT_CUDA(aw->err, cudaMemcpyAsync(d_m, aw->base + aw->k.first, bytes, cudaMemcpyDeviceToDevice, aw->st));
    ESSPT_CUDA(aw->err, cudaMemcpyAsync(d_second, aw->base + aw->k.second, bytes, cudaMemcpyDeviceToDevice, aw->st));
    return ESSPT_OK;
  }
  const int64_t blocks = aw->values / kBlock;
  moments_kernel<<<warps_for(blocks), kThreads, 0, aw->st>>>(aw->moments(), blocks, static_cast<__nv_bfloat16*>(d_m),
                                                             static_cast<__nv_bfloat16*>(d_second));
  ESSPT_CUDA(aw->err, cudaGetLastError());
  return ESSPT_OK;
}

esspt_status esspt_adamw_load(esspt_adamw* aw, const void* d_m, const void* d_second, int64_t steps) {
  if (!aw) return ESSPT_EINVAL;
  aw->err.text[0] = 0;
  if (steps < 0) return aw->err.fail(ESSPT_EINVAL, "steps must not be negative");
  if (aw->values > 0 && (!d_m || !d_second)) return aw->err.fail(ESSPT_EINVAL, "null pointer");
  const esspt_adamw_config& c = aw->cfg;
  const size_t size = c.state_bits == 32 ? 4 : 2;
  if (misaligned(d_m, size) || misaligned(d_second, size)) return aw->err.fail(ESSPT_EINVAL, "a pointer is not aligned to its type");
  if (const uint32_t tiles = aw->first_tile.back()) {
    const Tensor* rec = reinterpret_cast<const Tensor*>(aw->base + aw->k.tensors);
    const Tile* tile = reinterpret_cast<const Tile*>(aw->base + aw->k.tiles);
    if (c.state_bits == 32)
      load_kernel<32><<<tiles, kThreads, 0, aw->st>>>(rec, tile, aw->moments(), d_m, d_second);
    else
      load_kernel<8><<<tiles, kThreads, 0, aw->st>>>(rec, tile, aw->moments(), d_m, d_second);
  }
  ESSPT_CUDA(aw->err, cudaGetLastError());
  state_kernel<<<1, 1, 0, aw->st>>>(reinterpret_cast<State*>(aw->base + aw->k.state),
                                    State{steps, std::pow(c.beta1, (double)steps), std::pow(c.beta2, (double)steps), 0u});
  ESSPT_CUDA(aw->err, cudaGetLastError());
  return ESSPT_OK;
}

esspt_status esspt_adamw_steps(esspt_adamw* aw, int64_t* steps) {
  if (!aw) return ESSPT_EINVAL;
  aw->err.text[0] = 0;
  if (!steps) return aw->err.fail(ESSPT_EINVAL, "null pointer");
  ESSPT_CUDA(aw->err, cudaMemcpyAsync(steps, aw->base + aw->k.state, sizeof(*steps), cudaMemcpyDeviceToHost, aw->st));
  ESSPT_CUDA(aw->err, cudaStreamSynchronize(aw->st));
  return ESSPT_OK;
}

const char* esspt_adamw_last_error(const esspt_adamw* aw) { return aw ? aw->err.text : g_create.text; }

}  // extern "C"
