// AdamW over many tensors at once, moments in 32 or in 8 bits: kernels and C-ABI.
//
// The tensors are cut into tiles of 4096 values.  Blocks stay and go through tiles, the next one's record under way;
// a warp takes 512 values of a tile, four blocks of 128, four values a thread of each.  With 32-bit moments all loads of a
// tile come first, and memory is the bound: 31 million values with 16-bit copies move 28 bytes each at 6.4 TB/s.  With 8 bits
// the next tile is copied to shared memory meanwhile, and arithmetic is the bound, some 99 instructions a value: 192 million
// values take 621 us at 16 bytes each, 4.9 TB/s.
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstring>
#include <new>
#include <type_traits>
#include <utility>
#include <vector>

#include "operator.h"
#include "ptx.cuh"
#include "rows.cuh"

using namespace esspt;

namespace {

constexpr int kBlock = 128;     // values with an exponent of their own (8 bits)
constexpr int kTile = 4096;     // values a block takes
constexpr int kThreads = 256;
constexpr int kMine = kTile / (kThreads / 32), kBatch = kMine / kBlock;  // values and blocks of a warp
// Blocks of an SM: 128 registers for the loads of 32-bit moments (31 million values with 16-bit copies: 137 us, three blocks
// 145); for 8-bit ones 180 KB of stages.
constexpr int kResident = 2;
constexpr int kGroup = 440;     // tensors of a launch: their gradients' addresses are among its parameters
constexpr uint32_t kNoNumber = 255;  // exponent of a block that is NaN

// A tile: up to kTile values of a tensor, from `first` on.
struct alignas(16) Tile {
  float* p;           // the tile's first value
  void* copy;
  int64_t first, at;  // at: its place in the flat order
  uint32_t tensor;
  int32_t count;
  float decay;
  uint32_t vector;    // whether p and copy are aligned to four values
};

// Steps taken, and b1, b2 to that power.
struct State {
  int64_t steps;
  double b1t, b2t;
  uint32_t done;  // blocks of a step that have ended; 0 between steps
};

struct Moments {
  float *m, *v;             // 32 bits
  uint8_t *mc, *uc;         // 8 bits: codes, and
  uint32_t* e;              // exponents of a block, m's + 256 u's
};

struct Step {
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
// (both to a unit or two; of normal numbers, for which ftz does nothing)
__device__ __forceinline__ float reciprocal_fast(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float sqrt_fast(float x) {
  float r;
  asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// 8-bit magnitudes are fp32's bits without the low 23 - FRACTION ones, above an exponent: a floor of x is a
// shift of its bits, and so is floor(x / d + rho) with rho's bits added below.  Of m the highest bit is the sign (code 128
// is zero too).
template <int FRACTION>
__device__ __forceinline__ uint32_t block_exponent(float largest_of_four) {
  const uint32_t top = __reduce_max_sync(0xffffffffu, __float_as_uint(largest_of_four) & 0x7fffffffu);
  const uint32_t e = (top + ((1u << (23 - FRACTION)) - 1)) >> 23;
  return e < 16 ? 16 : e > kNoNumber ? kNoNumber : e;
}
// Codes in the low byte; bits above it are to be dropped.  All lanes of a warp come here together: values below the
// least code are rare, but for blocks of zeros, and have a way of their own.
template <int FRACTION, bool KEEP>  // KEEP: what is below the least code is held as it, not as it or zero
__device__ __forceinline__ void hold(const float (&x)[4], uint32_t e, const uint32_t (&r)[4], uint32_t (&code)[4]) {
  constexpr int kDrop = 23 - FRACTION;
  const uint32_t zero = (e - 15) << 23, least = zero + (1u << kDrop);
  uint32_t smallest = 0x7fffffffu;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t b = __float_as_uint(x[j]) & 0x7fffffffu;
    smallest = min(smallest, b);
    code[j] = (b - zero + (r[j] << (kDrop - 16))) >> kDrop;
  }
  if (__any_sync(0xffffffffu, smallest < least)) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float a = fabsf(x[j]);
      // a / least + rho >= 1, rho = r / 2^16: as a >= (2^16 - r) (least / 2^16), which has no rounding
      const uint32_t low = KEEP ? a > 0.f : a >= (float)(65536u - r[j]) * (__uint_as_float(least) * (1.f / 65536.f));
      if (__float_as_uint(a) < least) code[j] = low;
    }
  }
}
__device__ __forceinline__ void hold_m(const float (&x)[4], uint32_t e, const uint32_t (&r)[4], uint32_t (&code)[4]) {
  hold<3, false>(x, e, r, code);
#pragma unroll
  for (int j = 0; j < 4; ++j) code[j] = (code[j] & 127u) | (__float_as_uint(x[j]) >> 24 & 128u);
}
// What a code stands for in a block that is not NaN.
template <int FRACTION>
__device__ __forceinline__ float held(uint32_t code, uint32_t e) {
  return code ? __uint_as_float((code << (23 - FRACTION)) + ((e - 15) << 23)) : 0.f;
}
__device__ __forceinline__ float held_m(uint32_t code, uint32_t e) {
  return __uint_as_float(__float_as_uint(held<3>(code & 127u, e)) | (code & 128u) << 24);
}
__device__ __forceinline__ float unless_nan(float x, uint32_t e) { return e == kNoNumber ? __uint_as_float(0x7fffffffu) : x; }

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
    reinterpret_cast<uint32_t*>(to)[lane] = __byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410);
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

// What a step's blocks have in common.
struct Rates {
  float lr, rate, inv_root, scale;
  uint32_t key;
};

// What a thread has of a block of 128 values.
template <int BITS>
struct Values {
  float p[4], g[4], m[4], v[4];  // (moments of 32 bits)
  uint32_t mc[4], uc[4], e;      // (of 8)
};

template <int BITS, typename G, bool VECTOR>
__device__ __forceinline__ void read(const Step& a, const Tile& t, const G* grad, int lane, int i, int left, Values<BITS>& x) {
  const int64_t at = t.at + i;
  get4(t.p + i, VECTOR, lane, left, x.p);
  get4(grad + i, VECTOR, lane, left, x.g);
  if (BITS == 32) {
    get4(a.held.m + at, VECTOR, lane, left, x.m);
    get4(a.held.v + at, VECTOR, lane, left, x.v);
  } else {
    get_codes(a.held.mc + at, VECTOR, lane, x.mc);
    get_codes(a.held.uc + at, VECTOR, lane, x.uc);
    x.e = a.held.e[at / kBlock];
  }
}

// The step of a block.  Sums and products of moments are single operations (not contracted): 8-bit moments are the same
// wherever they are computed.
template <int BITS, typename H, bool COPY, bool VECTOR>
__device__ __forceinline__ void update(const Step& a, const Tile& t, const Rates& c, int lane, int i, int left, Values<BITS>& x) {
  const int64_t at = t.at + i;
  const uint32_t me = x.e & 255u, ue = x.e >> 8;
  // The decay's part is added to the step and taken off p with it: 1 - lr decay, rounded, would be the same for all values
  // and steps, and have two bits of an lr decay of 2^-23 and none of one below 2^-25.
  const float decay = c.lr * t.decay;
  // (a NaN block's codes count for nothing)
  const float b1 = BITS == 8 ? unless_nan(a.b1, me) : a.b1, b2 = BITS == 8 ? unless_nan(a.b2, ue) : a.b2;
  float u[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (BITS == 8) {
      const float old = held<4>(x.uc[j], ue);
      x.m[j] = held_m(x.mc[j], me), x.v[j] = __fmul_rn(old, old);
    }
    if (!VECTOR && lane + 32 * j >= left) x.m[j] = x.v[j] = 0.f;  // between tensors
    const float gs = __fmul_rn(x.g[j], c.scale);
    x.m[j] = __fadd_rn(__fmul_rn(x.m[j], b1), __fmul_rn(gs, a.one_b1));
    x.v[j] = __fadd_rn(__fmul_rn(x.v[j], b2), __fmul_rn(__fmul_rn(gs, gs), a.one_b2));
    u[j] = BITS == 8 ? __fsqrt_rn(x.v[j]) : sqrt_fast(x.v[j]);
    float step = c.rate * x.m[j] * reciprocal_fast(fmaf(u[j], c.inv_root, a.eps));
    if (decay != 0.f && fabsf(x.p[j]) <= FLT_MAX) step = fmaf(decay, x.p[j], step);  // (an infinite p stays that)
    x.p[j] -= step;
  }
  put4(t.p + i, VECTOR, lane, left, x.p);
  if (COPY) put4(static_cast<H*>(t.copy) + i, VECTOR, lane, left, x.p);
  if (BITS == 32) {
    put4(a.held.m + at, VECTOR, lane, left, x.m);
    put4(a.held.v + at, VECTOR, lane, left, x.v);
    return;
  }
  const uint32_t new_me = block_exponent<3>(largest(x.m)), new_ue = block_exponent<4>(largest(u));
  const int64_t place = at + (VECTOR ? lane * 4 : lane);
  // (a block does not cross a multiple of 2^32)
  const uint32_t from = (uint32_t)(place >> 32) * 0x85EBCA77u + (uint32_t)place * 0x9E3779B1u;
  uint32_t high[4], low[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t h = mix((from + (VECTOR ? j : 32 * j) * 0x9E3779B1u) ^ c.key);
    high[j] = h >> 16, low[j] = h & 0xffffu;
  }
  hold_m(x.m, new_me, high, x.mc);
  hold<4, true>(u, new_ue, low, x.uc);
  put_codes(a.held.mc + at, VECTOR, lane, x.mc);
  put_codes(a.held.uc + at, VECTOR, lane, x.uc);
  if (lane == 0) a.held.e[at / kBlock] = new_me | new_ue << 8;
}

// A warp's part of a tile whose values it cannot have four at a time, or not all of them.
template <int BITS, typename G, typename H, bool COPY>
__device__ __forceinline__ void update_singly(const Step& a, const Tile& t, const G* grad, bool aligned, const Rates& c, int lane, int begin) {
  for (int i = begin; i < begin + kMine && i < t.count; i += kBlock) {
    Values<BITS> x;
    if (aligned && t.count >= i + kBlock) {
      read<BITS, G, true>(a, t, grad, lane, i, kBlock, x);
      update<BITS, H, COPY, true>(a, t, c, lane, i, kBlock, x);
    } else {
      read<BITS, G, false>(a, t, grad, lane, i, t.count - i, x);
      update<BITS, H, COPY, false>(a, t, c, lane, i, t.count - i, x);
    }
  }
}

// Tiles of a block on their way to it (8 bits): a thread's part of a warp's four blocks of 128 values, in shared memory of
// its own.
struct Stage {
  float4 p[kBatch][kThreads];
  float4 g[kBatch][kThreads];  // (16-bit gradients: the first half of it)
  uint32_t mc[kBatch][kThreads], uc[kBatch][kThreads], e[kBatch][kThreads];
};

// A tile by the block, or (`stage` given) what of it has come to shared memory.
template <int BITS, typename H, bool COPY>
__device__ __forceinline__ void update_tile(const Step& a, const Tile& t, const void* grads, const Rates& c, int lane, int warp,
                                            const Stage* stage) {
  using G = std::conditional_t<COPY, H, float>;
  const G* grad = static_cast<const G*>(grads) + t.first;
  const bool aligned = t.vector && (uintptr_t)grad % (4 * sizeof(G)) == 0;
  const int begin = warp * kMine;
  if (!aligned || t.count < begin + kMine) return update_singly<BITS, G, H, COPY>(a, t, grad, aligned, c, lane, begin);
  if constexpr (BITS == 32) {
    Values<BITS> x[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) read<BITS, G, true>(a, t, grad, lane, begin + k * kBlock, kBlock, x[k]);
#pragma unroll
    for (int k = 0; k < kBatch; ++k) update<BITS, H, COPY, true>(a, t, c, lane, begin + k * kBlock, kBlock, x[k]);
  } else {
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      Values<BITS> x;
      const int tid = threadIdx.x;
      load_vec<float, 4>(reinterpret_cast<const float*>(&stage->p[k][tid]), x.p);
      load_vec<G, 4>(reinterpret_cast<const G*>(&stage->g[k][tid]), x.g);
      const uint32_t mc = stage->mc[k][tid], uc = stage->uc[k][tid];
#pragma unroll
      for (int j = 0; j < 4; ++j) x.mc[j] = mc >> 8 * j & 255u, x.uc[j] = uc >> 8 * j & 255u;
      x.e = stage->e[k][tid];
      update<BITS, H, COPY, true>(a, t, c, lane, begin + k * kBlock, kBlock, x);
    }
  }
}

// Sends for what update_tile() takes from a stage.
__device__ __forceinline__ void fetch_tile(const Step& a, const Tile& t, int lane, int warp, Stage* stage) {
  const void* grads = a.grads[t.tensor - a.first_tensor];
  const int size = t.copy ? 2 : 4, begin = warp * kMine, tid = threadIdx.x;
  const char* grad = static_cast<const char*>(grads) + t.first * size;
  if (!grads || !t.vector || (uintptr_t)grad % (4 * size) != 0 || t.count < begin + kMine) return;
#pragma unroll
  for (int k = 0; k < kBatch; ++k) {
    const int i = begin + k * kBlock + lane * 4;
    cp_async16(&stage->p[k][tid], t.p + i);
    if (t.copy)
      cp_async8(&stage->g[k][tid], grad + i * 2);
    else
      cp_async16(&stage->g[k][tid], grad + i * 4);
    cp_async4(&stage->mc[k][tid], a.held.mc + t.at + i);
    cp_async4(&stage->uc[k][tid], a.held.uc + t.at + i);
    cp_async4(&stage->e[k][tid], a.held.e + (t.at + i) / kBlock);
  }
}

template <int BITS, typename H>
__global__ void __launch_bounds__(kThreads, kResident) adamw_kernel(__grid_constant__ const Step a) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
  Tile next{};
  if (blockIdx.x < a.n_tiles) next = a.tiles[blockIdx.x];
  const State s = *a.state;
  Rates c;
  c.lr = a.d_lr ? *a.d_lr : a.lr, c.scale = a.grad_scale ? *a.grad_scale : 1.f;
  c.rate = c.lr / (float)(1.0 - s.b1t * a.b1d), c.inv_root = 1.f / sqrtf((float)(1.0 - s.b2t * a.b2d));
  c.key = mix(a.seed_lo ^ mix(a.seed_hi ^ mix((uint32_t)(s.steps + 1))));
  extern __shared__ __align__(16) char dynamic[];
  Stage *now = reinterpret_cast<Stage*>(dynamic), *later = now + 1;
  Tile t{};
  if (BITS == 8) {
    t = next;
    if (blockIdx.x < a.n_tiles) fetch_tile(a, t, lane, warp, now);
    cp_async_commit();
    if (blockIdx.x + gridDim.x < a.n_tiles) next = a.tiles[blockIdx.x + gridDim.x];
  }
  for (uint32_t k = blockIdx.x; k < a.n_tiles; k += gridDim.x) {
    Tile after{};
    if (BITS == 8) {
      if (k + gridDim.x < a.n_tiles) fetch_tile(a, next, lane, warp, later);
      cp_async_commit();
      if (k + 2 * (uint64_t)gridDim.x < a.n_tiles) after = a.tiles[k + 2 * gridDim.x];
      cp_async_wait<1>();
    } else {
      t = next;
      if (k + gridDim.x < a.n_tiles) next = a.tiles[k + gridDim.x];
    }
    if (const void* grads = a.grads[t.tensor - a.first_tensor]) {
      if (t.copy)
        update_tile<BITS, H, true>(a, t, grads, c, lane, warp, now);
      else
        update_tile<BITS, H, false>(a, t, grads, c, lane, warp, now);
    }
    if (BITS == 8) {
      Stage* free = now;
      now = later, later = free;
      t = next, next = after;
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

// Eight-bit moments as bf16, which holds all of a code's bits: a thread takes eight values of a block, four times.
constexpr int kEach = 4;
__global__ void __launch_bounds__(kThreads) moments_kernel(Moments from, int64_t values, __nv_bfloat16* m, __nv_bfloat16* u) {
  const int64_t first = ((int64_t)blockIdx.x * kThreads * kEach + threadIdx.x) * 8;
  uint2 mc[kEach], uc[kEach];
  uint32_t me[kEach], ue[kEach];
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const int64_t i = first + (int64_t)k * kThreads * 8;
    mc[k] = uc[k] = make_uint2(0, 0), me[k] = ue[k] = 16;
    if (i >= values) continue;
    mc[k] = *reinterpret_cast<const uint2*>(from.mc + i), uc[k] = *reinterpret_cast<const uint2*>(from.uc + i);
    me[k] = from.e[i / kBlock] & 255u, ue[k] = from.e[i / kBlock] >> 8;
  }
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const int64_t i = first + (int64_t)k * kThreads * 8;
    if (i >= values) break;
    float x[8], y[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      x[j] = unless_nan(held_m((j < 4 ? mc[k].x : mc[k].y) >> 8 * (j % 4) & 255u, me[k]), me[k]);
      y[j] = unless_nan(held<4>((j < 4 ? uc[k].x : uc[k].y) >> 8 * (j % 4) & 255u, ue[k]), ue[k]);
    }
    store_vec<__nv_bfloat16, 8>(m + i, x);
    store_vec<__nv_bfloat16, 8>(u + i, y);
  }
}

// Moments taken from outside (8 bits: to the nearest code).
template <int BITS>
__global__ void __launch_bounds__(kThreads) load_kernel(const Tile* tiles, Moments to, const void* m, const void* second) {
  const int lane = threadIdx.x & 31;
  const Tile t = tiles[blockIdx.x];
  for (int i = threadIdx.x / 32 * kBlock; i < t.count; i += kThreads / 32 * kBlock) {
    const int64_t at = t.at + i, left = t.count - i;
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
    const uint32_t half[4] = {0x8000u, 0x8000u, 0x8000u, 0x8000u};
    hold_m(x, me, half, mc);
    hold<4, true>(y, ue, half, uc);
    put_codes(to.mc + at, false, lane, mc);
    put_codes(to.uc + at, false, lane, uc);
    if (lane == 0) to.e[at / kBlock] = me | ue << 8;
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
  if (!((float)c->eps >= FLT_MIN) || !std::isfinite((float)c->eps)) return no("eps must be finite and 2^-126 at least");
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
  size_t first, second, exponents, state, tiles, total;
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
  if (c.state_bits == 8) k.exponents = take(z.values / kBlock * sizeof(uint32_t));
  k.state = take(sizeof(State));
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
    Moments h{};
    if (cfg.state_bits == 32) {
      h.m = reinterpret_cast<float*>(base + k.first), h.v = reinterpret_cast<float*>(base + k.second);
    } else {
      h.mc = reinterpret_cast<uint8_t*>(base + k.first), h.uc = reinterpret_cast<uint8_t*>(base + k.second);
      h.e = reinterpret_cast<uint32_t*>(base + k.exponents);
    }
    return h;
  }
};

namespace {

// Whether two tensors or copies share memory: their tiles would be written by two blocks at once.
bool overlap(const esspt_adamw_config& c, const esspt_adamw_tensor* tensors) {
  std::vector<std::pair<uintptr_t, uintptr_t>> spans;
  for (int k = 0; k < c.n_tensors; ++k) {
    const esspt_adamw_tensor& t = tensors[k];
    if (t.count == 0) continue;
    const uintptr_t p = reinterpret_cast<uintptr_t>(t.d_param), copy = reinterpret_cast<uintptr_t>(t.d_copy);
    spans.push_back({p, p + t.count * sizeof(float)});
    if (copy) spans.push_back({copy, copy + t.count * 2});
  }
  std::sort(spans.begin(), spans.end());
  for (size_t k = 1; k < spans.size(); ++k)
    if (spans[k].first < spans[k - 1].second) return true;
  return false;
}

esspt_status fill(esspt_adamw* aw, const esspt_adamw_tensor* tensors) {
  const esspt_adamw_config& c = aw->cfg;
  std::vector<Tile> tiles;
  int64_t at = 0;
  for (int k = 0; k < c.n_tensors; ++k) {
    const esspt_adamw_tensor& t = tensors[k];
    const bool vector = !misaligned(t.d_param, 16) && !misaligned(t.d_copy, 8);
    aw->sizes.push_back(t.count == 0 ? 0 : t.d_copy ? 2 : 4);
    if (k % kGroup == 0) aw->first_tile.push_back((uint32_t)tiles.size());
    for (int64_t i = 0; i < t.count; i += kTile) {
      const int64_t left = t.count - i;
      tiles.push_back(Tile{t.d_param + i, t.d_copy ? static_cast<uint16_t*>(t.d_copy) + i : nullptr, i, at + i, (uint32_t)k,
                           (int32_t)(left < kTile ? left : kTile), t.weight_decay, vector});
    }
    at += (t.count + kBlock - 1) / kBlock * kBlock;
  }
  aw->first_tile.push_back((uint32_t)tiles.size());
  ESSPT_CUDA(g_create, cudaMemsetAsync(aw->base, 0, aw->k.state, aw->st));
  ESSPT_CUDA(g_create, cudaMemcpyAsync(aw->base + aw->k.tiles, tiles.data(), tiles.size() * sizeof(Tile), cudaMemcpyHostToDevice, aw->st));
  state_kernel<<<1, 1, 0, aw->st>>>(reinterpret_cast<State*>(aw->base + aw->k.state), State{0, 1.0, 1.0, 0u});
  ESSPT_CUDA(g_create, cudaGetLastError());
  ESSPT_CUDA(g_create, cudaStreamSynchronize(aw->st));
  return ESSPT_OK;
}

template <int BITS>
cudaError_t launch(const esspt_adamw_config& c, unsigned blocks, cudaStream_t st, const Step& a) {
  auto* kernel = c.copy_dtype == ESSPT_BF16 ? adamw_kernel<BITS, __nv_bfloat16> : adamw_kernel<BITS, __half>;
  const int shared = BITS == 8 ? 2 * sizeof(Stage) : 0;
  if (shared > 0) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, shared);
    if (e != cudaSuccess) return e;
  }
  kernel<<<blocks, kThreads, shared, st>>>(a);
  return cudaGetLastError();
}

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
  try {
    if (overlap(*cfg, tensors)) return g_create.fail(ESSPT_EINVAL, "two tensors overlap");
  } catch (const std::bad_alloc&) {
    return g_create.fail(ESSPT_ENOSPC, "out of host memory");
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
    const unsigned most = (unsigned)(kResident * aw->sms), blocks = a.n_tiles == 0 ? 1 : a.n_tiles < most ? a.n_tiles : most;
    ESSPT_CUDA(aw->err, c.state_bits == 32 ? launch<32>(c, blocks, aw->st, a) : launch<8>(c, blocks, aw->st, a));
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
  const int64_t each = kThreads * kEach * 8, blocks = (aw->values + each - 1) / each;
  moments_kernel<<<(unsigned)blocks, kThreads, 0, aw->st>>>(aw->moments(), aw->values, static_cast<__nv_bfloat16*>(d_m),
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
    const Tile* tile = reinterpret_cast<const Tile*>(aw->base + aw->k.tiles);
    if (c.state_bits == 32)
      load_kernel<32><<<tiles, kThreads, 0, aw->st>>>(tile, aw->moments(), d_m, d_second);
    else
      load_kernel<8><<<tiles, kThreads, 0, aw->st>>>(tile, aw->moments(), d_m, d_second);
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
