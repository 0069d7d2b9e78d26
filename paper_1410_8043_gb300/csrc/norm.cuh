// Layer norm, forward and backward: kernels.
//
// A group of lanes (a part of a warp, a warp, or for wide rows a block) holds a row in registers, N vectors of
// VEC values a lane, so that a row is read once.  Groups stay and go through rows: their weights stay in registers, and
// each thread's parts of the next rows are copied to its own places in shared memory meanwhile.  All arithmetic is fp32,
// two values an instruction.
//
// Memory is the bound for rows of 16-byte vectors, with issue close behind for 16-bit ones (32771 rows of 2048 bf16 values:
// forward 47 us, 5.7 TB/s, issue 67% of the time; backward 65 us, 6.2 TB/s, and 14 us for the weights' sums; fp32: 93 and
// 129 us, 5.8 and 6.2 TB/s).  Sixteen values a thread halve what eight pay in sums over a row.  Rows of an odd number of 16-bit values
// go by single ones: 82 and 143 us for 2047 values.
#pragma once

#include <cfloat>
#include <type_traits>

#include "chained.cuh"
#include "norm.h"
#include "operator.h"
#include "ptx.cuh"
#include "rows.cuh"

namespace esspt {

constexpr int kThreads = kNormThreads, kMostWide = kNormWide, kMostWarps = kMostWide / 32;

// A thread's N vectors of a row as pairs of fp32 values (one value alone has a zero beside it).
template <int VEC, int N>
constexpr int kPairs = (VEC * N + 1) / 2;

template <typename T, int VEC>
struct alignas(VEC * sizeof(T)) Pack {
  T v[VEC];
};

template <typename T, int VEC, int N>
__device__ __forceinline__ void to_pairs(const Pack<T, VEC> (&p)[N], u64 (&x)[kPairs<VEC, N>]) {
#pragma unroll
  for (int q = 0; q < kPairs<VEC, N>; ++q) {
    const int e = 2 * q, f = e + 1;
    x[q] = pack2(to_float(p[e / VEC].v[e % VEC]), f < VEC * N ? to_float(p[f % (VEC * N) / VEC].v[f % VEC]) : 0.f);
  }
}

// Rows on their way to a thread.  Parts of 4 bytes or more go to shared memory, kDepth - 1 rows ahead; smaller ones
// stay in registers, a row ahead.  What lies outside a row or the rows is zero.
template <typename T, int VEC, int N>
struct Incoming {
  using P = Pack<T, VEC>;
  static constexpr bool kAsync = sizeof(P) >= 4;
  // (64 bytes a row for 512 threads, two such rows backward: 200 KB of three stages; four are not faster)
  static constexpr int kDepth = sizeof(P) < 16 ? 2 : 3;
  P *first, *read, *write;  // the thread's slot of the first stage, of the one to take from, of the one to fetch to
  int pitch;                // slots from one vector to the next
  int stage_read, stage_write;
  const T* at;              // its first vector of the next row to fetch
  int64_t step;             // values to that of the one after
  P next[kAsync ? 1 : N];

  __device__ __forceinline__ static int bytes(int threads) { return kAsync ? kDepth * N * threads * (int)sizeof(P) : 0; }
  __device__ __forceinline__ Incoming(char* slots, const T* from, int64_t step_, int D, int lane, int lanes)
      : first(reinterpret_cast<P*>(slots) + threadIdx.x), read(first), write(first), pitch(blockDim.x), stage_read(0),
        stage_write(0), at(from + lane * VEC), step(step_) {
    if constexpr (kAsync) {
#pragma unroll
      for (int k = 0; k < kDepth * N; ++k)
        if ((lane + k % N * lanes) * VEC >= D) first[k * pitch] = zero();
    }
  }
  __device__ __forceinline__ static P zero() {
    P p;
#pragma unroll
    for (int j = 0; j < VEC; ++j) p.v[j] = from_float<T>(0.f);
    return p;
  }
  __device__ __forceinline__ void advance(P*& slot, int& stage) {
    const bool wrap = stage == kDepth - 1;
    slot = wrap ? first : slot + N * pitch;
    stage = wrap ? 0 : stage + 1;
  }
  // The row taken last, until the next fetch.
  __device__ __forceinline__ const P* taken() const { return first + (stage_read == 0 ? kDepth - 1 : stage_read - 1) * N * pitch; }
  __device__ __forceinline__ void take_again(u64 (&x)[kPairs<VEC, N>]) const {
    P p[N];
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = taken()[i * pitch];
    to_pairs<T, VEC, N>(p, x);
  }
  __device__ __forceinline__ void fetch(int D, int lane, int lanes, bool live) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const bool inside = (lane + i * lanes) * VEC < D;
      if constexpr (kAsync) {
        if (inside && live) {
          if constexpr (sizeof(P) >= 16)
            cp_async16(write + i * pitch, at + i * lanes * VEC);
          else
            cp_async4(write + i * pitch, at + i * lanes * VEC);
        } else if (inside) {
          write[i * pitch] = zero();
        }
      } else {
        next[i].v[0] = inside && live ? at[i * lanes] : from_float<T>(0.f);
      }
    }
    if constexpr (kAsync) advance(write, stage_write);
    at += step;
  }
  __device__ __forceinline__ void take(u64 (&x)[kPairs<VEC, N>]) {
    P p[N];
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = kAsync ? read[i * pitch] : next[kAsync ? 0 : i];
    if constexpr (kAsync) advance(read, stage_read);
    to_pairs<T, VEC, N>(p, x);
  }
};

template <typename T>
__device__ __forceinline__ float weight_at(const Norm& a, const void* from, float otherwise, int c) {
  return !from ? otherwise : a.weight_f32 ? static_cast<const float*>(from)[c] : to_float(static_cast<const T*>(from)[c]);
}
// Weights by single values: they may stand anywhere, and are read once.
template <typename T, int VEC, int N>
__device__ __forceinline__ void load_weights(const Norm& a, const void* from, float otherwise, int lane, u64 (&x)[kPairs<VEC, N>]) {
  float w[2 * kPairs<VEC, N>];
#pragma unroll
  for (int e = 0; e < 2 * kPairs<VEC, N>; ++e) {
    const int c = (lane + e / VEC * a.lanes) * VEC + e % VEC;
    w[e] = e < VEC * N && c < a.D ? weight_at<T>(a, from, otherwise, c) : otherwise;
  }
#pragma unroll
  for (int q = 0; q < kPairs<VEC, N>; ++q) x[q] = pack2(w[2 * q], w[2 * q + 1]);
}

// The sum over the lanes of a warp that hold one row; over those that hold the warps' sums.
__device__ __forceinline__ float lanes_sum(float v, int lanes) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) {
    const float other = __shfl_xor_sync(0xffffffffu, v, off);
    if (off < lanes) v += other;
  }
  return v;
}
__device__ __forceinline__ float warps_sum(float v, int warps) {  // (a power of two)
  for (int off = warps / 2; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
  return v;
}
// Two sums over a warp: x's in the lower half of the lanes, y's in the upper.
__device__ __forceinline__ float warp_sums(float x, float y) {
  const bool upper = threadIdx.x & 16;
  float v = (upper ? y : x) + __shfl_xor_sync(0xffffffffu, upper ? x : y, 16);
#pragma unroll
  for (int off = 8; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
  return v;
}

template <typename T, int VEC, int N>
__device__ __forceinline__ void store_pairs(T* row, int D, int lane, int lanes, const u64 (&x)[kPairs<VEC, N>]) {
  float v[2 * kPairs<VEC, N>];
#pragma unroll
  for (int q = 0; q < kPairs<VEC, N>; ++q) unpack2(x[q], v[2 * q], v[2 * q + 1]);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int c = (lane + i * lanes) * VEC;
    float out[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) out[j] = v[i * VEC + j];
    if (c < D) store_vec<T, VEC>(row + c, out);
  }
}

// The mean is a rounded sum times a rounded 1 / D, off by some 10 units of its last place.  In rows that vary by little more than
// that, all differences to it are off, and the variance by that error's square.  Rows whose mean is more than kFar standard
// deviations (of variance + eps) from zero are corrected: the differences have no such error, and their own mean says how far
// the first one was off.  In others x^ is off by some 10 kFar units at most.  It is done once a row is written, from its copy in
// shared memory, for other rows' registers and speed: in line for all of them it took 10 to 25% more of the pass; now 32771 rows of
// 2048 bf16 values take 47 us, and 87 if all are far, 20000 of 8192 136 and 257.  Asking takes 3 to 7% of rows of up to 256 values.
constexpr float kFar = 8.f;

// What such rows take, in loops, for few registers.  `from`: a thread's first vector of the row, in shared memory where it was
// copied, `step` values to its next one.
template <typename T, int VEC>
__device__ __forceinline__ float2 far_sums(const T* from, int step, int c, int lanes, int D, float mean) {
  float2 sums = make_float2(0.f, 0.f);  // of differences to `mean`, and their squares
#pragma unroll 1
  for (; c < D; c += lanes * VEC, from += step) {
    float v[VEC];
    load_vec<T, VEC>(from, v);
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      const float d = v[j] - mean;
      sums.x += d, sums.y = fmaf(d, d, sums.y);
    }
  }
  return sums;
}

// (registers as spread() counts on them)
template <typename T, int VEC, int N, bool WIDE>
__global__ void __launch_bounds__(WIDE ? (VEC >= 4 ? 768 : kMostWide) : kThreads, WIDE ? 1 : VEC * N <= 8 ? 4 : VEC >= 4 ? 3 : 2)
    norm_forward_kernel(Norm a) {
  extern __shared__ __align__(16) char dynamic[];
  __shared__ float2 shared[2][kMostWarps], shared_far[kMostWarps];
  constexpr int Q = kPairs<VEC, N>;
  using In = Incoming<T, VEC, N>;
  const int lanes = WIDE ? blockDim.x : N > 1 ? 32 : a.lanes, lane = threadIdx.x & (WIDE ? ~0 : lanes - 1);  // (as spread() has them)
  const int groups = WIDE ? 1 : blockDim.x / lanes, group = WIDE ? 0 : threadIdx.x / lanes;
  int64_t t = (int64_t)blockIdx.x * groups + group, ahead = t;  // the row at hand, the next one to fetch
  const int64_t step = (int64_t)gridDim.x * groups;
  In in(dynamic, static_cast<const T*>(a.x) + t * a.x_stride, step * a.x_stride, a.D, lane, lanes);
  auto fetch = [&]() {
    in.fetch(a.D, lane, lanes, ahead < a.n);
    if (In::kAsync) cp_async_commit();
    ahead += step;
  };
#pragma unroll
  for (int k = 0; k < In::kDepth - 1; ++k) fetch();
  u64 w[Q], b[Q];
  load_weights<T, VEC, N>(a, a.weight, 1.f, lane, w);
  load_weights<T, VEC, N>(a, a.bias, 0.f, lane, b);
  auto count = [&](int warp) {  // values of a warp
    int c = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int left = a.D - (warp * 32 + i * lanes) * VEC;
      c += left < 0 ? 0 : left < 32 * VEC ? left : 32 * VEC;
    }
    return (float)c;
  };
  int warps = 1;
  while (WIDE && warps * 32 < blockDim.x) warps *= 2;
  const int warp = threadIdx.x / 32, other = threadIdx.x & (warps - 1);
  const float inv_own = WIDE ? 1.f / fmaxf(count(warp), 1.f) : a.inv_D;
  const float count_other = WIDE && other < blockDim.x / 32 ? count(other) : 0.f;
  int turn = 0;
  for (int64_t t0 = (int64_t)blockIdx.x * groups; t0 < a.n; t0 += step, t += step, turn ^= 1) {
    u64 x[Q];
    if (In::kAsync) {
      fetch();
      cp_async_wait<In::kDepth - 1>();
    }
    in.take(x);
    if (!In::kAsync) fetch();
    // Mean and squares of differences to it, of the lanes of a warp.
    u64 sum = x[0];
#pragma unroll
    for (int q = 1; q < Q; ++q) sum = add2(sum, x[q]);
    float mean = lanes_sum(sum2(sum), WIDE ? 32 : lanes) * inv_own;
    const u64 minus = pack2(-mean, -mean);
    u64 squares = 0;
    float single = 0.f;  // (of vectors of one value each its own)
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if ((lane + i * lanes) * VEC >= a.D) continue;
      if constexpr (VEC == 1) {
        float lo, hi;
        unpack2(x[i / 2], lo, hi);
        const float d = (i % 2 ? hi : lo) - mean;
        single = fmaf(d, d, single);
      } else {
#pragma unroll
        for (int q = i * VEC / 2; q < (i + 1) * VEC / 2; ++q) {
          const u64 d = add2(x[q], minus);
          squares = fma2(d, d, squares);
        }
      }
    }
    float m2 = lanes_sum(sum2(squares) + single, WIDE ? 32 : lanes);
    if (WIDE) {
      // Of the warps: squares about the row's mean are those about a warp's and their distance's.
      if ((threadIdx.x & 31) == 0) shared[turn][warp] = make_float2(mean, m2);
      __syncthreads();  // (the next row's go to the other half)
      const float2 v = count_other > 0.f ? shared[turn][other] : make_float2(0.f, 0.f);
      // (a product by itself: fused with the first sum, threads would have different last bits, and `far` has to be the block's)
      mean = warps_sum(__fmul_rn(count_other, v.x), warps) * a.inv_D;
      m2 = warps_sum(v.y + count_other * (v.x - mean) * (v.x - mean), warps);
    }
    const float rstd = rsqrtf(m2 * a.inv_D + a.eps);
    const bool far = fabsf(mean) * rstd > kFar;  // (not where squares overflow or are NaN)
    if ((WIDE || t < a.n) && (In::kAsync || !far)) {
      const u64 m = pack2(-mean, -mean), r = pack2(rstd, rstd);
#pragma unroll
      for (int q = 0; q < Q; ++q) x[q] = fma2(mul2(add2(x[q], m), r), w[q], b[q]);
      store_pairs<T, VEC, N>(static_cast<T*>(a.y) + t * a.D, a.D, lane, lanes, x);
      if (lane == 0 && a.mean) a.mean[t] = mean, a.rstd[t] = rstd;
    }
    if (__builtin_expect(!__any_sync(0xffffffffu, far), 1)) continue;  // (of a wide row's block all say the same)
    // Once more (over what was written, if the row is still in shared memory).
    const T* from = In::kAsync ? reinterpret_cast<const T*>(in.taken()) : static_cast<const T*>(a.x) + t * a.x_stride + lane;
    const int pitch = In::kAsync ? in.pitch * VEC : lanes;
    float2 v = far ? far_sums<T, VEC>(from, pitch, lane * VEC, lanes, a.D, mean) : make_float2(0.f, 0.f);
    if (WIDE) {
      const float own = warp_sums(v.x, v.y);
      if ((threadIdx.x & 15) == 0) (threadIdx.x & 16 ? shared_far[warp].y : shared_far[warp].x) = own;
      __syncthreads();  // (and the next row's above before it is written again)
      v = count_other > 0.f ? shared_far[other] : make_float2(0.f, 0.f);
      v = make_float2(warps_sum(v.x, warps), warps_sum(v.y, warps));
    } else {
      v = make_float2(lanes_sum(v.x, lanes), lanes_sum(v.y, lanes));
    }
    if (!far) continue;
    const float rest = v.y <= FLT_MAX ? v.x * a.inv_D : 0.f, rstd_far = rsqrtf((v.y - fminf(v.x * rest, v.y)) * a.inv_D + a.eps);
    T* row = static_cast<T*>(a.y) + t * a.D;
    if constexpr (VEC > 1) {
      in.take_again(x);
      const u64 m = pack2(-mean, -mean), m_far = pack2(-rest, -rest), r = pack2(rstd_far, rstd_far);
#pragma unroll
      for (int q = 0; q < Q; ++q) x[q] = fma2(mul2(add2(add2(x[q], m), m_far), r), w[q], b[q]);
      store_pairs<T, VEC, N>(row, a.D, lane, lanes, x);
    } else {
#pragma unroll 1
      for (int c = lane; c < a.D; c += lanes, from += pitch)
        row[c] = from_float<T>(fmaf((to_float(*from) - mean - rest) * rstd_far, weight_at<T>(a, a.weight, 1.f, c), weight_at<T>(a, a.bias, 0.f, c)));
    }
    if (lane == 0 && a.mean) a.mean[t] = mean + rest, a.rstd[t] = rstd_far;
  }
}

// A thread's columns are the same in all rows, and it keeps their sums for dw and db; at the end those of a
// block are added, the groups of a warp by shuffles, then warp behind warp.
template <typename T, int VEC, int N, bool WIDE>
__global__ void __launch_bounds__(WIDE ? kMostWide : kThreads) norm_backward_kernel(Norm a) {
  extern __shared__ __align__(16) char dynamic[];
  __shared__ float2 shared[2][kMostWarps];
  constexpr int Q = kPairs<VEC, N>;
  using In = Incoming<T, VEC, N>;
  const int lanes = WIDE ? blockDim.x : a.lanes, lane = threadIdx.x & (WIDE ? ~0 : lanes - 1);
  const int groups = WIDE ? 1 : blockDim.x / lanes, group = WIDE ? 0 : threadIdx.x / lanes;
  int64_t t = (int64_t)blockIdx.x * groups + group, ahead = t;  // the row at hand, the next one to fetch
  const int64_t step = (int64_t)gridDim.x * groups;
  In in_x(dynamic, static_cast<const T*>(a.x) + t * a.x_stride, step * a.x_stride, a.D, lane, lanes);
  In in_dy(dynamic + In::bytes(blockDim.x), static_cast<const T*>(a.dy) + t * a.dy_stride, step * a.dy_stride, a.D, lane, lanes);
  auto fetch = [&]() {
    in_x.fetch(a.D, lane, lanes, ahead < a.n);
    in_dy.fetch(a.D, lane, lanes, ahead < a.n);
    if (In::kAsync) cp_async_commit();
    ahead += step;
  };
  auto stats = [&](int64_t at) { return at < a.n ? make_float2(a.mean[at], a.rstd[at]) : make_float2(0.f, 0.f); };
#pragma unroll
  for (int k = 0; k < In::kDepth - 1; ++k) fetch();
  // Statistics of as many rows as a warp's part of a row has lanes, a lane each, and the next so many under way.
  const int own_lanes = WIDE ? 32 : lanes, own_lane = threadIdx.x & (own_lanes - 1), lane0 = (threadIdx.x & 31) - own_lane;
  float2 now = stats(t + own_lane * step), later = stats(t + (own_lanes + own_lane) * step);
  int turns_left = own_lanes;
  u64 w[Q], dw[Q], db[Q];
  load_weights<T, VEC, N>(a, a.weight, 1.f, lane, w);
#pragma unroll
  for (int q = 0; q < Q; ++q) dw[q] = db[q] = 0;
  int warps = 1;
  while (WIDE && warps * 32 < blockDim.x) warps *= 2;
  int turn = 0;
  for (int64_t t0 = (int64_t)blockIdx.x * groups; t0 < a.n; t0 += step, t += step, turn ^= 1) {
    u64 x[Q], dy[Q];
    if (In::kAsync) {
      fetch();
      cp_async_wait<In::kDepth - 1>();
    }
    in_x.take(x);
    in_dy.take(dy);
    if (turns_left == 0) {
      now = later, later = stats(t + (own_lanes + own_lane) * step);
      turns_left = own_lanes;
    }
    float2 s;
    s.x = __shfl_sync(0xffffffffu, now.x, lane0 + own_lanes - turns_left);
    s.y = __shfl_sync(0xffffffffu, now.y, lane0 + own_lanes - turns_left);
    --turns_left;
    if (!In::kAsync) fetch();
    const float rstd = s.y;
    const u64 m = pack2(-s.x, -s.x), r = pack2(rstd, rstd);
    u64 sum_g = 0, sum_gx = 0;  // (outside a row dy is zero)
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      x[q] = mul2(add2(x[q], m), r);
      dw[q] = fma2(dy[q], x[q], dw[q]);
      db[q] = add2(dy[q], db[q]);
      dy[q] = mul2(dy[q], w[q]);
      sum_g = add2(sum_g, dy[q]);
      sum_gx = fma2(dy[q], x[q], sum_gx);
    }
    if (!a.y) continue;
    if (WIDE) {
      const float v = warp_sums(sum2(sum_g), sum2(sum_gx));
      if ((threadIdx.x & 15) == 0) (threadIdx.x & 16 ? shared[turn][threadIdx.x / 32].y : shared[turn][threadIdx.x / 32].x) = v;
      __syncthreads();  // (the next row's go to the other half)
      const int other = threadIdx.x & (warps - 1);
      s = other < blockDim.x / 32 ? shared[turn][other] : make_float2(0.f, 0.f);
      s = make_float2(warps_sum(s.x, warps), warps_sum(s.y, warps));
    } else {
      s = make_float2(lanes_sum(sum2(sum_g), lanes), lanes_sum(sum2(sum_gx), lanes));
    }
    if (t >= a.n) continue;
    const u64 g = pack2(-s.x * a.inv_D, -s.x * a.inv_D), gx = pack2(-s.y * a.inv_D, -s.y * a.inv_D);
#pragma unroll
    for (int q = 0; q < Q; ++q) x[q] = mul2(add2(fma2(x[q], gx, dy[q]), g), r);
    store_pairs<T, VEC, N>(static_cast<T*>(a.y) + t * a.D, a.D, lane, lanes, x);
  }
  if (!a.want_w) return;
  float* sums = reinterpret_cast<float*>(dynamic);  // [2][D] (rows of a warp: the copies' places, which are done with)
  if (!WIDE) {
    for (int off = 16; off >= lanes; off >>= 1)
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        dw[q] = add2(dw[q], __shfl_xor_sync(0xffffffffu, dw[q], off));
        db[q] = add2(db[q], __shfl_xor_sync(0xffffffffu, db[q], off));
      }
    cp_async_wait_all();
    __syncthreads();
  }
  float* part = a.part + (int64_t)blockIdx.x * 2 * a.D;
  const int turns = WIDE ? 1 : blockDim.x / 32;
  for (int k = 0; k < turns; ++k) {
    if (WIDE || (threadIdx.x / 32 == k && (threadIdx.x & 31) < lanes)) {
      float* to = k == turns - 1 ? part : sums;
      float v[2 * Q], u[2 * Q];
#pragma unroll
      for (int q = 0; q < Q; ++q) unpack2(dw[q], v[2 * q], v[2 * q + 1]), unpack2(db[q], u[2 * q], u[2 * q + 1]);
#pragma unroll
      for (int e = 0; e < VEC * N; ++e) {
        const int c = (lane + e / VEC * lanes) * VEC + e % VEC;
        if (c < a.D) {
          to[c] = (k ? sums[c] : 0.f) + v[e];
          to[a.D + c] = (k ? sums[a.D + c] : 0.f) + u[e];
        }
      }
    }
    if (k < turns - 1) __syncthreads();
  }
}

template <bool BACK, typename T, int VEC, int N, bool WIDE>
cudaError_t launch(const Spread& s, const Norm& a, unsigned blocks, cudaStream_t st) {
  using In = Incoming<T, VEC, N>;
  auto bytes = [](int threads, int D) {
    const size_t rows = (size_t)(BACK ? 2 : 1) * (In::kAsync ? In::kDepth * N * threads * VEC * (int)sizeof(T) : 0), sums = 2 * D * sizeof(float);
    return BACK && !WIDE && rows < sums ? sums : rows;
  };
  const size_t shared = bytes(s.threads, a.D);
  auto* kernel = BACK ? norm_backward_kernel<T, VEC, N, WIDE> : norm_forward_kernel<T, VEC, N, WIDE>;
  if (shared > 47 * 1024) {  // (static shared memory counts too)
    // The limit is the kernel's, not this call's: always what its widest rows take, as another thread may be about to launch it.
    const size_t most = bytes(WIDE ? kMostWide : kThreads, 32 * N * VEC);
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most);
    if (e != cudaSuccess) return e;
  }
  kernel<<<blocks, s.threads, shared, st>>>(a);
  return cudaGetLastError();
}

template <bool BACK, typename T, int VEC>
cudaError_t launch_by_size(Norm& a, int sms, unsigned* blocks, cudaStream_t st) {
  const Spread s = spread(a.D, VEC, BACK);
  a.lanes = s.lanes;
  const int64_t groups = (a.n + s.threads / s.lanes - 1) / (s.threads / s.lanes);
  *blocks = (unsigned)(groups > sms * s.resident ? sms * s.resident : groups);
  if (s.wide) return launch<BACK, T, VEC, kNormValues / VEC, true>(s, a, *blocks, st);
  auto go = [&](auto n) { return launch<BACK, T, VEC, n, false>(s, a, *blocks, st); };
  if (s.n == 1) return go(std::integral_constant<int, 1>{});
  if (s.n == 2) return go(std::integral_constant<int, 2>{});
  if constexpr (VEC <= 4) {
    if (s.n == 4) return go(std::integral_constant<int, 4>{});
  }
  if constexpr (VEC <= 2) {
    if (s.n == 8) return go(std::integral_constant<int, 8>{});
  }
  if constexpr (VEC == 1) {
    if (s.n == 16) return go(std::integral_constant<int, 16>{});
  }
  return cudaErrorInvalidConfiguration;
}

template <typename T>
cudaError_t launch_norm(Norm& a, bool back, int bytes, int sms, unsigned* blocks, cudaStream_t st) {
  constexpr int kWhole = 16 / sizeof(T);
  auto go = [&](auto vec) {
    return back ? launch_by_size<true, T, vec>(a, sms, blocks, st) : launch_by_size<false, T, vec>(a, sms, blocks, st);
  };
  if (bytes >= 16) return go(std::integral_constant<int, kWhole>{});
  if constexpr (sizeof(T) == 2) {
    if (bytes >= 4) return go(std::integral_constant<int, 2>{});
  }
  return go(std::integral_constant<int, 1>{});
}

}  // namespace esspt
