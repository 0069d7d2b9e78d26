// Softmax operators for a few rows (single users, single tokens): one pass over
// W gives the scores of up to kFewRows rows, a second one both gradients.
#include <algorithm>

#include "softmax.cuh"

namespace esspt {

namespace {

constexpr int kThreads = 256;

// Shares of a teacher's lists, a warp per row: q_k = 2^((z_k - m) b / ln 2) / l with
// (m, l) over the present entries, and sum q log q.  (Differences first: they are
// exact where they matter, for logits of any size.)
__global__ void targets_kernel(TargetArgs a) {
  const int64_t t = (int64_t)blockIdx.x * (blockDim.x / 32) + threadIdx.x / 32;
  const int lane = threadIdx.x & 31;
  if (t >= a.n) return;
  const int32_t* ids = a.ids + t * a.top;
  if (!a.logits) {
    if (lane == 0 && ids[0] >= a.V) atomicOr(a.status, kErrTarget);
    return;
  }
  const float* z = a.logits + t * a.top;
  const float scale = a.b * kLog2e;
  float m = -INFINITY, l = 0.f;
  bool present = false, nan = false;
  for (int k = lane; k < a.top; k += 32) {
    const int32_t id = ids[k];
    if (id >= a.V) atomicOr(a.status, kErrTarget);
    const float s = z[k];
    if ((uint32_t)id < (uint32_t)a.V) {
      m = fmaxf(m, s);
      nan |= s != s;
      present |= s != -INFINITY;
    }
  }
  m = warp_max(m);
  nan = __any_sync(0xffffffffu, nan);
  present = __any_sync(0xffffffffu, present);
  if (nan) m = NAN;
  for (int k = lane; k < a.top; k += 32)
    if ((uint32_t)ids[k] < (uint32_t)a.V) l += present ? exp2f((z[k] - m) * scale) : 0.f;
  l = warp_sum(l);
  const float log2_l = log2f(l);
  float self = 0.f;
  for (int k = lane; k < a.top; k += 32) {
    float q = 0.f;
    if (present && (uint32_t)ids[k] < (uint32_t)a.V) {
      const float d = (z[k] - m) * scale;
      q = exp2f(d) / l;
      if (q != 0.f) self += q * (d - log2_l);  // (NaN takes part)
    }
    a.q[t * a.top + k] = q;
  }
  self = warp_sum(self);
  if (lane == 0) a.self[t] = present ? self * kLn2 : kIgnored;
}

struct Few {
  SoftmaxArgs a;
  FewScratch s;
  int64_t t0;  // first row of the group
  int32_t rows;
  int32_t blocks;
  int first, last;  // of the call's groups
};

// Scores of all items: four lanes to an item (each a quarter of its slices of VEC
// values), eight items to a warp side by side, U deep; rows of H from shared memory, where
// the four lanes read one 64-byte line for all items.  The lanes' sums meet by
// halving: each lane ends with two rows' totals, so no exponential is taken twice.
template <typename T, int VEC>
__global__ void __launch_bounds__(kThreads) few_scores_kernel(Few f) {
  constexpr int U = 4, R = kFewRows;
  extern __shared__ __align__(16) float hs[];  // [slices][R][VEC]
  __shared__ float2 warp_part[kThreads / 32][R];
  const SoftmaxArgs& a = f.a;
  const int lane = threadIdx.x & 31, ql = lane & 3;
  const int32_t slices = (a.D + VEC - 1) / VEC;
  const T* h = static_cast<const T*>(a.h);
  for (int i = threadIdx.x; i < slices * R * VEC; i += kThreads) {
    const int d = i / (R * VEC) * VEC + i % VEC, r = i / VEC % R;
    const int64_t t = f.t0 + r;
    hs[i] = r < f.rows && d < a.D && row_kept(a.target, t) ? to_float(h[t * a.h_stride + d]) : 0.f;
  }
  __syncthreads();
  const T* w = static_cast<const T*>(a.w);
  const float k2 = a.b * kLog2e;
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
  const int row0 = (lane & 2) * 2 + (lane & 1) * 2;  // this lane's rows after halving: row0, row0 + 1
  const int64_t step = (int64_t)gridDim.x * (kThreads / 32) * 8 * U;
  for (int64_t v0 = ((int64_t)blockIdx.x * (kThreads / 32) + threadIdx.x / 32) * 8 * U; v0 < a.V; v0 += step) {
    float acc[U][R];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int r = 0; r < R; ++r) acc[u][r] = 0.f;
    const T* row[U];
#pragma unroll
    for (int u = 0; u < U; ++u) row[u] = w + min(v0 + u * 8 + lane / 4, (int64_t)a.V - 1) * a.w_stride;
    for (int i = ql; i < slices; i += 4) {
      float x[U][VEC];
#pragma unroll
      for (int u = 0; u < U; ++u) load_vec<T, VEC>(row[u] + i * VEC, x[u]);
      const float* hv = hs + i * R * VEC;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float y[VEC];
        if constexpr (VEC >= 4) {
#pragma unroll
          for (int e = 0; e < VEC; e += 4) {
            const float4 q = *reinterpret_cast<const float4*>(hv + r * VEC + e);
            y[e] = q.x, y[e + 1] = q.y, y[e + 2] = q.z, y[e + 3] = q.w;
          }
        } else {
          y[0] = hv[r];
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int e = 0; e < VEC; ++e) acc[u][r] = fmaf(x[u][e], y[e], acc[u][r]);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float half[4], s[2];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float give = (lane & 2) ? acc[u][r] : acc[u][r + 4], keep = (lane & 2) ? acc[u][r + 4] : acc[u][r];
        half[r] = keep + __shfl_xor_sync(0xffffffffu, give, 2);
      }
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const float give = (lane & 1) ? half[r] : half[r + 2], keep = (lane & 1) ? half[r + 2] : half[r];
        s[r] = (keep + __shfl_xor_sync(0xffffffffu, give, 1)) * k2;
      }
      const int64_t v = v0 + u * 8 + lane / 4;
      if (v < a.V) {
        *reinterpret_cast<float2*>(f.s.scores + v * R + row0) = make_float2(s[0], s[1]);
#pragma unroll
        for (int r = 0; r < 2; ++r) merge_stat(m[r], l[r], s[r], 1.f);
      }
    }
  }
#pragma unroll
  for (int r = 0; r < 2; ++r) {
#pragma unroll
    for (int off = 4; off < 32; off <<= 1) {
      const float m2 = __shfl_xor_sync(0xffffffffu, m[r], off), l2 = __shfl_xor_sync(0xffffffffu, l[r], off);
      merge_stat(m[r], l[r], m2, l2);
    }
    if (lane < 4) warp_part[threadIdx.x / 32][row0 + r] = make_float2(m[r], l[r]);
  }
  __syncthreads();
  if (threadIdx.x < R) {
    float2 t = warp_part[0][threadIdx.x];
    for (int i = 1; i < kThreads / 32; ++i) merge_stat(t.x, t.y, warp_part[i][threadIdx.x].x, warp_part[i][threadIdx.x].y);
    f.s.part[blockIdx.x * R + threadIdx.x] = t;
  }
}

// One warp per row: its maximum and sum over the blocks, its loss.
__global__ void few_stat_kernel(Few f) {
  const SoftmaxArgs& a = f.a;
  const int r = blockIdx.x, lane = threadIdx.x;
  const int64_t t = f.t0 + r;
  const bool kept = row_kept(a.target, t);
  float m = -INFINITY, l = 0.f;
  for (int i = lane; i < f.blocks; i += 32) {
    const float2 p = f.s.part[i * kFewRows + r];
    merge_stat(m, l, p.x, p.y);
  }
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) {
    const float m2 = __shfl_xor_sync(0xffffffffu, m, off), l2 = __shfl_xor_sync(0xffffffffu, l, off);
    merge_stat(m, l, m2, l2);
  }
  const float lse2 = m + log2f(l);
  float loss2 = 0.f;  // sum q (lse - s), in units of log 2
  if (kept) {
    const int32_t* ids = a.target.ids + t * a.target.top;
    for (int k = lane; k < a.target.top; k += 32) {
      const float q = a.target.logits ? a.target.q[t * a.target.top + k] : 1.f;
      if (q != 0.f) loss2 += q * (lse2 - f.s.scores[(int64_t)ids[k] * kFewRows + r]);
    }
  }
  loss2 = warp_sum(loss2);
  if (lane == 0) {
    if (!a.target.logits && a.target.ids[t] >= a.V) atomicOr(a.target.status, kErrTarget);
    a.loss[t] = kept ? loss2 * kLn2 + (a.target.logits ? a.target.self[t] : 0.f) : 0.f;
    a.lse[t] = kept ? lse2 * kLn2 : 0.f;
    f.s.stat[2 * r] = m;
    f.s.stat[2 * r + 1] = 1.f / l;
  }
}

// Both gradients, from the scores: a tile's coefficients g_vr = b weight_r (p_vr -
// q_vr) go to shared memory, then each thread takes one slice of VEC columns of
// every TY-th item: dw_v = sum_r g_vr h_r is written, dh_r += g_vr w_v summed in registers.
constexpr int kTile = 64;
template <typename T, int VEC>
__global__ void __launch_bounds__(kThreads, 2) few_grads_kernel(Few f, int tx) {
  constexpr int R = kFewRows;
  __shared__ __align__(16) float g[kTile][R];
  __shared__ __align__(16) float red[kThreads * VEC];
  __shared__ float bw[R], mx[R], inv[R];
  __shared__ bool used[R];
  const SoftmaxArgs& a = f.a;
  const int ty_n = kThreads / tx, x = threadIdx.x % tx, y = threadIdx.x / tx;
  const int col = (blockIdx.y * tx + x) * VEC;
  const bool on = col < a.D;
  if (threadIdx.x < R) {
    const int r = threadIdx.x;
    const int64_t t = f.t0 + r;
    const bool kept = r < f.rows && row_kept(a.target, t);
    used[r] = kept;
    bw[r] = kept ? a.b * (a.weight ? a.weight[t] : 1.f) : 0.f;
    mx[r] = f.s.stat[2 * r];
    inv[r] = f.s.stat[2 * r + 1];
  }
  __syncthreads();
  float h[R][VEC], o[R][VEC];
#pragma unroll
  for (int r = 0; r < R; ++r) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) h[r][e] = o[r][e] = 0.f;
    if (on && used[r]) load_vec<T, VEC>(static_cast<const T*>(a.h) + (f.t0 + r) * a.h_stride + col, h[r]);
  }
  const T* w = static_cast<const T*>(a.w);
  for (int64_t v0 = (int64_t)blockIdx.x * kTile; v0 < a.V; v0 += (int64_t)gridDim.x * kTile) {
    const int32_t items = (int32_t)min((int64_t)kTile, a.V - v0);
    for (int i = threadIdx.x; i < items * R; i += kThreads) {
      const int r = i % R;
      g[i / R][r] = !used[r] ? 0.f : exp2f(f.s.scores[v0 * R + i] - mx[r]) * inv[r] * bw[r];
    }
    __syncthreads();
    // A warp per row takes its targets in this tile off, in the list's order where
    // two name one item.
    for (int r = threadIdx.x / 32; r < f.rows; r += kThreads / 32) {
      if (!used[r]) continue;
      const int64_t t = f.t0 + r;
      const int lane = threadIdx.x & 31;
      for (int k0 = 0; k0 < a.target.top; k0 += 32) {
        const int k = k0 + lane;
        const int64_t at = k < a.target.top ? (int64_t)a.target.ids[t * a.target.top + k] - v0 : -1;
        const bool hit = at >= 0 && at < items;
        const float q = !hit ? 0.f : a.target.logits ? a.target.q[t * a.target.top + k] : 1.f;
        for (unsigned left = __ballot_sync(0xffffffffu, hit); left != 0u; left &= left - 1u) {
          if (lane == __ffs(left) - 1) g[at][r] -= q * bw[r];
          __syncwarp();
        }
      }
    }
    __syncthreads();
    if (on)
      for (int i = y; i < items; i += ty_n) {
        float x4[VEC], dw[VEC];
        load_vec<T, VEC>(w + (v0 + i) * a.w_stride + col, x4);
        const int64_t at = (v0 + i) * a.D + col;
#pragma unroll
        for (int e = 0; e < VEC; ++e) dw[e] = f.first ? 0.f : f.s.dw[at + e];
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const float c = g[i][r];
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            o[r][e] = fmaf(c, x4[e], o[r][e]);
            dw[e] = fmaf(c, h[r][e], dw[e]);
          }
        }
        if (f.last)
          store_vec<T, VEC>(static_cast<T*>(a.grad_w) + at, dw);
        else
          for (int e = 0; e < VEC; ++e) f.s.dw[at + e] = dw[e];
      }
    __syncthreads();
  }
#pragma unroll 1
  for (int r = 0; r < R; ++r) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      float out = 0.f;
#pragma unroll
      for (int k = 0; k < R; ++k) out = k == r ? o[k][e] : out;
      red[threadIdx.x * VEC + e] = out;
    }
    __syncthreads();
    if (y == 0 && on)
      for (int e = 0; e < VEC; ++e) {
        float sum = 0.f;
        for (int k = 0; k < ty_n; ++k) sum += red[(k * tx + x) * VEC + e];
        f.s.dh[((int64_t)blockIdx.x * R + r) * a.D + col + e] = sum;
      }
    __syncthreads();
  }
}

// dh of the group: the blocks' sums in the order of the blocks.
template <typename T>
__global__ void few_finish_kernel(Few f, int blocks) {
  const int r = blockIdx.y, d = blockIdx.x * blockDim.x + threadIdx.x;
  if (d >= f.a.D) return;
  float sum = 0.f;
#pragma unroll 8
  for (int i = 0; i < blocks; ++i) sum += f.s.dh[((int64_t)i * kFewRows + r) * f.a.D + d];
  static_cast<T*>(f.a.grad_h)[(f.t0 + r) * f.a.D + d] = from_float<T>(sum);
}

// The widest vector of values that rows of W (and of the gradients, and H) can be read by.
template <typename T>
int vector_of(const void* p, int64_t stride, int32_t D, int most) {
  for (int v = most; v > 1; v /= 2)
    if (D % v == 0 && stride % v == 0 && reinterpret_cast<uintptr_t>(p) % (v * sizeof(T)) == 0) return v;
  return 1;
}

template <typename T, int VEC>
void scores(const Few& f) {
  const int32_t slices = (f.a.D + VEC - 1) / VEC;
  few_scores_kernel<T, VEC><<<f.blocks, kThreads, sizeof(float) * slices * kFewRows * VEC, f.a.st>>>(f);
}
template <typename T, int VEC>
int grads(const Few& f) {
  const int32_t slices = (f.a.D + VEC - 1) / VEC;
  int tx = 1;
  while (tx < slices && tx < kThreads) tx *= 2;
  const int gx = (int)std::min<int64_t>(f.blocks, (f.a.V + kTile - 1) / kTile);
  few_grads_kernel<T, VEC><<<dim3(gx, (slices + tx - 1) / tx), kThreads, 0, f.a.st>>>(f, tx);
  return gx;
}

template <typename T>
cudaError_t run(const SoftmaxArgs& a, const FewScratch& s) {
  constexpr int kWide = 16 / sizeof(T);
  const int vw = vector_of<T>(a.w, a.w_stride, a.D, kWide);
  const int vg = std::min(std::min(vw, 4), std::min(vector_of<T>(a.h, a.h_stride, a.D, 4), vector_of<T>(a.grad_w, a.D, a.D, 4)));
  for (int64_t t0 = 0; t0 < a.n; t0 += kFewRows) {
    Few f{a, s, t0, (int32_t)std::min<int64_t>(kFewRows, a.n - t0), few_blocks(a.sms), t0 == 0, t0 + kFewRows >= a.n};
    if (vw == kWide) scores<T, kWide>(f);
    else if (vw >= 4) scores<T, 4>(f);
    else scores<T, 1>(f);
    few_stat_kernel<<<f.rows, 32, 0, a.st>>>(f);
    if (!a.grad_h) continue;
    const int gx = vg == 4 ? grads<T, 4>(f) : grads<T, 1>(f);
    few_finish_kernel<T><<<dim3((a.D + 127) / 128, f.rows), 128, 0, a.st>>>(f, gx);
  }
  return cudaGetLastError();
}

}  // namespace

int few_blocks(int sms) { return 2 * sms; }

cudaError_t launch_targets(const TargetArgs& a, cudaStream_t st) {
  targets_kernel<<<(unsigned)((a.n + 7) / 8), 256, 0, st>>>(a);
  return cudaGetLastError();
}

cudaError_t launch_few_rows(const SoftmaxArgs& a, const FewScratch& s) {
  if (a.dtype == ESSPT_BF16) return run<__nv_bfloat16>(a, s);
  if (a.dtype == ESSPT_F16) return run<__half>(a, s);
  return run<float>(a, s);
}

}  // namespace esspt
