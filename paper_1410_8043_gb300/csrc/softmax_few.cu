// Softmax operators for a few rows (single users, single tokens) and for small
// problems, where launches and latency count: the scores of groups of kFewRows rows
// are kept, W is read once for them and once for dh.  All in fp32.
//
// 1M items, K = 64, fp32, eight rows, GB300: scores that are kept 63 us (288 MB, 4.5 TB/s:
// loads in flight), dw 98 (320 MB, 3.3 TB/s), dh 94 (288 MB, 3.1 TB/s), where 256 MB are 38
// us.  A single row's scores without gradients: a call of 49 us in fp32 and 33 in bf16,
// where the kernel for eight rows takes 64 and 55.
#include <algorithm>

#include "ptx.cuh"
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
  float* shares = a.q + t * a.top;
  for (int k0 = 0; k0 < a.top; k0 += 32) {
    const int k = k0 + lane;
    float q = 0.f;
    if (k < a.top && present && (uint32_t)ids[k] < (uint32_t)a.V) {
      const float d = (z[k] - m) * scale;
      q = exp2f(d) / l;
      if (q != 0.f) self += q * (d - log2_l);  // (NaN takes part)
    }
    if (k < a.top) shares[k] = q;
    if (!a.again) continue;
    const int32_t id = q != 0.f ? ids[k] : -1;
    bool again = (__match_any_sync(0xffffffffu, id) & ((1u << lane) - 1u)) != 0u;
    for (int j0 = 0; j0 < k0; j0 += 32) {
      const int32_t before = shares[j0 + lane] != 0.f ? ids[j0 + lane] : -1;
      for (int j = 0; j < 32; ++j) again |= __shfl_sync(0xffffffffu, before, j) == id;
    }
    if (k < a.top) a.again[t * a.top + k] = again && id >= 0;
  }
  self = warp_sum(self);
  if (lane == 0) a.self[t] = present ? self * kLn2 : kIgnored;
}

struct Few {
  SoftmaxArgs a;
  FewScratch s;
  int32_t groups;  // of kFewRows rows
  int32_t blocks;  // per group, of the kernel whose partial results are read
  int store;       // whether scores are kept: gradients and long lists want them
};

// One warp per row: its maximum and sum over the blocks, its loss.  Other blocks wrote
// what it reads (past L1).
template <typename T>
__device__ void few_loss(const Few& f, int group, int r) {
  const SoftmaxArgs& a = f.a;
  const int lane = threadIdx.x & 31;
  const int64_t t = (int64_t)group * kFewRows + r;
  if (t >= a.n) return;
  const bool kept = row_kept(a.target, t);
  float m = -INFINITY, l = 0.f;
  for (int i = lane; i < gridDim.x; i += 32) {
    const float2 p = __ldcg(f.s.part + (group * gridDim.x + i) * kFewRows + r);
    merge_stat(m, l, p.x, p.y);
  }
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) {
    const float m2 = __shfl_xor_sync(0xffffffffu, m, off), l2 = __shfl_xor_sync(0xffffffffu, l, off);
    merge_stat(m, l, m2, l2);
  }
  const float lse2 = m + log2f(l);
  float loss2 = 0.f;  // sum q (lse - s), in units of log 2
  const int32_t* ids = a.target.ids + t * a.target.top;
  if (kept && f.store) {
    for (int k = lane; k < a.target.top; k += 32) {
      const float q = a.target.logits ? a.target.q[t * a.target.top + k] : 1.f;
      if (q != 0.f) loss2 += q * (lse2 - __ldcg(f.s.scores + ((int64_t)group * a.V + ids[k]) * kFewRows + r));
    }
  } else if (kept) {
    for (int k = 0; k < a.target.top; ++k) {
      const float q = a.target.logits ? a.target.q[t * a.target.top + k] : 1.f;
      if (q == 0.f) continue;
      const T *h = static_cast<const T*>(a.h) + t * a.h_stride, *w = static_cast<const T*>(a.w) + ids[k] * a.w_stride;
      float s = 0.f;
      for (int d = lane; d < a.D; d += 32) s = fmaf(to_float(w[d]), to_float(h[d]), s);
      s = warp_sum(s);
      if (lane == 0) loss2 += q * (lse2 - s * (a.b * kLog2e));
    }
  }
  loss2 = warp_sum(loss2);
  if (lane == 0) {
    if (!a.target.logits && a.target.ids[t] >= a.V) atomicOr(a.target.status, kErrTarget);
    a.loss[t] = kept ? loss2 * kLn2 + (a.target.logits ? a.target.self[t] : 0.f) : 0.f;
    a.lse[t] = kept ? lse2 * kLn2 : 0.f;
    f.s.stat[2 * t] = m;
    f.s.stat[2 * t + 1] = 1.f / l;
  }
}

// Scores of all items: four lanes to an item (each a quarter of its slices of VEC
// values), eight items to a warp side by side, U deep; rows of H from shared memory, where
// the four lanes read one 64-byte line for all items.  The lanes' sums meet by
// halving: each lane ends with two rows' totals, so no exponential is taken twice.
// A single row (R = 1) has its four lanes' sums in all of them, and each lane keeps
// every fourth item.
template <typename T, int VEC, int U, int R, bool SINGLE>
__global__ void __launch_bounds__(kThreads, U == 1 || SINGLE ? 2 : 4) few_scores_kernel(Few f) {
  constexpr int kDeep = U == 1 ? 8 : VEC == 8 ? 1 : 2;  // slices under way
  constexpr int kMine = R == 1 ? 1 : 2;                 // rows of a lane's statistics
  extern __shared__ __align__(16) float hs[];           // [R][slices][VEC]
  __shared__ float2 warp_part[kThreads / 32][R];
  const SoftmaxArgs& a = f.a;
  const int lane = threadIdx.x & 31, ql = lane & 3;
  const int32_t slices = (a.D + VEC - 1) / VEC;
  const T* h = static_cast<const T*>(a.h);
  for (int i = threadIdx.x; i < slices * R * VEC; i += kThreads) {
    const int r = i / (slices * VEC), d = i - r * slices * VEC;
    const int64_t t = (int64_t)blockIdx.y * kFewRows + r;
    hs[i] = t < a.n && d < a.D && row_kept(a.target, t) ? to_float(h[t * a.h_stride + d]) : 0.f;
  }
  __syncthreads();
  const T* w = static_cast<const T*>(a.w);
  const float k2 = a.b * kLog2e;
  float m[kMine], l[kMine];
#pragma unroll
  for (int r = 0; r < kMine; ++r) m[r] = -INFINITY, l[r] = 0.f;
  const int row0 = R == 1 ? 0 : (lane & 2) * 2 + (lane & 1) * 2;  // this lane's rows after halving: row0, row0 + 1
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
#pragma unroll(kDeep)
    for (int i = ql; i < slices; i += 4) {
      float x[U][VEC];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if constexpr (SINGLE) {
#pragma unroll
          for (int e = 0; e < VEC; ++e) x[u][e] = i * VEC + e < a.D ? to_float(row[u][i * VEC + e]) : 0.f;
        } else {
          load_vec<T, VEC>(row[u] + i * VEC, x[u]);
        }
      }
      const float* hv = hs + i * VEC;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float y[VEC];
#pragma unroll
        for (int e = 0; e < VEC; e += 4) {
          const float4 q = *reinterpret_cast<const float4*>(hv + r * slices * VEC + e);
          y[e] = q.x, y[e + 1] = q.y, y[e + 2] = q.z, y[e + 3] = q.w;
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int e = 0; e < VEC; ++e) acc[u][r] = fmaf(x[u][e], y[e], acc[u][r]);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t v = v0 + u * 8 + lane / 4;
      float* kept = f.s.scores + ((int64_t)blockIdx.y * a.V + v) * kFewRows;
      if constexpr (R == 1) {
        float s = acc[u][0] + __shfl_xor_sync(0xffffffffu, acc[u][0], 2);
        s = (s + __shfl_xor_sync(0xffffffffu, s, 1)) * k2;
        if (v < a.V && ql == u % 4) {
          if (f.store) kept[0] = s;
          merge_stat(m[0], l[0], s, 1.f);
        }
      } else {
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
        if (v < a.V) {
          if (f.store) *reinterpret_cast<float2*>(kept + row0) = make_float2(s[0], s[1]);
#pragma unroll
          for (int r = 0; r < 2; ++r) merge_stat(m[r], l[r], s[r], 1.f);
        }
      }
    }
  }
#pragma unroll
  for (int r = 0; r < kMine; ++r) {
#pragma unroll
    for (int off = R == 1 ? 1 : 4; off < 32; off <<= 1) {
      const float m2 = __shfl_xor_sync(0xffffffffu, m[r], off), l2 = __shfl_xor_sync(0xffffffffu, l[r], off);
      merge_stat(m[r], l[r], m2, l2);
    }
    if (lane < (R == 1 ? 1 : 4)) warp_part[threadIdx.x / 32][row0 + r] = make_float2(m[r], l[r]);
  }
  __syncthreads();
  if (threadIdx.x < R) {
    float2 t = warp_part[0][threadIdx.x];
    for (int i = 1; i < kThreads / 32; ++i) merge_stat(t.x, t.y, warp_part[i][threadIdx.x].x, warp_part[i][threadIdx.x].y);
    f.s.part[(blockIdx.y * gridDim.x + blockIdx.x) * kFewRows + threadIdx.x] = t;
  }
  // The block of a group that ends last goes on with its rows' losses: a launch less.
  __shared__ bool last;
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    last = atomicAdd(f.s.done + blockIdx.y, 1u) == gridDim.x - 1;
    __threadfence();
  }
  __syncthreads();
  if (!last) return;
  for (int r = threadIdx.x / 32; r < R; r += kThreads / 32) few_loss<T>(f, blockIdx.y, r);
  if (threadIdx.x == 0) f.s.done[blockIdx.y] = 0u;
}

// Four columns of a row per thread: side by side, or (SPREAD, rows that no vector of
// four can be read from) one of each of four groups of tx, so that a warp's loads join.
constexpr int kCols = 4;
template <bool SPREAD>
__device__ __forceinline__ int first_col(int chunk, int x, int tx) {
  return SPREAD ? chunk * kCols * tx + x : (chunk * tx + x) * kCols;
}
template <typename T, bool SPREAD>
__device__ __forceinline__ void load_cols(const T* row, int col, int tx, int D, float (&x)[kCols]) {
  if constexpr (SPREAD) {
#pragma unroll
    for (int e = 0; e < kCols; ++e) x[e] = col + e * tx < D ? to_float(row[col + e * tx]) : 0.f;
  } else {
    load_vec<T, kCols>(row + col, x);
  }
}
template <typename T, bool SPREAD>
__device__ __forceinline__ void store_cols(T* row, int col, int tx, int D, const float (&x)[kCols]) {
  if constexpr (SPREAD) {
#pragma unroll
    for (int e = 0; e < kCols; ++e)
      if (col + e * tx < D) row[col + e * tx] = from_float<T>(x[e]);
  } else {
    store_vec<T, kCols>(row + col, x);
  }
}

// dw_v = sum_r g_vr h_r, with g_vr = b weight_r (p_vr - q_vr) taken from the scores of
// a tile of items for all rows at once, and left in their place for dh.  Threads take
// four columns (tx threads to a row) of every ty-th item, four items deep.
template <typename T, bool SPREAD, int kTile>
__global__ void __launch_bounds__(kThreads, SPREAD ? 2 : 3) few_grad_w_kernel(Few f, int tx) {
  constexpr int R = kFewRows, U = SPREAD ? 2 : 4, VEC = kCols;
  extern __shared__ __align__(32) float g[];  // [groups][kTile][R]
  __shared__ __align__(16) float red[kTile == 8 ? kThreads * VEC : 1];
  __shared__ float bw[kSmallRows], mx[kSmallRows], inv[kSmallRows];
  __shared__ bool used[kSmallRows];
  const SoftmaxArgs& a = f.a;
  const int n = (int)a.n, ty_n = kThreads / tx, x = threadIdx.x % tx, y = threadIdx.x / tx, lane = threadIdx.x & 31;
  int span = 1;  // lanes to a row's targets
  while (span < a.target.top && span < 32) span *= 2;
  for (int t = threadIdx.x; t < f.groups * R; t += kThreads) {
    const bool kept = t < n && row_kept(a.target, t);
    used[t] = kept;
    bw[t] = kept ? a.b * (a.weight ? a.weight[t] : 1.f) : 0.f;
    mx[t] = t < n ? f.s.stat[2 * t] : 0.f;
    inv[t] = t < n ? f.s.stat[2 * t + 1] : 0.f;
  }
  __syncthreads();
  for (int64_t v0 = (int64_t)blockIdx.x * kTile; v0 < a.V; v0 += (int64_t)gridDim.x * kTile) {
    const int32_t items = (int32_t)min((int64_t)kTile, a.V - v0);
#pragma unroll 4
    for (int i = threadIdx.x; i < f.groups * items * R; i += kThreads) {
      const int group = i / (items * R), in = i - group * items * R, t = group * R + in % R;
      const float s = f.s.scores[((int64_t)group * a.V + v0) * R + in];
      g[group * kTile * R + in] = !used[t] ? 0.f : exp2f(s - mx[t]) * inv[t] * bw[t];
    }
    __syncthreads();
    // Rows' targets in this tile come off, `span` lanes to a row, in the list's order
    // where two entries name one item.
    for (int t0 = threadIdx.x / 32 * (32 / span); t0 < n; t0 += kThreads / span) {
      const int t = t0 + lane / span;
      for (int k0 = 0; k0 < a.target.top; k0 += span) {
        const int k = k0 + lane % span;
        const int64_t e = (int64_t)t * a.target.top + k;
        const int64_t at = t < n && used[t] && k < a.target.top ? (int64_t)a.target.ids[e] - v0 : -1;
        const bool hit = at >= 0 && at < items;
        const float q = !hit ? 0.f : a.target.logits ? a.target.q[e] : 1.f;
        for (unsigned left = __ballot_sync(0xffffffffu, hit); left != 0u; left &= left - 1u) {
          if (lane == __ffs(left) - 1) g[(t / R * kTile + at) * R + t % R] -= q * bw[t];
          __syncwarp();
        }
      }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < f.groups * items * R; i += kThreads) {
      const int group = i / (items * R), in = i - group * items * R;
      f.s.scores[((int64_t)group * a.V + v0) * R + in] = g[group * kTile * R + in];
    }
    for (int chunk = 0; chunk * tx * VEC < a.D; ++chunk) {
      const int col = first_col<SPREAD>(chunk, x, tx);
      float h[R][VEC];
      auto load_rows = [&](int group) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
#pragma unroll
          for (int e = 0; e < VEC; ++e) h[r][e] = 0.f;
          if (used[group * R + r])
            load_cols<T, SPREAD>(static_cast<const T*>(a.h) + (group * R + r) * a.h_stride, col, tx, a.D, h[r]);
        }
      };
      auto add = [&](int group, int item, float (&dw)[VEC]) {
        float c[R];
        load_vec<float, R>(g + (group * kTile + item) * R, c);
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int e = 0; e < VEC; ++e) dw[e] = fmaf(c[r], h[r][e], dw[e]);
      };
      if constexpr (kTile == 8) {
        // Threads past the tile's items take a share of the groups each; the shares meet
        // in shared memory (97 rows, 1000 items, K = 16, fp32: 6 us, where eight
        // threads to an item took all groups in turn 14).
        const int shares = max(1, ty_n / kTile), share = shares > 1 ? y / kTile : 0;
        for (int i = shares > 1 ? y % kTile : y; i < kTile; i += shares > 1 ? kTile : ty_n) {
          float dw[VEC] = {};
          if (col < a.D && i < items)
            for (int group = share; group < f.groups; group += shares) {
              load_rows(group);
              add(group, i, dw);
            }
          if (shares > 1) {  // (all threads come here once)
            store_vec<float, VEC>(red + threadIdx.x * VEC, dw);
            __syncthreads();
            for (int k = 1; share == 0 && k < shares; ++k)
#pragma unroll
              for (int e = 0; e < VEC; ++e) dw[e] += red[(threadIdx.x + k * kTile * tx) * VEC + e];
            __syncthreads();
          }
          if (share == 0 && col < a.D && i < items)
            store_cols<T, SPREAD>(static_cast<T*>(a.grad_w) + (v0 + i) * a.D, col, tx, a.D, dw);
        }
        continue;
      }
      if (col >= a.D) break;
      if (f.groups == 1) load_rows(0);
      for (int i0 = y; i0 < items; i0 += ty_n * U) {
        float dw[U][VEC] = {};
        for (int group = 0; group < f.groups; ++group) {
          if (f.groups > 1) load_rows(group);
#pragma unroll
          for (int u = 0; u < U; ++u) add(group, min(i0 + u * ty_n, items - 1), dw[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (i0 + u * ty_n < items)
            store_cols<T, SPREAD>(static_cast<T*>(a.grad_w) + (v0 + i0 + u * ty_n) * a.D, col, tx, a.D, dw[u]);
      }
    }
    __syncthreads();
  }
}

// dh_r = sum_v g_vr w_v of a group of rows (blockIdx.z) by blocks, each over a part of
// the items: threads as above, coefficients by tiles through shared memory, the rows'
// sums in registers.
template <typename T, bool SPREAD>
__global__ void __launch_bounds__(kThreads, SPREAD ? 2 : 3) few_grad_h_kernel(Few f, int tx) {
  constexpr int R = kFewRows, VEC = kCols, U = SPREAD ? 4 : 8, kTile = 256;
  __shared__ __align__(32) float tiles[2][kTile * R];
  const SoftmaxArgs& a = f.a;
  const int ty_n = kThreads / tx, x = threadIdx.x % tx, y = threadIdx.x / tx;
  const int col = first_col<SPREAD>(blockIdx.y, x, tx);
  const bool on = col < a.D;
  const float* g = f.s.scores + (int64_t)blockIdx.z * a.V * R;
  const T* w = static_cast<const T*>(a.w);
  float o[R][VEC];
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int e = 0; e < VEC; ++e) o[r][e] = 0.f;
  const int64_t end = a.V * (int64_t)(blockIdx.x + 1) / gridDim.x;
  auto fetch = [&](float* to, int64_t v) {  // coefficients of a tile, while the one before is at work
    const int quads = (int)min((int64_t)kTile, end - v) * (R / 4);
    for (int i = threadIdx.x; i < quads; i += kThreads) cp_async16_if(to + 4 * i, g + v * R + 4 * i, true);
    cp_async_commit();
  };
  int64_t v0 = a.V * (int64_t)blockIdx.x / gridDim.x;
  fetch(tiles[0], v0);
  for (int turn = 0; v0 < end; v0 += kTile, turn ^= 1) {
    const int items = (int)min((int64_t)kTile, end - v0);
    const float* c = tiles[turn];
    cp_async_wait_all();
    __syncthreads();
    if (v0 + kTile < end) fetch(tiles[turn ^ 1], v0 + kTile);
    if (on)
      for (int i = y; i < items; i += U * ty_n) {
        float k[U][VEC];
#pragma unroll
        for (int u = 0; u < U; ++u) load_cols<T, SPREAD>(w + (v0 + min(i + u * ty_n, items - 1)) * a.w_stride, col, tx, a.D, k[u]);
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (i + u * ty_n >= items) break;
          float cu[R];
          load_vec<float, R>(c + (i + u * ty_n) * R, cu);
#pragma unroll
          for (int r = 0; r < R; ++r)
#pragma unroll
            for (int e = 0; e < VEC; ++e) o[r][e] = fmaf(cu[r], k[u][e], o[r][e]);
        }
      }
  }
  // Sums meet in the warp where it holds several items' threads, then in shared memory,
  // four rows at a time (97 rows, 1000 items, K = 16, fp32: 6.5 us, by shared memory alone 18.6).
  const int parts = tx < 32 ? kThreads / 32 : ty_n, part = tx < 32 ? threadIdx.x / 32 : y;
  float* red = tiles[0];  // [parts][4][tx * VEC]
  static_assert(4 * kThreads * VEC <= 2 * kTile * R, "sums outgrow the tiles");
#pragma unroll
  for (int r0 = 0; r0 < R; r0 += 4) {
    __syncthreads();
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        float v = o[r0 + r][e];
        for (int to = tx; to < 32; to *= 2) v += __shfl_xor_sync(0xffffffffu, v, to);
        if (tx >= 32 || (threadIdx.x & 31) < tx) red[((part * 4 + r) * VEC + e) * tx + x] = v;
      }
    __syncthreads();
    for (int i = threadIdx.x; i < 4 * VEC * tx; i += kThreads) {
      const int r = i / (VEC * tx), e = i / tx % VEC, d = first_col<SPREAD>(blockIdx.y, i % tx, tx) + e * (SPREAD ? tx : 1);
      float sum = 0.f;
      for (int k = 0; k < parts; ++k) sum += red[k * 4 * VEC * tx + i];
      if (d < a.D) f.s.dh[((int64_t)(blockIdx.z * gridDim.x + blockIdx.x) * R + r0 + r) * a.D + d] = sum;
    }
  }
}

// dh: the blocks' sums, eight parts of them side by side and then in order.
template <typename T>
__global__ void few_finish_kernel(Few f) {
  __shared__ float part[8][32];
  const int t = blockIdx.y, d = blockIdx.x * 32 + threadIdx.x;
  const float* from = f.s.dh + ((int64_t)t / kFewRows * f.blocks * kFewRows + t % kFewRows) * f.a.D + d;
  float sum = 0.f;
  if (d < f.a.D)
#pragma unroll 8
    for (int i = threadIdx.y; i < f.blocks; i += 8) sum += from[(int64_t)i * kFewRows * f.a.D];
  part[threadIdx.y][threadIdx.x] = sum;
  __syncthreads();
  if (threadIdx.y > 0 || d >= f.a.D) return;
  for (int i = 1; i < 8; ++i) sum += part[i][threadIdx.x];
  const bool kept = row_kept(f.a.target, t);
  static_cast<T*>(f.a.grad_h)[(int64_t)t * f.a.D + d] = from_float<T>(kept ? sum : 0.f);
}

// The widest vector of values that rows of W (and of the gradients, and H) can be read by.
template <typename T>
int vector_of(const void* p, int64_t stride, int32_t D, int most) {
  for (int v = most; v > 1; v /= 2)
    if (D % v == 0 && stride % v == 0 && reinterpret_cast<uintptr_t>(p) % (v * sizeof(T)) == 0) return v;
  return 1;
}

// Warps take 8 items at a time where that gives the GPU few warps, else 16 (of a single
// row 32).
template <typename T, int VEC, bool SINGLE>
void scores(Few& f) {
  const int32_t slices = (f.a.D + VEC - 1) / VEC;
  const bool one = f.a.n == 1;
  const size_t smem = sizeof(float) * slices * (one ? 1 : kFewRows) * VEC;
  const int64_t most = std::max(1, few_blocks(f.a.sms) / f.groups);
  const int many = one ? 256 : 128, take = (int64_t)f.a.V < most * many ? 64 : many;  // items of a block at a time
  f.blocks = (int)std::min<int64_t>(most, ((int64_t)f.a.V + take - 1) / take);
  const dim3 grid(f.blocks, f.groups);
  if (one && take == 64) few_scores_kernel<T, VEC, 1, 1, SINGLE><<<grid, kThreads, smem, f.a.st>>>(f);
  else if (one) few_scores_kernel<T, VEC, 4, 1, SINGLE><<<grid, kThreads, smem, f.a.st>>>(f);
  else if (take == 64) few_scores_kernel<T, VEC, 1, kFewRows, SINGLE><<<grid, kThreads, smem, f.a.st>>>(f);
  else few_scores_kernel<T, VEC, 2, kFewRows, SINGLE><<<grid, kThreads, smem, f.a.st>>>(f);
}
template <typename T, bool SPREAD>
void grads(Few f) {
  const int32_t slices = (f.a.D + kCols - 1) / kCols;
  int tx = 1;
  while (tx < slices && tx < 64) tx *= 2;
  // Tiles of 8 items where there are few, of 256 where a few rows meet many, else of 64.
  const int kTile = (int64_t)f.a.V < 64 * f.a.sms ? 8 : f.groups == 1 && (int64_t)f.a.V >= 1024 * f.a.sms ? 256 : 64;
  const int64_t tiles = ((int64_t)f.a.V + kTile - 1) / kTile;
  const size_t smem = sizeof(float) * f.groups * kTile * kFewRows;
  const unsigned grid = (unsigned)std::min<int64_t>(tiles, (SPREAD ? 2 : 3) * f.a.sms);  // (what is resident at once)
  if (kTile == 8) few_grad_w_kernel<T, SPREAD, 8><<<grid, kThreads, smem, f.a.st>>>(f, tx);
  else if (kTile == 256) few_grad_w_kernel<T, SPREAD, 256><<<grid, kThreads, smem, f.a.st>>>(f, tx);
  else few_grad_w_kernel<T, SPREAD, 64><<<grid, kThreads, smem, f.a.st>>>(f, tx);
  // Blocks of a group: as many as fill the GPU, each with 4 items per thread at least.
  const int64_t most = ((int64_t)f.a.V * tx + 4 * kThreads - 1) / (4 * kThreads);
  f.blocks = (int)std::min<int64_t>(std::max(1, (SPREAD ? 2 : 3) * f.a.sms / f.groups), most);
  few_grad_h_kernel<T, SPREAD><<<dim3(f.blocks, (slices + tx - 1) / tx, f.groups), kThreads, 0, f.a.st>>>(f, tx);
  few_finish_kernel<T><<<dim3((f.a.D + 31) / 32, (unsigned)f.a.n), dim3(32, 8), 0, f.a.st>>>(f);
}

template <typename T>
cudaError_t run(const SoftmaxArgs& a, const FewScratch& s) {
  constexpr int kWide = 16 / sizeof(T);
  const int vw = vector_of<T>(a.w, a.w_stride, a.D, kWide);
  const int vg = std::min(std::min(vw, 4), std::min(vector_of<T>(a.h, a.h_stride, a.D, 4), vector_of<T>(a.grad_w, a.D, a.D, 4)));
  Few f{a, s, (int32_t)((a.n + kFewRows - 1) / kFewRows), 0, a.grad_h || a.target.top > 4};
  if (vw == kWide) scores<T, kWide, false>(f);
  else if (vw >= 4) scores<T, 4, false>(f);
  else scores<T, kWide, true>(f);
  if (a.grad_h) vg == 4 ? grads<T, false>(f) : grads<T, true>(f);
  return cudaGetLastError();
}

}  // namespace

int few_blocks(int sms) { return 4 * sms; }

// By what both ways take, in us, fitted to 12 to 128 rows on 1000 to 800k items of 4 to
// 500 values (fp32 and bf16, with gradients and without), the tensor cores' by type, and
// 2^24 scores kept at most.  Where they part, here and by tensor cores, with gradients:
// 200k items, K = 64, fp32 42 rows 281 and 252, bf16 25 rows 177 and 171; K = 256, fp32 35
// rows 662 and 650, bf16 23 rows 430 and 358.  Forward: 200k, K = 64, fp32 48 rows 70 and
// 70, bf16 32 rows 43 and 43.
bool few_rows(int64_t n, int64_t V, int32_t D, int32_t dtype, bool grads) {
  if (n <= kFewRows || n > kSmallRows) return n <= kFewRows;
  if (n * V > (1 << 24)) return false;
  const double items = (double)V, scores = n * items;
  const double few = grads ? 34 + items * (1.8e-4 + 3.5e-7 * D) + scores * (6.8e-6 + 2.4e-7 * D) : 10 + scores * (1e-6 + 8e-8 * D);
  const double type = dtype == ESSPT_F32 ? grads ? 1.26 : 1.18 : grads ? 0.9 : 0.85;
  return few <= type * (grads ? 88 + items * (2e-4 + 6.3e-6 * D) : 36 + items * (5e-5 + 1e-6 * D));
}
int few_groups(int64_t max_rows, int64_t V, int32_t D, int32_t dtype, bool backward) {
  int64_t n = std::min<int64_t>(max_rows, kSmallRows);
  while (!few_rows(n, V, D, dtype, false) && !(backward && few_rows(n, V, D, dtype, true))) --n;
  return (int)((n + kFewRows - 1) / kFewRows);
}

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
