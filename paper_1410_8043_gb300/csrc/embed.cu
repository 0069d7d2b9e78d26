// Embedding lookup with scaling, and its gradient by sorted tokens: kernels and C-ABI.
#include <cmath>
#include <new>
#include <type_traits>

#include "chained.cuh"
#include "operator.h"
#include "ptx.cuh"
#include "rows.cuh"

using namespace esspt;

struct esspt_embed {
  esspt_embed_config cfg{};
  cudaStream_t st = nullptr;
  char* base = nullptr;
  cudaStream_t side = nullptr;  // gradients are set to zero there, beside the sort
  cudaEvent_t fork = nullptr, join = nullptr;
  Errors err;
};

namespace {

constexpr uint32_t kErrId = 1u;
constexpr int kThreads = 256;

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

// Loads that a thread has under way: 64 bytes, or eight of them.
template <typename T, int VEC>
constexpr int kDeep = VEC * sizeof(T) >= 16 ? 4 : 8;

// A block takes kThreads * kDeep vectors of the result, one behind the other, whatever rows they are of.  Memory is the bound of
// wide rows (60000 of 1000 fp32 values: 69 us, 7 TB/s), latency and issue of short ones: 262147 rows of 64 out of a million take
// 16 us for 88 MB, with DRAM at 22% and issue at 57%, and a thread asks for an id only when the one before it is there.  PAIRS: rows
// of an odd number of 16-bit values, of which two of the result, from one row or two, make a word to write.  (60000 rows of
// 1001 bf16 values: 146 us value by value.)
template <typename T, int VEC, bool PAIRS>
__global__ void __launch_bounds__(kThreads) lookup_kernel(Lookup a) {
  constexpr int kMany = kDeep<T, VEC>, kEach = PAIRS ? 2 : VEC;
  const int64_t first = (int64_t)blockIdx.x * (kThreads * kMany), all = PAIRS ? (a.n * a.D + 1) / 2 : a.n * a.per_row;
  const int64_t row0 = (PAIRS ? 2 * first : first) / a.per_row;
  const uint32_t rest = (uint32_t)((PAIRS ? 2 * first : first) - row0 * a.per_row);
  const T* w = static_cast<const T*>(a.w);
  T* out = static_cast<T*>(a.out);
  const float inv = 1.f / (float)a.per_row;
  auto row_of = [&](uint32_t row) -> const T* {  // null: padding, or behind the last
    const int32_t id = row0 + row < a.n ? a.ids[row0 + row] : -1;
    if (id >= a.V) atomicOr(a.status, kErrId);
    return (uint32_t)id < (uint32_t)a.V ? w + id * a.w_stride : nullptr;
  };
  float x[kMany][kEach];
#pragma unroll
  for (int k = 0; k < kMany; ++k) {
    const uint32_t at = rest + (k * kThreads + threadIdx.x) * (PAIRS ? 2 : 1);
    uint32_t row = (uint32_t)((float)at * inv);  // (of numbers below 2^14: off by one at most)
    int32_t col = (int32_t)(at - row * a.per_row);
    if (col < 0) --row, col += a.per_row;
    if (col >= a.per_row) ++row, col -= a.per_row;
#pragma unroll
    for (int i = 0; i < kEach; ++i) x[k][i] = 0.f;
    if (first + k * kThreads + threadIdx.x >= all) continue;
    if constexpr (PAIRS) {
      const T* from = row_of(row);
      if (from) x[k][0] = to_float(from[col]);
      if (++col == a.per_row) from = row_of(row + 1), col = 0;
      if (from) x[k][1] = to_float(from[col]);
    } else {
      const int32_t id = a.ids[row0 + row];
      if (id >= a.V) atomicOr(a.status, kErrId);
      if ((uint32_t)id < (uint32_t)a.V) load_vec<T, VEC>(w + id * a.w_stride + col * VEC, x[k]);
    }
  }
#pragma unroll
  for (int k = 0; k < kMany; ++k) {
    const int64_t at = first + k * kThreads + threadIdx.x;
    if (at >= all) break;
#pragma unroll
    for (int i = 0; i < kEach; ++i) x[k][i] *= a.scale;
    if (PAIRS && 2 * at + 1 == a.n * a.D)
      out[2 * at] = from_float<T>(x[k][0]);
    else
      store_vec<T, kEach>(out + at * kEach, x[k]);
  }
}

// ---- the gradient of few tokens: one kernel --------------------------------------------------------------------
//
// A block owns a range of the table's rows, of a tile of columns.  It reads all ids, keeps the tokens of its
// rows, sorts them by row and place in shared memory, and sums them: a row's tokens by one group of lanes, or
// by all groups in turn where there are more than kLong.  One launch, no scratch memory; the block of the most popular row
// bounds it (8195 tokens of 100 fp32 values, some 500 of them one row's: 19 us, of which a quarter each are the ids, the sort and
// that row's sum; 97 tokens of 16: 4 us).
struct Gradient {
  const int32_t* ids;
  const void* grad;
  int64_t grad_stride;
  int64_t n;
  int32_t V, D, per_row;  // per_row: vectors of a row
  int32_t lanes;          // of a group: a power of two
  float scale;
  int accumulate;
  void* out;
  uint32_t* status;
  uint2* pairs;           // (row, place) of the tokens, sorted
  float* part;            // [blocks][2][D]
  int32_t rows, place_bits;  // (few tokens) rows of a block; bits of a place
  int32_t chunk;             // (many tokens) tokens of a group
};

constexpr int kFew = 16384;      // tokens that go this way at most
constexpr int kFewThreads = 512;
constexpr int kFewBlocks = 304;  // two for each of 152 SMs
constexpr int kLong = 32;
constexpr int kStarts = 2048;

// A vector as it stands in memory (half the registers of fp32 values for 16-bit types): 16 bytes, or one value.
template <typename T, int VEC>
using Raw = std::conditional_t<VEC == 1, T, uint4>;
template <typename T, int VEC>
__device__ __forceinline__ Raw<T, VEC> load_raw(const T* p, bool there) {  // zeros where it is not
  if constexpr (VEC == 1) {
    T r = from_float<T>(0.f);
    if (there) r = *p;
    return r;
  } else {
    uint4 r = make_uint4(0, 0, 0, 0);
    if (there) r = *reinterpret_cast<const uint4*>(p);
    return r;
  }
}
__device__ __forceinline__ float2 halves(uint32_t w, const __nv_bfloat16*) {
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
__device__ __forceinline__ float2 halves(uint32_t w, const __half*) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
template <typename T, int VEC>
__device__ __forceinline__ void to_floats(const Raw<T, VEC>& r, float (&x)[VEC]) {
  if constexpr (VEC == 1) {
    x[0] = to_float(r);
  } else if constexpr (VEC == 4) {
    x[0] = __uint_as_float(r.x), x[1] = __uint_as_float(r.y), x[2] = __uint_as_float(r.z), x[3] = __uint_as_float(r.w);
  } else {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 v = halves(w[j], (const T*)nullptr);
      x[2 * j] = v.x, x[2 * j + 1] = v.y;
    }
  }
}
template <typename T, int VEC>
__device__ __forceinline__ void add_raw(const Raw<T, VEC>& r, float (&sum)[VEC]) {
  float x[VEC];
  to_floats<T, VEC>(r, x);
#pragma unroll
  for (int j = 0; j < VEC; ++j) sum[j] += x[j];
}

// A row's columns lane + k * lanes of a tile (in vectors): what the result holds before (zeros if it is overwritten), and
// the result from that and the sums.
template <typename T, int VEC, int K>
__device__ __forceinline__ void read_old(const Gradient& a, int64_t row, int c0, Raw<T, VEC> (&old)[K]) {
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int c = c0 + k * a.lanes;
    old[k] = load_raw<T, VEC>(static_cast<const T*>(a.out) + row * a.D + c * VEC, a.accumulate && c < a.per_row);
  }
}
template <typename T, int VEC, int K>
__device__ __forceinline__ void write_zeros(const Gradient& a, int64_t row, uint32_t rows, int c0, int step) {
  T* to = static_cast<T*>(a.out) + row * a.D + c0 * VEC;
  for (uint32_t v = 0; v < rows; v += step, to += step * a.D)
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (c0 + k * a.lanes < a.per_row) {
        if constexpr (VEC * sizeof(T) == 16)
          *reinterpret_cast<uint4*>(to + k * a.lanes * VEC) = make_uint4(0, 0, 0, 0);
        else
          to[k * a.lanes] = from_float<T>(0.f);
      }
}
template <typename T, int VEC, int K>
__device__ __forceinline__ void emit(const Gradient& a, int64_t row, int c0, const float (&sum)[K][VEC], const Raw<T, VEC> (&old)[K]) {
  T* out = static_cast<T*>(a.out) + row * a.D;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int c = c0 + k * a.lanes;
    if (c >= a.per_row) break;
    float x[VEC];
    if (a.accumulate) to_floats<T, VEC>(old[k], x);
#pragma unroll
    for (int j = 0; j < VEC; ++j) x[j] = a.accumulate ? fmaf(sum[k][j], a.scale, x[j]) : sum[k][j] * a.scale;
    store_vec<T, VEC>(out + c * VEC, x);
  }
}

// Adds U tokens' rows to `sum`, one behind the other, all loads first; place[u] < 0: none.
template <typename T, int VEC, int K, int U>
__device__ __forceinline__ void add_rows(const Gradient& a, const int64_t (&place)[U], int c0, float (&sum)[K][VEC]) {
  const T* grad = static_cast<const T*>(a.grad);
  Raw<T, VEC> x[U][K];
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = c0 + k * a.lanes;
      x[u][k] = load_raw<T, VEC>(grad + place[u] * a.grad_stride + c * VEC, place[u] >= 0 && c < a.per_row);
    }
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int k = 0; k < K; ++k) add_raw<T, VEC>(x[u][k], sum[k]);
}

// Sorts up to two entries a thread, in a list with room for 4 * kFewThreads: by exchanges that get ever longer and back (bitonic), within
// a warp by shuffles, between warps through two halves of the list in turn.  (Exchanges in the list alone, with every warp at work for
// every size: 23 us for 19 of a call of 8195 tokens.)
__device__ __forceinline__ void sort_in_registers(uint32_t* list, uint32_t m, uint32_t size) {
  const uint32_t tid = threadIdx.x;
  const bool two = size > kFewThreads, live = (tid & ~31u) < size;  // (other warps have nothing but sentinels)
  uint32_t x = tid < m ? list[tid] : 0xffffffffu, y = kFewThreads + tid < m ? list[kFewThreads + tid] : 0xffffffffu;
  uint32_t half = 2 * kFewThreads;  // (the entries were in the other one)
  for (uint32_t run = 2; run <= size; run *= 2) {
    const bool up_x = (tid & run) == 0, up_y = ((kFewThreads + tid) & run) == 0;
    uint32_t dist = run / 2;
    if (dist == kFewThreads) {  // (the last run's first)
      const uint32_t low = min(x, y);
      y = max(x, y), x = low;
      dist /= 2;
    }
    for (; dist >= 32; dist /= 2) {
      if (live) list[half + tid] = x;
      if (two) list[half + kFewThreads + tid] = y;
      __syncthreads();
      const bool lower = (tid & dist) == 0;
      if (live) {
        const uint32_t other = list[half + (tid ^ dist)];
        x = lower == up_x ? min(x, other) : max(x, other);
      }
      if (two) {
        const uint32_t other = list[half + kFewThreads + (tid ^ dist)];
        y = lower == up_y ? min(y, other) : max(y, other);
      }
      half ^= 2 * kFewThreads;
    }
    if (!live) continue;
#pragma unroll 1
    for (uint32_t d = run < 32 ? run / 2 : 16; d > 0; d /= 2) {  // (a loop: unrolled, its instructions take longer to come)
      const bool lower = (tid & d) == 0;
      const uint32_t ox = __shfl_xor_sync(0xffffffffu, x, d);
      x = lower == up_x ? min(x, ox) : max(x, ox);
      if (two) {
        const uint32_t oy = __shfl_xor_sync(0xffffffffu, y, d);
        y = lower == up_y ? min(y, oy) : max(y, oy);
      }
    }
  }
  __syncthreads();
  if (tid < m) list[tid] = x;
  if (kFewThreads + tid < m) list[kFewThreads + tid] = y;
}

template <typename T, int VEC, int K>
__global__ void __launch_bounds__(kFewThreads) few_kernel(Gradient a) {
  extern __shared__ uint32_t list[];  // (row in the range, place) of the block's tokens
  __shared__ uint32_t count, n_long, longs[kFew / kLong], warp_starts[kFewThreads / 32];
  __shared__ uint16_t starts[kStarts];
  __shared__ float red[kFewThreads * K * VEC];
  constexpr int U = 8 / K;
  const int tid = threadIdx.x, lane = tid & (a.lanes - 1), group = tid / a.lanes, groups = kFewThreads / a.lanes;
  const int c0 = blockIdx.y * a.lanes * K + lane;
  const int64_t lo = (int64_t)blockIdx.x * a.rows, hi = lo + a.rows < a.V ? lo + a.rows : a.V;
  if (tid == 0) count = n_long = 0;
  __syncthreads();
  for (int base = 0; base < (int)a.n; base += kFewThreads * 8) {
    const int i0 = base + tid;
    int32_t id[8];
    uint32_t mine = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) id[k] = i0 + k * kFewThreads < (int)a.n ? a.ids[i0 + k * kFewThreads] : -1;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (id[k] >= a.V && blockIdx.x == 0) atomicOr(a.status, kErrId);
      mine += id[k] >= lo && id[k] < hi;
    }
    if (!__any_sync(0xffffffffu, mine)) continue;
    // One addition for a warp (a popular row's tokens would queue for the counter).
    uint32_t at = mine;
#pragma unroll
    for (int off = 1; off < 32; off *= 2) {
      const uint32_t x = __shfl_up_sync(0xffffffffu, at, off);
      if ((tid & 31) >= off) at += x;
    }
    uint32_t first = 0;
    if ((tid & 31) == 31) first = atomicAdd(&count, at);
    at += __shfl_sync(0xffffffffu, first, 31) - mine;
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (id[k] >= lo && id[k] < hi) list[at++] = (uint32_t)(id[k] - lo) << a.place_bits | (uint32_t)(i0 + k * kFewThreads);
  }
  if (!a.accumulate)  // rows without tokens; the others are written again below
    if (lo + group < hi) write_zeros<T, VEC, K>(a, lo + group, (uint32_t)(hi - lo - group), c0, groups);
  __syncthreads();
  const uint32_t m = count;
  if (m == 0) return;
  uint32_t size = 2;
  while (size < m) size *= 2;
  if (size <= 2 * kFewThreads) {
    sort_in_registers(list, m, size);
  } else {
    for (uint32_t i = m + tid; i < size; i += kFewThreads) list[i] = 0xffffffffu;
    for (uint32_t run = 2; run <= size; run *= 2)
      for (uint32_t dist = run / 2; dist > 0; dist /= 2) {
        __syncthreads();
        for (uint32_t t = tid; t < size / 2; t += kFewThreads) {
          const uint32_t i = 2 * t - (t & (dist - 1)), j = i + dist;
          const uint32_t x = list[i], y = list[j];
          if ((x > y) == ((i & run) == 0)) list[i] = y, list[j] = x;
        }
      }
  }
  __syncthreads();
  const uint32_t place_mask = (1u << a.place_bits) - 1;
  auto row_at = [&](uint32_t i) { return list[i] >> a.place_bits; };
  auto segment = [&](uint32_t begin, uint32_t end) {  // a row's tokens
    if (end - begin > kLong) {
      if (lane == 0) longs[atomicAdd(&n_long, 1u)] = begin | end << 16;
      return;
    }
    const int64_t row = lo + row_at(begin);
    float sum[K][VEC] = {};
    Raw<T, VEC> old[K];
    read_old<T, VEC, K>(a, row, c0, old);
    for (uint32_t at = begin; at < end; at += U) {
      int64_t place[U];
#pragma unroll
      for (int u = 0; u < U; ++u) place[u] = at + u < end ? (int64_t)(list[at + u] & place_mask) : -1;
      add_rows<T, VEC, K, U>(a, place, c0, sum);
    }
    emit<T, VEC, K>(a, row, c0, sum, old);
  };
  // Where rows begin, in order, for the groups to take in turn; past kStarts entries they look for themselves.
  if (m <= kStarts) {
    uint32_t many = 0;
    for (uint32_t base = 0; base < m; base += kFewThreads) {
      const uint32_t t = base + tid;
      const bool begins = t < m && (t == 0 || row_at(t) != row_at(t - 1));
      const uint32_t some = __ballot_sync(0xffffffffu, begins);
      if ((tid & 31) == 0) warp_starts[tid / 32] = __popc(some);
      __syncthreads();
      uint32_t before = many, all = 0;
#pragma unroll
      for (int w = 0; w < kFewThreads / 32; ++w) {
        const uint32_t c = warp_starts[w];
        before += w < tid / 32 ? c : 0;
        all += c;
      }
      if (begins) starts[before + __popc(some & ((1u << (tid & 31)) - 1))] = (uint16_t)t;
      many += all;
      __syncthreads();
    }
    for (uint32_t k = group; k < many; k += groups) segment(starts[k], k + 1 < many ? starts[k + 1] : m);
  } else {
    for (uint32_t i = group; i < m; i += groups) {
      const uint32_t row = row_at(i);
      if (i > 0 && row_at(i - 1) == row) continue;
      uint32_t end = i, left = m - i;
      while (left > 0) {
        const uint32_t half = left / 2;
        if (row_at(end + half) <= row)
          end += half + 1, left -= half + 1;
        else
          left = half;
      }
      segment(i, end);
    }
  }
  __syncthreads();
  for (uint32_t k = 0; k < n_long; ++k) {
    const uint32_t begin = longs[k] & 0xffffu, end = longs[k] >> 16, row = row_at(begin);
    float sum[K][VEC] = {};
    Raw<T, VEC> old[K];
    if (group == 0) read_old<T, VEC, K>(a, lo + row, c0, old);
    for (uint32_t at = begin + group; at < end; at += U * groups) {
      int64_t place[U];
#pragma unroll
      for (int u = 0; u < U; ++u) place[u] = at + u * groups < end ? (int64_t)(list[at + u * groups] & place_mask) : -1;
      add_rows<T, VEC, K, U>(a, place, c0, sum);
    }
#pragma unroll
    for (int q = 0; q < K * VEC; ++q) red[q * kFewThreads + tid] = sum[q / VEC][q % VEC];
    for (int s = groups / 2; s > 0; s /= 2) {
      __syncthreads();
      if (group < s)
#pragma unroll
        for (int q = 0; q < K * VEC; ++q) red[q * kFewThreads + tid] += red[q * kFewThreads + tid + s * a.lanes];
    }
    if (group == 0) {
#pragma unroll
      for (int q = 0; q < K * VEC; ++q) sum[q / VEC][q % VEC] = red[q * kFewThreads + tid];
      emit<T, VEC, K>(a, lo + row, c0, sum, old);
    }
    __syncthreads();
  }
}

// ---- many tokens: sorted by row and place, digit by digit -----------------------------------------------------------
//
// A pass over a digit of the rows: `count_kernel` counts a tile's tokens by digit, `scan_kernel` turns the
// counts of a digit into places among its tokens, `move_kernel` moves the tokens there; equal digits keep
// their order.  Padding has the key V, behind all rows.  What bounds it are the kernels' own chains of loads and
// exchanges in shared memory (a million tokens of a million rows, two digits of ten bits: 4 + 6 + 14 us and 5 + 6 + 13).
constexpr int kMostBits = 11, kMostBins = 1 << kMostBits;
constexpr int kRound = 2048;     // tokens that a block moves at once, 256 a warp
constexpr int kMostTiles = 1216;
constexpr int kFewTiles = 64;    // (33 tiles: the call took 42 us with a scan)

struct Sort {
  const int32_t* ids;  // first pass; null: `from`
  const uint2* from;
  uint2* to;
  int64_t n;
  int32_t V;
  int shift, bits, bins, tiles;
  int64_t tile;        // tokens of a tile: a multiple of kRound
  uint32_t* counts;    // [tiles][bins]
  int direct;          // few tiles: each block adds the counts of those before it, and nothing is scanned
  uint32_t* totals;    // [bins]
  uint32_t* status;
};

__device__ __forceinline__ uint32_t key_of(const Sort& a, int64_t i) {
  if (!a.ids) return a.from[i].x;
  const int32_t id = a.ids[i];
  return (uint32_t)id < (uint32_t)a.V ? (uint32_t)id : (uint32_t)a.V;
}

__global__ void __launch_bounds__(kThreads) count_kernel(Sort a) {
  __shared__ uint32_t bins[kMostBins];
  const int64_t first = blockIdx.x * a.tile, end = first + a.tile < a.n ? first + a.tile : a.n;
  for (int d = threadIdx.x; d < a.bins; d += kThreads) bins[d] = 0;
  await_previous_kernel();
  __syncthreads();
  for (int64_t r = first + threadIdx.x; r < end; r += kRound) {
    uint32_t key[kRound / kThreads];
#pragma unroll
    for (int k = 0; k < kRound / kThreads; ++k) {
      const int64_t i = r + k * kThreads;
      key[k] = i >= end ? 0 : a.ids ? (uint32_t)a.ids[i] : a.from[i].x;
    }
#pragma unroll
    for (int k = 0; k < kRound / kThreads; ++k) {
      if (r + k * kThreads >= end) break;
      if (a.ids && key[k] - (uint32_t)a.V < 0x80000000u - (uint32_t)a.V) atomicOr(a.status, kErrId);
      atomicAdd(&bins[(min(key[k], (uint32_t)a.V) >> a.shift) & (a.bins - 1)], 1u);
    }
  }
  __syncthreads();
  for (int d = threadIdx.x; d < a.bins; d += kThreads) a.counts[(int64_t)blockIdx.x * a.bins + d] = bins[d];
}

// 32 digits a block, one a lane; each warp has a run of tiles.
constexpr int kScanWarps = 32 /* one for each digit of a block */, kScanTiles = (kMostTiles + kScanWarps - 1) / kScanWarps;
__global__ void __launch_bounds__(32 * kScanWarps) scan_kernel(Sort a) {
  __shared__ uint32_t sums[kScanWarps][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32, d = blockIdx.x * 32 + lane;
  const int each = (a.tiles + kScanWarps - 1) / kScanWarps, begin = warp * each, end = min(begin + each, a.tiles);
  await_previous_kernel();
  const bool live = d < a.bins;
  uint32_t* column = a.counts + (begin * a.bins + d);  // (fewer than 2^22 counts)
  uint32_t own[kScanTiles], sum = 0;
#pragma unroll
  for (int k = 0; k < kScanTiles; ++k) own[k] = 0;
#pragma unroll
  for (int k = 0; k < kScanTiles; ++k) {
    if (begin + k >= end) break;
    if (live) own[k] = column[k * a.bins];
  }
#pragma unroll
  for (int k = 0; k < kScanTiles; ++k) sum += own[k];
  sums[warp][lane] = sum;
  __syncthreads();
  {  // a warp adds up the runs of one digit, a run a lane
    const uint32_t own_run = sums[lane][warp];
    uint32_t up = own_run;
#pragma unroll
    for (int off = 1; off < 32; off *= 2) {
      const uint32_t x = __shfl_up_sync(0xffffffffu, up, off);
      if (lane >= off) up += x;
    }
    sums[lane][warp] = up - own_run;
  }
  __syncthreads();
  uint32_t before = sums[warp][lane];
  if (!live) return;
  if (warp == kScanWarps - 1) a.totals[d] = before + sum;
#pragma unroll
  for (int k = 0; k < kScanTiles; ++k) {
    if (begin + k >= end) break;
    column[k * a.bins] = before;
    before += own[k];
  }
}

__global__ void __launch_bounds__(kThreads, 4) move_kernel(Sort a) {
  constexpr int kWarps = kThreads / 32, kEach = kRound / kThreads, kRuns = kMostBins / kThreads / 4;
  __shared__ uint32_t place[kMostBins], warp_sum[kWarps];
  __shared__ __align__(16) uint16_t ahead[kWarps][kMostBins];  // a digit's tokens in a round before a warp's next ones
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32, tid = threadIdx.x;
  const int64_t first = blockIdx.x * a.tile, end = first + a.tile < a.n ? first + a.tile : a.n;
  const int each = (a.bins + kThreads - 1) / kThreads;
  uint32_t key[kEach], val[kEach];
  auto load = [&](int64_t r) {
    const int64_t mine = r + warp * (32 * kEach) + lane;
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      const int64_t i = mine + k * 32;
      key[k] = val[k] = 0;
      if (i >= end) continue;
      if (a.ids) {
        key[k] = key_of(a, i), val[k] = (uint32_t)i;
      } else {
        const uint2 p = a.from[i];
        key[k] = p.x, val[k] = p.y;
      }
    }
  };
  await_previous_kernel();
  load(first);
  {  // where the digits begin: each thread's run of digits, warps, all
    uint32_t total[4 * kRuns], count[4 * kRuns], sum = 0;
#pragma unroll
    for (int j = 0; j < 4 * kRuns; ++j) {
      const int d = tid * each + j;
      const bool live = j < each && d < a.bins;
      total[j] = live && !a.direct ? a.totals[d] : 0;
      count[j] = live && !a.direct ? a.counts[(int64_t)blockIdx.x * a.bins + d] : 0;
    }
    if (a.direct)
      for (int t = 0; t < a.tiles; t += 8) {
#pragma unroll
        for (int j = 0; j < 4 * kRuns; ++j) {
          const int d = tid * each + j;
          if (j >= each || d >= a.bins) break;
          uint32_t c[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) c[k] = t + k < a.tiles ? a.counts[(t + k) * a.bins + d] : 0;
#pragma unroll
          for (int k = 0; k < 8; ++k) total[j] += c[k], count[j] += t + k < (int)blockIdx.x ? c[k] : 0;
        }
      }
#pragma unroll
    for (int j = 0; j < 4 * kRuns; ++j) sum += total[j];
    uint32_t up = sum;
#pragma unroll
    for (int off = 1; off < 32; off *= 2) {
      const uint32_t x = __shfl_up_sync(0xffffffffu, up, off);
      if (lane >= off) up += x;
    }
    if (lane == 31) warp_sum[warp] = up;
    __syncthreads();
    uint32_t before = up - sum;
    for (int w = 0; w < warp; ++w) before += warp_sum[w];
#pragma unroll
    for (int j = 0; j < 4 * kRuns; ++j) {
      if (j < each && tid * each + j < a.bins) place[tid * each + j] = before + count[j];
      before += total[j];
    }
  }
  for (int64_t r = first; r < end; r += kRound) {
    if (r > first) load(r);
    for (int d = lane * 8; d < a.bins; d += 256) *reinterpret_cast<uint4*>(&ahead[warp][d]) = make_uint4(0, 0, 0, 0);
    __syncwarp();
    const int64_t mine = r + warp * (32 * kEach) + lane;
    uint32_t rank[kEach];
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      const bool live = mine + k * 32 < end;
      const uint32_t d = (key[k] >> a.shift) & (a.bins - 1);
      // The lanes with the same digit, bit by bit (a million tokens: 14 us; by one instruction that matches whole digits
      // 17).
      uint32_t same = __ballot_sync(0xffffffffu, live);
      for (int b = 0; b < a.bits; ++b) {
        const bool one = d >> b & 1u;
        const uint32_t ones = __ballot_sync(0xffffffffu, one);
        same &= one ? ones : ~ones;
      }
      rank[k] = live ? ahead[warp][d] + __popc(same & ((1u << lane) - 1)) : 0;
      __syncwarp();
      if (live && lane == __ffs(same) - 1) ahead[warp][d] += (uint16_t)__popc(same);
      __syncwarp();
    }
    __syncthreads();
    // Four digits at once in two words (a round's counts of a digit stay below 2^16).
    uint2 all[kRuns];
#pragma unroll
    for (int j = 0; j < kRuns; ++j) {
      const int d = (tid + j * kThreads) * 4;
      if (d >= a.bins) break;
      uint2 sum = make_uint2(0, 0);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        uint2* at = reinterpret_cast<uint2*>(&ahead[w][d]);
        const uint2 c = *at;
        *at = sum;
        sum.x += c.x, sum.y += c.y;
      }
      all[j] = sum;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      if (mine + k * 32 >= end) continue;
      const uint32_t d = (key[k] >> a.shift) & (a.bins - 1);
      a.to[place[d] + ahead[warp][d] + rank[k]] = make_uint2(key[k], val[k]);
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kRuns; ++j) {
      const int d = (tid + j * kThreads) * 4;
      if (d >= a.bins) break;
      place[d] += all[j].x & 0xffffu, place[d + 1] += all[j].x >> 16;
      place[d + 2] += all[j].y & 0xffffu, place[d + 3] += all[j].y >> 16;
    }
  }
}

// Zeros beside the sort, past the caches' older lines.
__global__ void __launch_bounds__(kThreads) zero_kernel(char* to, int64_t bytes) {
  const int64_t first = (16 - (reinterpret_cast<uintptr_t>(to) & 15)) & 15, head = first < bytes ? first : bytes;
  const int64_t body = (bytes - head) / 16, step = (int64_t)gridDim.x * kThreads;
  uint4* words = reinterpret_cast<uint4*>(to + head);
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < body; i += step) __stcs(words + i, make_uint4(0, 0, 0, 0));
  if (blockIdx.x != 0) return;
  for (int64_t k = 2 * threadIdx.x; k < head; k += 2 * kThreads) *reinterpret_cast<uint16_t*>(to + k) = 0;
  for (int64_t k = head + body * 16 + 2 * threadIdx.x; k < bytes; k += 2 * kThreads) *reinterpret_cast<uint16_t*>(to + k) = 0;
}

// ---- many tokens: the sums ------------------------------------------------------------------------------------
//
// A group of lanes adds a chunk of sorted tokens.  Rows that begin and end among them are written; the sums of those
// that do not are joined over the groups of a block, and what crosses blocks goes to `part`: [block][0] the sum of the
// row that the block's first token shares with the block before, [block][1] of the row that goes on behind the block.
// Rows without tokens have been set to zero beside the sort.  Every group has the same number of tokens, however popular
// a row is; eight loads are under way (a million tokens of 64 fp32 values: 52 us, 230 MB read and 50 written).
constexpr int kMostTokens = 2048;  // of a block

template <typename T, int VEC, int K, bool ADD>
__global__ void __launch_bounds__(kThreads, ADD ? 4 : 3) sums_kernel(Gradient a) {
  constexpr int U = (ADD ? 4 : 8) / K;
  __shared__ float head[K * VEC][kThreads], tail[K * VEC][kThreads];
  __shared__ uint8_t flags[kThreads];  // of a group: 1 a head, 2 a tail, 4 the head is the whole chunk and goes on
  __shared__ uint2 pairs[kMostTokens];
  __shared__ uint32_t key_before, key_behind;
  const int tid = threadIdx.x;
  await_previous_kernel();
  const int lane = tid & (a.lanes - 1), group = tid / a.lanes, groups = kThreads / a.lanes, chunk = a.chunk;
  const int c0 = blockIdx.y * a.lanes * K + lane;
  const int64_t block = blockIdx.x, first = block * groups * chunk;
  const int many = a.n - first < groups * chunk ? (int)(a.n - first) : groups * chunk;  // the block's tokens
  for (int i = tid; i < many; i += kThreads) pairs[i] = a.pairs[first + i];
  if (tid == 0) {
    key_before = first > 0 ? a.pairs[first - 1].x : 0xffffffffu;
    key_behind = first + many < a.n ? a.pairs[first + many].x : 0xffffffffu;
  }
  __syncthreads();
  const uint32_t V = (uint32_t)a.V;
  auto key = [&](int i) { return i < many ? pairs[i].x : key_behind; };
  const int begin = group * chunk, end = begin + chunk < many ? begin + chunk : many;
  float sum[K][VEC] = {};
  uint32_t f = 0;
  if (begin < end) {
    const uint32_t before = begin > 0 ? pairs[begin - 1].x : key_before;
    bool shared_row = before == pairs[begin].x;
    for (int i = begin; i < end; i += U) {
      uint2 p[U];
      uint32_t after[U];
      Raw<T, VEC> x[U][K], old[ADD ? U : 1][K];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        p[u] = i + u < end ? pairs[i + u] : make_uint2(0xffffffffu, 0);
        after[u] = key(i + u + 1);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
          const int c = c0 + k * a.lanes;
          x[u][k] = load_raw<T, VEC>(static_cast<const T*>(a.grad) + p[u].y * a.grad_stride + c * VEC, p[u].x < V && c < a.per_row);
        }
        if (ADD && p[u].x < V && after[u] != p[u].x) read_old<T, VEC, K>(a, p[u].x, c0, old[u]);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (p[u].x >= V) break;
#pragma unroll
        for (int k = 0; k < K; ++k) add_raw<T, VEC>(x[u][k], sum[k]);
        if (after[u] == p[u].x) continue;
        if (shared_row) {
          f |= 1;
#pragma unroll
          for (int q = 0; q < K * VEC; ++q) head[q][tid] = sum[q / VEC][q % VEC];
        } else {
          emit<T, VEC, K>(a, p[u].x, c0, sum, old[ADD ? u : 0]);
        }
        shared_row = false;
#pragma unroll
        for (int q = 0; q < K * VEC; ++q) sum[q / VEC][q % VEC] = 0.f;
      }
    }
    const uint32_t last = pairs[end - 1].x;
    if (last < V && key(end) == last) {  // the row goes on behind the chunk
      f |= shared_row ? 5 : 2;
#pragma unroll
      for (int q = 0; q < K * VEC; ++q) (shared_row ? head : tail)[q][tid] = sum[q / VEC][q % VEC];
    }
  }
  if (lane == 0) flags[group] = (uint8_t)f;
  __syncthreads();
  // Rows shared by the block's groups: from a tail on, and from the block's first token on.
  for (int from_head = 0; from_head < 2; ++from_head) {
    if (from_head ? group != 0 || !(flags[0] & 1) : !(flags[group] & 2)) continue;
    int g = group;
    bool open = true;
    if (from_head) {
#pragma unroll
      for (int q = 0; q < K * VEC; ++q) sum[q / VEC][q % VEC] = head[q][tid];
      open = flags[0] & 4;
    } else {
#pragma unroll
      for (int q = 0; q < K * VEC; ++q) sum[q / VEC][q % VEC] = tail[q][tid];
    }
    while (open && ++g < groups) {
#pragma unroll
      for (int q = 0; q < K * VEC; ++q) sum[q / VEC][q % VEC] += head[q][g * a.lanes + lane];
      open = flags[g] & 4;
    }
    if (!from_head && !open) {
      Raw<T, VEC> old[K];
      const uint32_t row = pairs[end - 1].x;
      read_old<T, VEC, K>(a, row, c0, old);
      emit<T, VEC, K>(a, row, c0, sum, old);
      continue;
    }
    float* to = a.part + (2 * block + (from_head ? 0 : 1)) * a.D;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = c0 + k * a.lanes;
      if (c >= a.per_row) break;
#pragma unroll
      for (int j = 0; j < VEC; ++j) to[c * VEC + j] = sum[k][j];
    }
  }
}

// Rows that cross blocks of the sums: a warp for each block in which one begins, all warps in turn for rows of more than
// kFewParts of them.
constexpr int kFewParts = 16, kJoinColumns = 128;

template <typename T>
__global__ void __launch_bounds__(kThreads) join_kernel(Gradient a, int64_t block_tokens) {
  constexpr int kWarps = kThreads / 32, K = kJoinColumns / 32;
  __shared__ float red[kWarps][kJoinColumns];
  __shared__ int64_t parts[kWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32, c0 = blockIdx.y * kJoinColumns + lane;
  const int64_t first = (int64_t)blockIdx.x * kWarps, b = first + warp, end = (b + 1) * block_tokens;
  int64_t more = 0;  // parts behind the first
  await_previous_kernel();
  if (end < a.n) {
    const uint32_t row = a.pairs[end - 1].x;
    const bool begins = b == 0 || a.pairs[end - block_tokens - 1].x != row;
    if (row < (uint32_t)a.V && begins && a.pairs[end].x == row)
      for (bool on = true; on;) {
        const int64_t at = end + (more + lane) * block_tokens;  // whether the row goes on into that block
        const uint32_t yes = __ballot_sync(0xffffffffu, at < a.n && a.pairs[at < a.n ? at : end].x == row);
        on = yes == 0xffffffffu;
        more += on ? 32 : __ffs(~yes) - 1;
      }
  }
  if (lane == 0) parts[warp] = more;
  auto sum_parts = [&](int64_t from, int64_t many, int64_t k0, int step, float (&sum)[K]) {
    for (int64_t k = k0; k < many; k += 4 * step) {
      float x[4][K];
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int q = 0; q < K; ++q) {
          const bool live = k + u * step < many && c0 + q * 32 < a.D;
          x[u][q] = live ? a.part[2 * (from + 1 + k + u * step) * a.D + c0 + q * 32] : 0.f;
        }
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int q = 0; q < K; ++q) sum[q] += x[u][q];
    }
  };
  auto write = [&](int64_t from, const float (&sum)[K]) {
    T* out = static_cast<T*>(a.out) + (int64_t)a.pairs[(from + 1) * block_tokens - 1].x * a.D;
#pragma unroll
    for (int q = 0; q < K; ++q) {
      const int c = c0 + q * 32;
      if (c >= a.D) break;
      const float all = a.part[(2 * from + 1) * a.D + c] + sum[q];
      out[c] = from_float<T>(a.accumulate ? fmaf(all, a.scale, to_float(out[c])) : all * a.scale);
    }
  };
  if (more > 0 && more <= kFewParts) {
    float sum[K] = {};
    sum_parts(b, more, 0, 1, sum);
    write(b, sum);
  }
  __syncthreads();
  for (int w = 0; w < kWarps; ++w) {
    if (parts[w] <= kFewParts) continue;
    float sum[K] = {};
    sum_parts(first + w, parts[w], warp, kWarps, sum);
#pragma unroll
    for (int q = 0; q < K; ++q) red[warp][q * 32 + lane] = sum[q];
    __syncthreads();
    if (warp == 0) {
#pragma unroll
      for (int q = 0; q < K; ++q)
#pragma unroll
        for (int k = 1; k < kWarps; ++k) sum[q] += red[k][q * 32 + lane];
      write(first + w, sum);
    }
    __syncthreads();
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

// Passes of the sort over keys 0..V and bits of a pass's digit.
struct Digits {
  int passes, bits;
};
Digits digits(int64_t V) {
  const int all = bits_of((uint32_t)V), passes = (all + kMostBits - 1) / kMostBits;
  const int bits = (all + passes - 1) / passes;
  return {passes, bits < 3 ? 3 : bits};  // (digits are taken by eights)
}

int64_t tile_tokens(int64_t n) {  // at most kMostTiles tiles
  const int64_t rounds = (n + (int64_t)kRound * kMostTiles - 1) / ((int64_t)kRound * kMostTiles);
  return kRound * (rounds > 0 ? rounds : 1);
}

// Lanes of a group: the power of two that holds a row's `vectors`, up to a warp.
int lanes_of(int vectors) {
  int lanes = 1;
  while (lanes < 32 && lanes < vectors) lanes *= 2;
  return lanes;
}

// Whether a call of n tokens goes by one kernel: up to kAlwaysFew of them, or 3.5 MB of rows (a popular row's are added by one
// SM), and a block's rows and a place fit 32 bits.  Measured in a graph, one kernel and by the sort, us: 4000 tokens, 5000
// rows of 100 fp32 values 11 and 20, of 1000 19 and 25; 8000 of 100 values 16 and 21, of 257 20 and 23, of 1000
// 27 and 29 (500 rows: 16 and 16, 23 and 18, 27 and 21); 16000 of 16 values 25 and 22, of 100 30 and 22.  So the table's
// rows count too, and the rule, which leaves them out, is up to 3 us off in a graph; the sort's six or seven launches cost
// the host of an eager call 20 us.
constexpr int kAlwaysFew = 4096;
bool does_few(int64_t n, int64_t V, int32_t D, size_t size) {
  if (n > kFew || (n > kAlwaysFew && n * D * (int64_t)size > 3'500'000)) return false;
  const int columns = (D + 31) / 32;  // at most so many tiles of columns
  const int64_t blocks = columns < kFewBlocks ? kFewBlocks / columns : 1;
  return (uint64_t)((V + blocks - 1) / blocks) << bits_of((uint32_t)n - 1) <= 0xffffffffull;
}

// Tokens of a group of the sums: 32 (8 of a lane, where that is less), fewer where there would not be kSumWarps warps.
constexpr int64_t kSumWarps = 24 * 152;
int chunk_of(int64_t n, int lanes) {
  const int most = 8 * lanes < 32 ? 8 * lanes : 32;
  int chunk = most;
  while (chunk > 8 && n * lanes < kSumWarps * 32 * chunk) chunk /= 2;
  return chunk;
}
// Blocks of the sums of up to n tokens, in which a block has eight warps: those of shorter chunks are fewer than twice kSumWarps.
int64_t most_blocks(int64_t n, int lanes) {
  const int64_t tokens = kThreads / lanes * (8 * lanes < 32 ? 8 * lanes : 32), blocks = (n + tokens - 1) / tokens;
  const int64_t few = kSumWarps * 2 / (kThreads / 32) + 1;
  return blocks > few ? blocks : few;
}

struct Carve {
  size_t status, pairs[2], counts, totals, part, total;
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
  if (c.backward && !does_few(c.max_tokens, c.n_rows, c.width, size_of(c.dtype))) {
    const int64_t n = c.max_tokens;
    const Digits d = digits(c.n_rows);
    for (int i = 0; i < 2; ++i) k.pairs[i] = take(n * sizeof(uint2));
    const int64_t tiles = (n + kRound - 1) / kRound;  // (longer tiles are fewer)
    k.counts = take(((size_t)(tiles < kMostTiles ? tiles : kMostTiles) << d.bits) * sizeof(uint32_t));
    k.totals = take(((size_t)1 << d.bits) * sizeof(uint32_t));
    // (most blocks where rows take most lanes)
    k.part = take((size_t)most_blocks(n, lanes_of(c.width)) * 2 * c.width * sizeof(float));
  }
  k.total = o;
  return k;
}

// f(type, vector, K) for a type and the bytes that its rows can be read in: 16, or single values, where a lane
// takes four that lie a group apart.
template <typename F>
cudaError_t by_type(int dtype, int bytes, F f) {
  auto go = [&](auto* type) {
    using T = std::remove_pointer_t<decltype(type)>;
    if (bytes >= 16) return f(type, std::integral_constant<int, 16 / sizeof(T)>{}, std::integral_constant<int, 1>{});
    return f(type, std::integral_constant<int, 1>{}, std::integral_constant<int, 4>{});
  };
  if (dtype == ESSPT_F32) return go((float*)nullptr);
  if (dtype == ESSPT_BF16) return go((__nv_bfloat16*)nullptr);
  return go((__half*)nullptr);
}

template <typename T, int VEC, int K>
cudaError_t launch_few(Gradient a, cudaStream_t st) {
  a.per_row = a.D / VEC;
  a.lanes = lanes_of((a.per_row + K - 1) / K);
  const int columns = (a.per_row + a.lanes * K - 1) / (a.lanes * K);
  int64_t blocks = kFewBlocks / columns;
  blocks = blocks < 1 ? 1 : blocks > a.V ? a.V : blocks;
  a.rows = (int32_t)((a.V + blocks - 1) / blocks);
  blocks = (a.V + a.rows - 1) / a.rows;
  a.place_bits = bits_of((uint32_t)a.n - 1);
  if (((uint64_t)a.rows << a.place_bits) > 0xffffffffull) return cudaErrorInvalidValue;  // (does_few says no)
  uint32_t size = 4 * kFewThreads;
  while (size < a.n) size *= 2;
  auto* kernel = few_kernel<T, VEC, K>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kFew * sizeof(uint32_t));
  if (e != cudaSuccess) return e;
  kernel<<<dim3((unsigned)blocks, (unsigned)columns), kFewThreads, size * sizeof(uint32_t), st>>>(a);
  return cudaGetLastError();
}

constexpr int64_t kZeroBlocks = 304;
constexpr int64_t kZeroInLine = 48 << 20;  // zeros of up to so many bytes, 8 us, come before the sort: two streams' events cost as much
// `beside`: on the side stream, which the sums then wait for.
cudaError_t set_to_zero(const esspt_embed& em, const Gradient& a, int64_t bytes, bool beside) {
  cudaError_t e = beside ? cudaEventRecord(em.fork, em.st) : cudaSuccess;
  if (e == cudaSuccess && beside) e = cudaStreamWaitEvent(em.side, em.fork, 0);
  if (e != cudaSuccess) return e;
  const int64_t blocks = (bytes + kThreads * 64 - 1) / (kThreads * 64);
  zero_kernel<<<(unsigned)(blocks < kZeroBlocks ? blocks : kZeroBlocks), kThreads, 0, beside ? em.side : em.st>>>(
      static_cast<char*>(a.out), bytes);
  e = cudaGetLastError();
  if (e == cudaSuccess && beside) e = cudaEventRecord(em.join, em.side);
  return e;
}

void release(esspt_embed* em) {
  if (em->fork) cudaEventDestroy(em->fork);
  if (em->join) cudaEventDestroy(em->join);
  if (em->side) cudaStreamDestroy(em->side);
  delete em;
}

cudaError_t launch_sort(const esspt_embed& em, const Carve& k, Gradient& a) {
  const Digits d = digits(a.V);
  auto words = [&](size_t o) { return reinterpret_cast<uint32_t*>(em.base + o); };
  Sort s{};
  s.ids = a.ids, s.n = a.n, s.V = a.V, s.bits = d.bits, s.bins = 1 << d.bits;
  s.tile = tile_tokens(a.n), s.tiles = (int)((a.n + s.tile - 1) / s.tile);
  s.direct = s.tiles <= kFewTiles;
  s.counts = words(k.counts), s.totals = words(k.totals), s.status = a.status;
  for (int pass = 0; pass < d.passes; ++pass) {
    s.shift = pass * d.bits;
    s.to = reinterpret_cast<uint2*>(em.base + k.pairs[pass & 1]);
    cudaError_t e = launch_chained(count_kernel, s.tiles, kThreads, em.st, pass > 0, s);
    if (e == cudaSuccess && !s.direct) e = launch_chained(scan_kernel, (s.bins + 31) / 32, 32 * kScanWarps, em.st, true, s);
    if (e == cudaSuccess) e = launch_chained(move_kernel, s.tiles, kThreads, em.st, true, s);
    if (e != cudaSuccess) return e;
    s.ids = nullptr, s.from = s.to;
  }
  a.pairs = s.to;
  return cudaSuccess;
}

template <typename T, int VEC, int K>
cudaError_t launch_sums(Gradient a, cudaStream_t st) {
  a.per_row = a.D / VEC;
  a.lanes = lanes_of((a.per_row + K - 1) / K);
  const int columns = (a.per_row + a.lanes * K - 1) / (a.lanes * K);
  a.chunk = chunk_of(a.n, a.lanes);
  const int64_t tokens = kThreads / a.lanes * a.chunk, blocks = (a.n + tokens - 1) / tokens;
  const dim3 grid((unsigned)blocks, (unsigned)columns);
  cudaError_t e = a.accumulate ? launch_chained(sums_kernel<T, VEC, K, true>, grid, kThreads, st, true, a)
                               : launch_chained(sums_kernel<T, VEC, K, false>, grid, kThreads, st, false, a);  // (it waits for the zeros too)
  if (e != cudaSuccess) return e;
  constexpr int kWarps = kThreads / 32;
  const dim3 joins((unsigned)((blocks + kWarps - 1) / kWarps), (unsigned)((a.D + kJoinColumns - 1) / kJoinColumns));
  return launch_chained(join_kernel<T>, joins, kThreads, st, true, a, tokens);
}

}  // namespace

extern "C" {

size_t esspt_embed_workspace_bytes(const esspt_embed_config* cfg) { return config_fault(cfg) ? 0 : carve(*cfg).total; }

esspt_status esspt_embed_create(const esspt_embed_config* cfg, void* d_workspace, size_t bytes, esspt_embed** out) {
  g_create.text[0] = 0;
  if (const char* why = config_fault(cfg)) return g_create.fail(ESSPT_EINVAL, why);
  if (!out || !d_workspace || misaligned(d_workspace, 256)) return g_create.fail(ESSPT_EINVAL, "null or misaligned pointer");
  if (bytes < carve(*cfg).total) return g_create.fail(ESSPT_ENOSPC, "workspace too small");
  ESSPT_CUDA(g_create, cudaMemsetAsync(d_workspace, 0, 256, static_cast<cudaStream_t>(cfg->stream)));
  esspt_embed* em = new (std::nothrow) esspt_embed;
  if (!em) return g_create.fail(ESSPT_ENOSPC, "out of host memory");
  em->cfg = *cfg;
  em->st = static_cast<cudaStream_t>(cfg->stream);
  em->base = static_cast<char*>(d_workspace);
  if (cfg->backward && !does_few(cfg->max_tokens, cfg->n_rows, cfg->width, size_of(cfg->dtype))) {
    cudaError_t e = cudaStreamCreateWithFlags(&em->side, cudaStreamNonBlocking);
    if (e == cudaSuccess) e = cudaEventCreateWithFlags(&em->fork, cudaEventDisableTiming);
    if (e == cudaSuccess) e = cudaEventCreateWithFlags(&em->join, cudaEventDisableTiming);
    if (e != cudaSuccess) {
      release(em);
      return g_create.cuda(e, "esspt_embed_create");
    }
  }
  *out = em;
  return ESSPT_OK;
}

esspt_status esspt_embed_destroy(esspt_embed* em) {
  if (!em) return ESSPT_OK;
  cudaError_t e = cudaStreamSynchronize(em->st);
  if (e == cudaSuccess && em->side) e = cudaStreamSynchronize(em->side);  // (after a call that failed half-way)
  release(em);
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
  auto go = [&](auto* type, auto vec, auto pairs) {
    using T = std::remove_pointer_t<decltype(type)>;
    a.per_row = c.width / vec;
    const int64_t each = kThreads * kDeep<T, vec>, all = pairs ? (n * c.width + 1) / 2 : n * a.per_row;
    lookup_kernel<T, vec, pairs><<<(unsigned)((all + each - 1) / each), kThreads, 0, em->st>>>(a);
    return cudaGetLastError();
  };
  auto by_vector = [&](auto* type) {
    constexpr int kSize = sizeof(*type);
    if (bytes >= 16) return go(type, std::integral_constant<int, 16 / kSize>{}, std::false_type{});
    if (bytes >= 8) return go(type, std::integral_constant<int, 8 / kSize>{}, std::false_type{});
    if (bytes >= 4) return go(type, std::integral_constant<int, 4 / kSize>{}, std::false_type{});
    if constexpr (kSize == 2) {
      if (!misaligned(d_out, 4)) return go(type, std::integral_constant<int, 1>{}, std::true_type{});
    }
    return go(type, std::integral_constant<int, 1>{}, std::false_type{});
  };
  const cudaError_t launched = c.dtype == ESSPT_F32    ? by_vector((float*)nullptr)
                               : c.dtype == ESSPT_BF16 ? by_vector((__nv_bfloat16*)nullptr)
                                                       : by_vector((__half*)nullptr);
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
  Gradient a{};
  a.ids = d_ids, a.grad = d_grad, a.grad_stride = grad_stride, a.n = n, a.V = (int32_t)c.n_rows, a.D = c.width;
  a.scale = scale, a.accumulate = accumulate != 0, a.out = d_grad_w, a.status = reinterpret_cast<uint32_t*>(em->base);
  const int bytes = vector_bytes(c.width, size, (uintptr_t)d_grad | (uintptr_t)d_grad_w | (uintptr_t)grad_stride * size);
  const bool few = does_few(n, c.n_rows, c.width, size);
  if (!few) {
    const Carve k = carve(c);
    a.part = reinterpret_cast<float*>(em->base + k.part);
    const int64_t bytes = accumulate ? 0 : c.n_rows * c.width * (int64_t)size;
    const bool beside = bytes > kZeroInLine;
    if (bytes > 0) ESSPT_CUDA(em->err, set_to_zero(*em, a, bytes, beside));
    ESSPT_CUDA(em->err, launch_sort(*em, k, a));
    if (beside) ESSPT_CUDA(em->err, cudaStreamWaitEvent(em->st, em->join, 0));
  }
  const cudaError_t launched = by_type(c.dtype, bytes, [&](auto* type, auto vec, auto k) {
    using T = std::remove_pointer_t<decltype(type)>;
    return few ? launch_few<T, vec, k>(a, em->st) : launch_sums<T, vec, k>(a, em->st);
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
