// Softmax operators for many rows: operands laid out for the tensor cores, the
// passes over tiles of scores, and what joins their partial results.
//
//   compact    the kept rows in order (ignored ones cost nothing from here on)
//   max, units H (kept rows) and W in 16 KB units, fp32 in two halves by powers of two
//   stats      maximum and sum of every row, then its loss; or, with gradients, references
//              for the rows: their maxima, of large problems of bf16 rows over a part of W
//   rows       sum p w (and sum p), then dh and the loss
//   entries    targets sorted by item on a second stream, sums over long runs of one item
//   cols       fp32 rows (and fp16 rows of weights far apart): the largest weight p of every
//              item, in large problems where a tile of rows says so; sum weight p h, then dw
//
// The kernels here are bound by bytes or by latency: 2048 x 1M, K = 64, fp32, GB300:
// max 52 us (256 MB, 4.9 TB/s), units 84 (512 MB, 6.1 TB/s), dw 133 (512 MB, 3.9 TB/s,
// with its scattered targets) of the call's 2890.
#include <cub/device/device_radix_sort.cuh>

#include <algorithm>

#include "softmax_mma.cuh"

namespace esspt {

namespace {

struct Many {
  SoftmaxArgs a;
  ManyScratch s;
  MmaShape shape;
  int blocks;  // of the pass whose slots are read
  int ld;
  int parts;
  int32_t sample;  // rows of W that the rows' references are taken over, 0: all (exact maxima)
  float up;        // probabilities of the rows pass are taken 2^up times as large
  int if_redo;     // only where words->redo is set
  int high_tiles;  // tiles of the pass over high halves where that may have run, else 0
};

__device__ __forceinline__ uint32_t finite_bits(float x) {
  const uint32_t u = __float_as_uint(fabsf(x));
  return u < 0x7f800000u ? u : 0u;
}
__device__ __forceinline__ void block_max(uint32_t x, uint32_t* to) {
  x = __reduce_max_sync(0xffffffffu, x);
  if ((threadIdx.x & 31) == 0 && x != 0u) atomicMax(to, x);
}

// Places of the kept rows.  A block counts the kept rows before its own 1024 first, so
// one launch does: 4 us at 8k rows, of which a block reads 4k on average.
__global__ void __launch_bounds__(1024) compact_kernel(Many f) {
  __shared__ int32_t sums[32];
  const SoftmaxArgs& a = f.a;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t t0 = (int64_t)blockIdx.x * 1024, t = t0 + threadIdx.x;
  int32_t before = 0;
#pragma unroll 4
  for (int64_t i = threadIdx.x; i < t0; i += 1024) before += row_kept(a.target, i);
  before = __reduce_add_sync(0xffffffffu, before);
  if (lane == 0) sums[warp] = before;
  __syncthreads();
  int32_t base = 0;
  for (int i = 0; i < 32; ++i) base += sums[i];
  __syncthreads();
  const bool kept = t < a.n && row_kept(a.target, t);
  const unsigned votes = __ballot_sync(0xffffffffu, kept);
  if (lane == 0) sums[warp] = __popc(votes);
  __syncthreads();
  for (int i = 0; i < warp; ++i) base += sums[i];
  base += __popc(votes & ((1u << lane) - 1u));
  if (t < a.n) {
    f.s.pos[t] = kept ? base : -1;
    if (kept) f.s.act[base] = (int32_t)t;
    if (!a.target.logits && a.target.ids[t] >= a.V) atomicOr(a.target.status, kErrTarget);
    if (t == a.n - 1) f.s.words->rows = base + kept, f.s.words->low = f.high_tiles == 0;
  }
  if (a.weight && __any_sync(0xffffffffu, kept && a.weight[t] < 0.f) && lane == 0) f.s.words->negative = 1u;
  if (a.weight) {
    const uint32_t bits = kept ? finite_bits(a.weight[t]) : 0u;
    block_max(bits, &f.s.words->max_weight);
    block_max(bits ? 0x7f800000u - bits : 0u, &f.s.words->min_weight);
  } else if (t == 0) {
    f.s.words->max_weight = __float_as_uint(1.f);
    f.s.words->min_weight = 0x7f800000u - __float_as_uint(1.f);
  }
}

// Largest finite magnitude of W, and of the kept rows of H (blockIdx.y = 1): a warp
// takes rows as they come, or a matrix without gaps as one long row in parts of 4096.
template <int VEC>
__global__ void __launch_bounds__(256) max_kernel(Many f) {
  const SoftmaxArgs& a = f.a;
  const bool is_h = blockIdx.y == 1;
  const float* x = static_cast<const float*>(is_h ? a.h : a.w);
  const int64_t stride = is_h ? a.h_stride : a.w_stride, n = is_h ? f.s.words->rows : a.V;
  const bool flat = !is_h && stride == a.D;
  const int64_t rows = flat ? (n * a.D + 4095) / 4096 : n;
  uint32_t top = 0;
  for (int64_t r = (int64_t)blockIdx.x * 8 + threadIdx.x / 32; r < rows; r += (int64_t)gridDim.x * 8) {
    const float* row = x + (flat ? r * 4096 : (is_h ? f.s.act[r] : r) * stride);
    const int len = flat ? (int)min((int64_t)4096, n * a.D - r * 4096) : a.D;
#pragma unroll 8
    for (int d = (threadIdx.x & 31) * VEC; d < len; d += 32 * VEC) {
      float v[VEC];
      load_vec<float, VEC>(row + d, v);
#pragma unroll
      for (int e = 0; e < VEC; ++e) top = max(top, finite_bits(v[e]));
    }
  }
  block_max(top, is_h ? &f.s.words->max_h : &f.s.words->max_w);
}

// Where a row's piece of 8 values lies in its unit (tensor.cuh).
__device__ __forceinline__ char* piece_of(char* units, int64_t r, int parts, int32_t nk, int32_t kc, int piece) {
  const int row = (int)(r & 127);
  return units + (((r >> 7) * parts * nk + kc) * (int64_t)kUnitBytes) + row * 128 + ((piece ^ (row & 7)) << 4);
}
// Values d .. d + 7 of a row, zero from D on.
template <typename T, int VEC>
__device__ __forceinline__ void load_piece(const T* row, int32_t d, int32_t D, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = 0.f;
#pragma unroll
  for (int e = 0; e < 8; e += VEC)
    if (d + e < D) {  // (VEC divides D)
      float k[VEC];
      load_vec<T, VEC>(row + d + e, k);
#pragma unroll
      for (int q = 0; q < VEC; ++q) v[e + q] = k[q];
    }
}

// fp32 rows to units of halves, eight lanes to a row: its largest value first, which
// decides whether the row takes a power of two of its own.  Rows of one or two units (NK)
// are kept in registers, several at once, others (0) read again (100k x 64: 12 us, by one
// row at a time 16).  The rows after the last, up to the end of its tile, and the values
// after a row's last are zero.
template <int VEC, int NK>
__global__ void __launch_bounds__(256) units_f32_kernel(Many f, unsigned w_blocks) {
  const bool is_h = blockIdx.x >= w_blocks;
  const int64_t block = blockIdx.x - (is_h ? w_blocks : 0u), blocks = is_h ? gridDim.x - w_blocks : w_blocks;
  constexpr int kKept = NK == 0 ? 1 : NK, U = NK == 0 ? 1 : 4 / NK;
  constexpr int kApart = 8, kMost = 80;  // (2^80: sums of p stay in range)
  const SoftmaxArgs& a = f.a;
  const float* x = static_cast<const float*>(is_h ? a.h : a.w);
  const int64_t rows = is_h ? f.s.words->rows : a.V, stride = is_h ? a.h_stride : a.w_stride;
  char* units = is_h ? f.s.units_h : f.s.units_w;
  RowScale* scales = is_h ? f.s.scale_h : f.s.scale_w;
  const int32_t nk = f.shape.nk, lane8 = threadIdx.x & 7;
  const uint32_t max_bits = is_h ? f.s.words->max_h : f.s.words->max_w;
  const int shift = half_shift_of(max_bits);
  const int64_t padded = (rows + 127) / 128 * 128;
  bool any = false;
  float norm = 0.f;
  const int64_t step = blocks * 32;
  for (int64_t r0 = block * 32 + threadIdx.x / 8; r0 < padded; r0 += U * step) {
    float all[U][kKept][8];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t r = r0 + u * step;
      const float* row = x + (r >= rows ? 0 : is_h ? (int64_t)f.s.act[r] : r) * stride;
#pragma unroll
      for (int kc = 0; kc < kKept; ++kc) load_piece<float, VEC>(row, kc * 64 + lane8 * 8, r < rows ? a.D : 0, all[u][kc]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t r = r0 + u * step;
      if (r >= padded) break;  // (whole warps: their four rows are of one tile)
      const float* row = x + (r >= rows ? 0 : is_h ? (int64_t)f.s.act[r] : r) * stride;
      const int32_t D = r < rows ? a.D : 0;
      float(&kept)[kKept][8] = all[u];
      uint32_t top = 0;
      float squares = 0.f;
      auto look = [&](const float (&v)[8]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          top = max(top, finite_bits(v[e]));
          const float s = times_pow2(v[e], shift);
          squares = fmaf(s, s, squares);
        }
      };
#pragma unroll
      for (int kc = 0; kc < kKept; ++kc) look(kept[kc]);
      for (int32_t kc = kKept; kc < nk; ++kc) {
        float v[8];
        load_piece<float, VEC>(row, kc * 64 + lane8 * 8, D, v);
        look(v);
      }
#pragma unroll
      for (int off = 4; off > 0; off >>= 1) {
        top = max(top, __shfl_xor_sync(0xffffffffu, top, off));
        squares += __shfl_xor_sync(0xffffffffu, squares, off);
      }
      norm = fmaxf(norm, squares);  // (a row with NaN has no share in it, one with an infinity makes it infinite)
      int own = top == 0u ? 0 : (int)(max_bits >> 23) - (int)(top >> 23);
      own = own <= kApart ? 0 : min(own, kMost);
      any |= own != 0;
      if (lane8 == 0) {
        scales[r] = RowScale{__int_as_float((127 - own) << 23), -(float)own};
        if (!is_h && r < rows && f.s.col) f.s.item_top[r] = 0u;
      }
      auto put = [&](int32_t kc, const float (&v)[8]) {
        alignas(16) __half hi[8], lo[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float s = times_pow2(v[e], shift + own);
          hi[e] = __float2half_rn(s);
          lo[e] = __float2half_rn(s - __half2float(hi[e]));
        }
        char* to = piece_of(units, r, 2, nk, kc, lane8);
        *reinterpret_cast<uint4*>(to) = *reinterpret_cast<const uint4*>(hi);
        *reinterpret_cast<uint4*>(to + nk * (int64_t)kUnitBytes) = *reinterpret_cast<const uint4*>(lo);
      };
#pragma unroll
      for (int32_t kc = 0; kc < kKept; ++kc)
        put(kc, kept[kc]);
      for (int32_t kc = kKept; kc < nk; ++kc) {
        float v[8];
        load_piece<float, VEC>(row, kc * 64 + lane8 * 8, D, v);
        put(kc, v);
      }
    }
  }
  // (Only a larger one goes to the word that all blocks share.)
  const uint32_t most = __reduce_max_sync(0xffffffffu, __float_as_uint(norm));
  uint32_t* to = is_h ? &f.s.words->norm_h : &f.s.words->norm_w;
  if ((threadIdx.x & 31) == 0 && most > *(volatile uint32_t*)to) atomicMax(to, most);
  if (__any_sync(0xffffffffu, any) && (threadIdx.x & 31) == 0) (is_h ? f.s.words->spread_h : f.s.words->spread_w) = 1u;
}

// 16-bit rows to units: a thread makes 16 bytes (8 values) of a row.  Zeros as above.
template <typename T, int VEC>
__global__ void __launch_bounds__(256) units_kernel(Many f, unsigned w_blocks) {
  const bool is_h = blockIdx.x >= w_blocks;
  const int64_t block = blockIdx.x - (is_h ? w_blocks : 0u), blocks = is_h ? gridDim.x - w_blocks : w_blocks;
  const SoftmaxArgs& a = f.a;
  const T* x = static_cast<const T*>(is_h ? a.h : a.w);
  const int64_t rows = is_h ? f.s.words->rows : a.V, stride = is_h ? a.h_stride : a.w_stride;
  char* units = is_h ? f.s.units_h : f.s.units_w;
  const int32_t nk = f.shape.nk, pieces = nk * 8;
  const int64_t total = (rows + 127) / 128 * 128 * pieces;
  for (int64_t i = block * 256 + threadIdx.x; i < total; i += blocks * 256) {
    const int64_t r = i / pieces;
    const int32_t c = (int32_t)(i - r * pieces);
    if (!is_h && c == 0 && r < rows && f.s.col) f.s.item_top[r] = 0u;
    float v[8];
    load_piece<T, VEC>(x + (r >= rows ? 0 : is_h ? (int64_t)f.s.act[r] : r) * stride, c * 8, r < rows ? a.D : 0, v);
    alignas(16) T out[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) out[e] = from_float<T>(v[e]);
    *reinterpret_cast<uint4*>(piece_of(units, r, 1, nk, c >> 3, c & 7)) = *reinterpret_cast<const uint4*>(out);
  }
}

// Column data of dw (MmaArgs); what the kernel makes of a score by it.
template <int PARTS>
__device__ __forceinline__ void set_col(const Many& f, int64_t pos, float m, float factor) {
  f.s.col_m[pos] = -m, f.s.col_f[pos] = factor;
  if (PARTS == 2) {
    float* c = f.s.col + pos / 2 * 4 + (pos & 1);
    c[0] = -m, c[2] = factor;
    f.s.col_top[pos] = log2f(fabsf(factor)) - m;
  } else {
    f.s.col[pos] = __uint_as_float((__float_as_uint(log2f(fabsf(factor)) - m) & ~1u) | (factor < 0.f ? 1u : 0u));
  }
}
__device__ __forceinline__ float col_probability(const Many& f, int64_t pos, float score, float up) {  // (16-bit rows)
  const float c = f.s.col[pos], p = exp2_fast(score + (c + up));
  return __float_as_uint(c) & 1u && f.s.words->negative ? -p : p;
}

// A warp's row: the maximum and sum of its partial statistics over W's first `items` rows.
__device__ __forceinline__ void merge_slots(const Many& f, int64_t pos, int64_t items, int tiles, float& m, float& l) {
  const int64_t rows = f.s.words->rows;
  const Ranges r(rows, items, tiles, f.blocks);
  const int64_t g = pos / (128 * tiles);
  const int tile = (int)(pos / 128 - g * tiles), row = (int)(pos & 127);
  const bool two = tiles == 2 && (g * 2 + 1) * 128 < rows;  // half of the slot per tile, else all per row
  const int64_t i0 = r.block_of(g * r.n_b), i1 = r.block_of((g + 1) * r.n_b - 1);
  m = -INFINITY, l = 0.f;
  for (int64_t i = 4 * i0 + (threadIdx.x & 31); i < 4 * i1 + 4; i += 32) {
    const int part = (int)(i & 3);
    if (two && part / 2 != tile) continue;
    const float2 p = f.s.stat[((i / 4 + g) * 4 + part) * 128 + row];
    merge_stat(m, l, p.x, p.y);
  }
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) {
    const float m2 = __shfl_xor_sync(0xffffffffu, m, off), l2 = __shfl_xor_sync(0xffffffffu, l, off);
    merge_stat(m, l, m2, l2);
  }
}

// The scores of a row's targets, 8 lanes to an entry: use(entry of the row, q, score)
// by one of them, and by that one always.
template <typename T, int VEC, typename F>
__device__ __forceinline__ void target_scores(const SoftmaxArgs& a, int64_t t, F use) {
  const int lane = threadIdx.x & 31, sub = lane & 7;
  const float k2 = a.b * kLog2e;
  const T* h = static_cast<const T*>(a.h) + t * a.h_stride;
  const int32_t* ids = a.target.ids + t * a.target.top;
  for (int k0 = 0; k0 < a.target.top; k0 += 32) {
    // Entries by lane, so that no row's load waits for its id's.
    const int count = min(32, a.target.top - k0);
    const int64_t e = t * a.target.top + k0 + lane;
    const int32_t lane_id = lane < count ? ids[k0 + lane] : -1;
    const float lane_q = lane >= count ? 0.f : a.target.logits ? a.target.q[e] : 1.f;
#pragma unroll 2
    for (int i = 0; i < count; i += 4) {
      const int32_t id = __shfl_sync(0xffffffffu, lane_id, (i + lane / 8) & 31);
      const float q = __shfl_sync(0xffffffffu, lane_q, (i + lane / 8) & 31);
      float s = 0.f;
      if (q != 0.f) {
        const T* w = static_cast<const T*>(a.w) + id * a.w_stride;
#pragma unroll 2
        for (int d = sub * VEC; d < a.D; d += 8 * VEC) {
          float x[VEC], y[VEC];
          load_vec<T, VEC>(h + d, x);
          load_vec<T, VEC>(w + d, y);
#pragma unroll
          for (int c = 0; c < VEC; ++c) s = fmaf(x[c], y[c], s);
        }
      }
#pragma unroll
      for (int off = 4; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
      if (sub == 0 && q != 0.f) use(k0 + i + lane / 8, q, s * k2);
    }
  }
}

// Columns of dw past the last kept row: no term.
template <int PARTS>
__device__ __forceinline__ void pad_cols(const Many& f, int64_t t) {
  const int lane = threadIdx.x & 31;
  const int64_t rows = f.s.words->rows, padded = (rows + 127) / 128 * 128;
  if (lane == 0 && t >= rows && t < padded) set_col<PARTS>(f, t, 1e30f, 0.f);
  if (t == f.a.n - 1)
    for (int64_t i = max(t + 1, rows) + lane; i < padded; i += 32) set_col<PARTS>(f, i, 1e30f, 0.f);
}

// What one lane writes of a row with maximum (or reference) m and sum l over it.
template <int PARTS>
__device__ __forceinline__ void finish_row(const Many& f, int64_t t, int64_t pos, float m, float l, float loss2) {
  const SoftmaxArgs& a = f.a;
  a.loss[t] = loss2 * kLn2 + (a.target.logits ? a.target.self[t] : 0.f);
  a.lse[t] = (m + log2f(l)) * kLn2;
  if (!f.s.col) return;
  f.s.row_max[pos] = m;
  f.s.row_sum[pos] = l;
  const float weight = a.weight ? a.weight[t] : 1.f;
  // (l = 0: no item was within fp32's range of the reference, as with scores of infinity.)
  set_col<PARTS>(f, pos, m, l == 0.f ? 0.f : PARTS == 2 ? weight / l * f.s.scale_h[pos].c : weight / l);
  if (fabsf(m) > kHuge) f.s.words->huge = 1u;
}

// A warp per row: its statistics, the scores of its targets, its loss.
template <typename T, int VEC>
__global__ void __launch_bounds__(256) loss_kernel(Many f) {
  constexpr int kParts = sizeof(T) == 4 ? 2 : 1;
  const SoftmaxArgs& a = f.a;
  const int64_t t = (int64_t)blockIdx.x * 8 + threadIdx.x / 32;
  const int lane = threadIdx.x & 31;
  if (t >= a.n || (f.if_redo && f.s.words->redo == 0u)) return;
  const int64_t pos = f.s.pos[t];
  if (f.s.col) pad_cols<kParts>(f, t);
  if (pos < 0) {
    if (lane == 0) a.loss[t] = a.lse[t] = 0.f;
    return;
  }
  float m, l, loss2 = 0.f;
  merge_slots(f, pos, a.V, f.shape.tiles, m, l);
  const float lse2 = m + log2f(l);
  target_scores<T, VEC>(a, t, [&](int k, float q, float s) {
    loss2 += q * (lse2 - s);
    if (f.s.col) f.s.score[t * a.target.top + k] = s;
  });
  loss2 = warp_sum(loss2);
  if (lane == 0) finish_row<kParts>(f, t, pos, m, l, loss2);
}

// A warp per row: the reference of its probabilities, the largest of the scores of its
// targets and of W's first f.sample rows.  fp16 probabilities (the halves of fp32 rows
// too) are kept 2^14 times as large, in steps of 2^-24, so that a tail of a million items
// of 2^-30 of the largest is still there; that leaves no room above one, and the sample
// is all of W.  bf16 has fp32's range: there a sample does, probabilities may be larger
// than one, and where they leave that range, which shows in the sums, the exact passes
// run (grad_h_kernel).  (Of fp32 rows it is the maximum of what the
// products hold: RowScale.)
template <typename T, int VEC>
__global__ void __launch_bounds__(256) reference_kernel(Many f) {
  const SoftmaxArgs& a = f.a;
  const int64_t t = (int64_t)blockIdx.x * 8 + threadIdx.x / 32;
  if (t >= a.n) return;
  const int64_t pos = f.s.pos[t];
  if (pos < 0) return;
  float m, l;
  merge_slots(f, pos, f.sample, f.high_tiles != 0 && high_halves_do(*f.s.words, a.b) ? f.high_tiles : f.shape.tiles, m, l);
  target_scores<T, VEC>(a, t, [&](int k, float q, float s) {
    if (f.sample < a.V) m = fmaxf(m, s);
    f.s.score[t * a.target.top + k] = s;
  });
  m = warp_max(m);
  // (fp32 rows: in sixteenths, so that 14 - m and -m are exact and dh and dw have the same
  // p.  16-bit rows: as it is, so that near a fit the target itself has p = 1, not rounded.)
  if (sizeof(T) == 4 && fabsf(m) <= kHuge) m = rintf(m * 16.f) * 0.0625f;
  if ((threadIdx.x & 31) == 0) f.s.row_max[pos] = m == -INFINITY ? 0.f : m;
}

// Sum of a row of partial gradients over the slots of its group, columns d ...
template <int VEC>
__device__ __forceinline__ void add_slots(const Many& f, int64_t rows_a, int64_t rows_b, int64_t row, int d, float (&x)[VEC]) {
  const Ranges r(rows_a, rows_b, f.shape.tiles, f.blocks);
  const int64_t g = row / (128 * f.shape.tiles), in = row - g * 128 * f.shape.tiles;
  const int64_t i0 = r.block_of(g * r.n_b), i1 = r.block_of((g + 1) * r.n_b - 1);
#pragma unroll
  for (int e = 0; e < VEC; ++e) x[e] = 0.f;
#pragma unroll 8
  for (int64_t i = i0; i <= i1; ++i) {
    float y[VEC];
    load_vec<float, VEC>(f.s.out + ((i + g) * f.shape.tiles * 128 + in) * f.ld + d, y);
#pragma unroll
    for (int e = 0; e < VEC; ++e) x[e] += y[e];
  }
}

// What rounding p to 16 bits took from the sum of a target's product.  Near a fit p - q
// is small beside p, and that rounding would be most of it (p = 0.99, q = 1: 0.004 of
// 0.01); other items' p are off by their own half-unit only.  (The score here and the
// tensor core's differ in their last bits, so now and then p rounds the other way there;
// past kHuge they have nothing in common, but there p is zero or one.)  Of a list that
// names an item more than once the first entry has it: p was rounded once.
template <typename T>
__device__ __forceinline__ float rounded_off(float p) {
  return sizeof(T) == 4 ? 0.f : p - to_float(from_float<T>(p));
}

// dh, a warp per row and 32 VEC columns: b weight (sum p w / l - sum q w_id).  After a pass by references
// (BY_REF) the row's sum and loss come first, and of bf16 rows a sum that is no number
// asks for the exact passes.
template <typename T, int VEC, bool BY_REF>
__global__ void __launch_bounds__(256) grad_h_kernel(Many f) {
  constexpr int kParts = sizeof(T) == 4 ? 2 : 1;
  constexpr bool kMayRedo = BY_REF && std::is_same<T, __nv_bfloat16>::value;
  const SoftmaxArgs& a = f.a;
  const int64_t t = (int64_t)blockIdx.x * 8 + threadIdx.x / 32;
  if (t >= a.n || (f.if_redo && f.s.words->redo == 0u)) return;
  const int64_t pos = f.s.pos[t];
  if (BY_REF && blockIdx.y == 0) {
    pad_cols<kParts>(f, t);
    if (pos < 0 && (threadIdx.x & 31) == 0) a.loss[t] = a.lse[t] = 0.f;
  }
  float row_sum = 1.f;
  if (BY_REF && pos >= 0) {
    const int lane = threadIdx.x & 31;
    const Ranges r(f.s.words->rows, a.V, 1, f.blocks);
    const int64_t g = pos / 128, i0 = r.block_of(g * r.n_b), i1 = r.block_of((g + 1) * r.n_b - 1);
    const float* sums = reinterpret_cast<const float*>(f.s.stat);
    float l = 0.f, loss2 = 0.f;
    for (int64_t i = 4 * i0 + lane; i < 4 * i1 + 4; i += 32) l += sums[((i / 4 + g) * 4 + (i & 3)) * 128 + (pos & 127)];
    row_sum = l = warp_sum(l) * exp2f(-f.up);
    const float lse2 = f.s.row_max[pos] + log2f(l);
    for (int64_t k = t * a.target.top + lane; k < (t + 1) * a.target.top; k += 32) {
      const float q = a.target.logits ? a.target.q[k] : 1.f;
      if (q != 0.f) loss2 += q * (lse2 - f.s.score[k]);
    }
    loss2 = warp_sum(loss2);
    if (lane == 0 && blockIdx.y == 0) {
      finish_row<kParts>(f, t, pos, f.s.row_max[pos], l, loss2);
      if (kMayRedo && !(l < 3e38f && l > 1e-30f)) f.s.words->redo = 1u;
    }
  } else if (pos >= 0) {
    row_sum = f.s.row_sum[pos];
  }
  T* to = static_cast<T*>(a.grad_h) + t * a.D;
  const float bw = pos < 0 ? 0.f : a.b * (a.weight ? a.weight[t] : 1.f);
  const float up = f.up;
  const int shift = (f.parts == 2 ? half_shift_of(f.s.words->max_w) : 0) + (int)up;
  const float inv = 1.f / row_sum, m = pos < 0 ? 0.f : f.s.row_max[pos];
  const int lane = threadIdx.x & 31, d = blockIdx.y * 32 * VEC + lane * VEC;
  const bool on = d < a.D;
  float x[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) x[e] = 0.f;
  if (pos >= 0) {
    if (on) add_slots<VEC>(f, f.s.words->rows, a.V, pos, d, x);
    if (kMayRedo) {
      bool fine = true;
#pragma unroll
      for (int e = 0; e < VEC; ++e) fine &= fabsf(x[e]) < 3e38f;
      if (!fine) f.s.words->redo = 1u;
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e) x[e] = ldexpf(x[e] * inv, -shift);
    for (int k0 = 0; k0 < a.target.top; k0 += 32) {
      const int count = min(32, a.target.top - k0);
      const int64_t entry = t * a.target.top + k0 + lane;
      const int32_t lane_id = lane < count ? a.target.ids[entry] : -1;
      float c = lane >= count ? 0.f : a.target.logits ? -a.target.q[entry] : -1.f;
      if (sizeof(T) == 2 && c != 0.f && fabsf(m) <= kHuge && !(a.target.top > 1 && f.s.again[entry])) c += ldexpf(rounded_off<T>(exp2_fast(f.s.score[entry] - m + up)) * inv, -shift);
      const unsigned share = __ballot_sync(0xffffffffu, c != 0.f);
#pragma unroll 4
      for (int i = 0; i < count; ++i) {
        const float ci = __shfl_sync(0xffffffffu, c, i);
        const int32_t id = __shfl_sync(0xffffffffu, lane_id, i);
        if (!on || !(share >> i & 1u)) continue;
        float y[VEC];
        load_vec<T, VEC>(static_cast<const T*>(a.w) + id * a.w_stride + d, y);
#pragma unroll
        for (int e = 0; e < VEC; ++e) x[e] = fmaf(ci, y[e], x[e]);
      }
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e) x[e] *= bw;
  }
  if (on) store_vec<T, VEC>(to + d, x);
}

// The targets as (item, entry) pairs; what has no share sorts behind the last item.
__global__ void entries_kernel(Many f) {
  const TargetArgs& a = f.a.target;
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= a.n * a.top) return;
  const uint32_t id = (uint32_t)a.ids[i];
  const bool share = id < (uint32_t)a.V && (!a.logits || a.q[i] != 0.f);
  f.s.key[0][i] = share ? id : (uint32_t)a.V;
  f.s.val[0][i] = (uint32_t)i;
}

// Whether the row of a sorted entry has named its item before.  The sort keeps the entries'
// order, so that a row's entries of one item lie side by side.
__device__ __forceinline__ bool named_again(const uint32_t* key, const uint32_t* val, int64_t i, uint32_t top) {
  return i > 0 && key[i - 1] == key[i] && val[i - 1] / top == val[i] / top;
}
__global__ void again_kernel(Many f, const uint32_t* key, const uint32_t* val) {
  const uint32_t top = (uint32_t)f.a.target.top;
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= f.a.n * top) return;
  f.s.again[val[i]] = named_again(key, val, i, top);
}

// First entry of every tile of 128 items.
__global__ void tile_first_kernel(Many f, const uint32_t* key) {
  const int64_t tiles = ((int64_t)f.a.V + 127) / 128, i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i > tiles) return;
  const uint32_t item = (uint32_t)min(i * 128, (int64_t)f.a.V);
  int64_t lo = 0, hi = f.a.n * f.a.target.top;
  while (lo < hi) {
    const int64_t mid = (lo + hi) / 2;
    if (key[mid] < item) lo = mid + 1;
    else hi = mid;
  }
  f.s.tile_first[i] = (int32_t)lo;
}

// The power of two by which an item's sum over columns is to be multiplied.
template <typename T>
__device__ __forceinline__ int item_shift(const Many& f, int64_t item) {
  const ManyWords& w = *f.s.words;
  return -(int)item_up<std::is_same<T, __nv_bfloat16>::value, sizeof(T) == 4 ? 2 : 1>(w, f.s.item_top, item) -
         (sizeof(T) == 4 ? half_shift_of(w.max_h) : 0);
}

// Of every entry in order of the items its row of H, and weight q less what rounding took.
template <typename T>
__global__ void factors_kernel(Many f, const uint32_t* key, const uint32_t* val, int32_t* row, float* factor) {
  const SoftmaxArgs& a = f.a;
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= a.n * a.target.top || key[i] == (uint32_t)a.V) return;
  const uint32_t entry = val[i];
  const int32_t t = (int32_t)(entry / (uint32_t)a.target.top);
  const float q = a.target.logits ? a.target.q[entry] : 1.f;
  float g = a.weight ? q * a.weight[t] : q;
  if (sizeof(T) == 2 && fabsf(f.s.row_max[f.s.pos[t]]) <= kHuge && !named_again(key, val, i, (uint32_t)a.target.top)) {
    const int shift = item_shift<T>(f, key[i]);
    g -= ldexpf(rounded_off<T>(col_probability(f, f.s.pos[t], f.s.score[entry], (float)-shift)), shift);
  }
  row[i] = t;
  factor[i] = g;
}
// x += g h_t [d ...] over the first `count` lanes' entries, all lanes taking part.
template <typename T, int VEC>
__device__ __forceinline__ void add_rows(const SoftmaxArgs& a, int count, int32_t lane_t, float lane_g, int d, float (&x)[VEC]) {
#pragma unroll 8
  for (int i = 0; i < count; ++i) {
    const float g = __shfl_sync(0xffffffffu, lane_g, i);
    const int64_t t = __shfl_sync(0xffffffffu, lane_t, i);
    if (d >= a.D) continue;
    float y[VEC];
    load_vec<T, VEC>(static_cast<const T*>(a.h) + t * a.h_stride + d, y);
#pragma unroll
    for (int e = 0; e < VEC; ++e) x[e] = fmaf(g, y[e], x[e]);
  }
}
template <int VEC>
__device__ __forceinline__ void add_sums(const float* sums, int32_t begin, int32_t end, int32_t D, int d, float (&x)[VEC]) {
  if (d < D)
#pragma unroll 4
    for (int32_t i = begin; i < end; ++i) {
      float y[VEC];
      load_vec<float, VEC>(sums + (int64_t)i * D + d, y);
#pragma unroll
      for (int e = 0; e < VEC; ++e) x[e] += y[e];
    }
}

// Sums over the runs of kRun entries (at multiples of kRun) that name one item, and of
// kRun such runs (level 1), a warp each: no item of dw then adds more than 30 rows, 30
// runs and what its entries make of runs of runs.
template <typename T, int VEC, int LEVEL>
__global__ void __launch_bounds__(256) runs_kernel(Many f, const uint32_t* key, const int32_t* row, const float* factor) {
  constexpr int kLong = LEVEL == 0 ? kRun : kRun * kRun;
  const SoftmaxArgs& a = f.a;
  const int64_t run = (int64_t)blockIdx.x * 8 + threadIdx.x / 32, first = run * kLong;
  const int lane = threadIdx.x & 31;
  if (first + kLong > a.n * a.target.top) return;
  if (key[first] != key[first + kLong - 1] || key[first] == (uint32_t)a.V) return;
  int32_t t = 0;
  float g = 0.f;
  if (LEVEL == 0 && lane < kRun) t = row[first + lane], g = factor[first + lane];
  const int d = blockIdx.y * 32 * VEC + lane * VEC;
  float x[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) x[e] = 0.f;
  if (LEVEL == 0)
    add_rows<T, VEC>(a, kRun, t, g, d, x);
  else
    add_sums<VEC>(f.s.run_sum[0], (int32_t)(run * kRun), (int32_t)(run * kRun + kRun), a.D, d, x);
  if (d < a.D) store_vec<float, VEC>(f.s.run_sum[LEVEL] + run * a.D + d, x);
}

// dw: b (sum weight p h - sum weight q h), some items to a block.  Most items are
// nobody's target: those rows go through all threads side by side, the others a warp
// each (2048 x 1M, K = 64: a warp for every item took 470 us, this 133).
// Items of a block: 16 where 64 would leave SMs idle, 64 up to 32 blocks of them per SM,
// else 128 (that case: a tenth less than by 64).
constexpr int kItems = 128;
template <typename T, int VEC>
__global__ void __launch_bounds__(256) grad_w_kernel(Many f, int per_block, const uint32_t* key, const int32_t* row,
                                                     const float* factor) {
  __shared__ int32_t first[kItems + 1];
  __shared__ int shifts[kItems];
  __shared__ int64_t slots[2];
  const SoftmaxArgs& a = f.a;
  const int64_t v0 = (int64_t)blockIdx.x * per_block, rows = f.s.words->rows;
  const int lane = threadIdx.x & 31, items = (int)min((int64_t)per_block, a.V - v0);
  if (threadIdx.x <= items) {
    int32_t lo = f.s.tile_first[v0 / 128], hi = f.s.tile_first[v0 / 128 + 1];
    while (lo < hi) {
      const int32_t mid = (lo + hi) / 2;
      if (key[mid] < (uint32_t)(v0 + threadIdx.x)) lo = mid + 1;
      else hi = mid;
    }
    first[threadIdx.x] = lo;
    if (threadIdx.x < items) shifts[threadIdx.x] = item_shift<T>(f, v0 + threadIdx.x);
  }
  if (threadIdx.x == 255) {  // (divisions, beside the searches)
    slots[0] = 1, slots[1] = 0;
    if (rows > 0) {
      const Ranges r(a.V, rows, 1, f.blocks);
      const int64_t g = v0 / 128;
      slots[0] = r.block_of(g * r.n_b) + g, slots[1] = r.block_of((g + 1) * r.n_b - 1) + g;
    }
  }
  __syncthreads();
  auto sum = [&](int item, int d, float (&x)[VEC]) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) x[e] = 0.f;
    for (int64_t s = slots[0]; s <= slots[1]; ++s) {
      float y[VEC];
      load_vec<float, VEC>(f.s.out + (s * 128 + v0 % 128 + item) * f.ld + d, y);
#pragma unroll
      for (int e = 0; e < VEC; ++e) x[e] += y[e];
    }
  };
  T* to = static_cast<T*>(a.grad_w) + v0 * a.D;
  const int slices = a.D / VEC;
  constexpr int U = 4;  // loads of a thread under way
  for (int i0 = threadIdx.x; i0 < items * slices; i0 += U * 256) {
    float x[U][VEC] = {};
    int from[U], shift[U];  // where in its slots; < 0: none, or an item with targets
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * 256, item = i / slices;
      from[u] = i < items * slices && first[item] == first[item + 1] ? item * f.ld + (i - item * slices) * VEC : -1;
      shift[u] = from[u] >= 0 ? shifts[item] : 0;
    }
    for (int64_t s = slots[0]; s <= slots[1]; ++s) {
      const float* part = f.s.out + (s * 128 + v0 % 128) * f.ld;
      float y[U][VEC] = {};
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (from[u] >= 0) load_vec<float, VEC>(part + from[u], y[u]);
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < VEC; ++e) x[u][e] += y[u][e];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (from[u] < 0) continue;
#pragma unroll
      for (int e = 0; e < VEC; ++e) x[u][e] = a.b * ldexpf(x[u][e], shift[u]);
      store_vec<T, VEC>(to + (i0 + u * 256) * VEC, x[u]);
    }
  }
  // (By item and 32 VEC columns.)
  const int chunks = (a.D + 32 * VEC - 1) / (32 * VEC);
  for (int part = threadIdx.x / 32; part < items * chunks; part += 8) {
    const int item = part / chunks, d = (part - item * chunks) * 32 * VEC + lane * VEC;
    const int32_t begin = first[item], end = first[item + 1];
    if (begin == end) continue;
    // Whole runs [r0, r1), whole runs of runs [q0, q1), and single entries at both ends, one per lane.
    int32_t r0 = (begin + kRun - 1) / kRun, r1 = end / kRun;
    int32_t head = r0 * kRun - begin, tail = end - r1 * kRun;
    if (r0 >= r1) r0 = r1 = 0, head = end - begin, tail = 0;
    int32_t q0 = (r0 + kRun - 1) / kRun, q1 = r1 / kRun;
    if (q0 >= q1) q0 = q1 = 0;
    int32_t t = 0;
    float g = 0.f;
    if (lane < head + tail) {
      const int32_t i = lane < head ? begin + lane : end - tail + lane - head;
      t = row[i], g = factor[i];
    }
    float x[VEC], y[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) x[e] = y[e] = 0.f;
    if (d < a.D) sum(item, d, x);
    add_rows<T, VEC>(a, head + tail, t, g, d, y);
    add_sums<VEC>(f.s.run_sum[0], r0, q0 < q1 ? q0 * kRun : r1, a.D, d, y);
    add_sums<VEC>(f.s.run_sum[0], q0 < q1 ? q1 * kRun : r1, r1, a.D, d, y);
    add_sums<VEC>(f.s.run_sum[1], q0, q1, a.D, d, y);
#pragma unroll
    for (int e = 0; e < VEC; ++e) x[e] = a.b * (ldexpf(x[e], shifts[item]) - y[e]);
    if (d < a.D) store_vec<T, VEC>(to + item * a.D + d, x);
  }
}

template <typename T>
bool rows_by(int vec, const SoftmaxArgs& a, bool grads) {
  auto ok = [&](const void* p, int64_t stride) { return stride % vec == 0 && reinterpret_cast<uintptr_t>(p) % (vec * sizeof(T)) == 0; };
  return a.D % vec == 0 && ok(a.h, a.h_stride) && ok(a.w, a.w_stride) && (!grads || (ok(a.grad_h, a.D) && ok(a.grad_w, a.D)));
}

template <typename T, int VEC>
void launch_units(const Many& f) {  // W's and H's
  auto padded = [](int64_t rows) { return (rows + 127) / 128 * 128; };
  if constexpr (sizeof(T) == 4) {
    // As many blocks as give each row of a thread its turn, or four to an SM.
    const int each = f.shape.nk == 1 ? 4 : f.shape.nk == 2 ? 2 : 1;
    auto blocks = [&](int64_t rows) {
      return (unsigned)std::max(padded(rows) / 32 / each, std::min<int64_t>(padded(rows) / 32, 4ll * f.a.sms));
    };
    const unsigned w = blocks(f.a.V), both = w + blocks(f.a.n);
    if (each == 4) units_f32_kernel<VEC, 1><<<both, 256, 0, f.a.st>>>(f, w);
    else if (each == 2) units_f32_kernel<VEC, 2><<<both, 256, 0, f.a.st>>>(f, w);
    else units_f32_kernel<VEC, 0><<<both, 256, 0, f.a.st>>>(f, w);
  } else {
    auto blocks = [&](int64_t rows) {
      return (unsigned)std::min<int64_t>((padded(rows) * f.shape.nk * 8 + 255) / 256, 32ll * f.a.sms);
    };
    const unsigned w = blocks(f.a.V);
    units_kernel<T, VEC><<<w + blocks(f.a.n), 256, 0, f.a.st>>>(f, w);
  }
}

int bits_of(uint32_t most) {
  int bits = 1;
  while (bits < 32 && (most >> bits)) ++bits;
  return bits;
}

template <typename T, int VEC>
cudaError_t run(const SoftmaxArgs& a, const ManyScratch& s) {
  constexpr int kParts = sizeof(T) == 4 ? 2 : 1;
  constexpr bool kBf16 = std::is_same<T, __nv_bfloat16>::value;
  const bool grads = a.grad_h != nullptr;
  const unsigned by_row = (unsigned)((a.n + 7) / 8), col_chunks = (unsigned)((a.D + 32 * VEC - 1) / (32 * VEC));
  Many f{a, s, mma_shape(Pass::kStats, a.D, kParts), a.sms, (a.D + 15) / 16 * 16, kParts, 0, 0.f, 0, 0};
  if (!grads) f.s.col = nullptr;
  cudaError_t e = cudaMemsetAsync(s.words, 0, sizeof(ManyWords), a.st);
  if (e != cudaSuccess) return e;
  // The targets by item, on the handle's second stream beside what follows.
  const bool join_early = sizeof(T) == 2 && a.target.top > 1 && !a.target.again;  // (dh asks for repeats)
  auto join = [&] { return cudaStreamWaitEvent(a.st, s.join, 0); };
  const int64_t entries = a.n * a.target.top, tiles = ((int64_t)a.V + 127) / 128;
  cub::DoubleBuffer<uint32_t> key(s.key[0], s.key[1]), val(s.val[0], s.val[1]);
  // (The sort leaves one of its buffers of each pair free.)
  int32_t* entry_row = nullptr;
  float* entry_factor = nullptr;
  auto launch_runs = [&](cudaStream_t st) {
    entry_row = reinterpret_cast<int32_t*>(val.Alternate()), entry_factor = reinterpret_cast<float*>(key.Alternate());
    factors_kernel<T><<<(unsigned)((entries + 255) / 256), 256, 0, st>>>(f, key.Current(), val.Current(), entry_row, entry_factor);
    if (entries >= kRun)
      runs_kernel<T, VEC, 0>
          <<<dim3((unsigned)((entries / kRun + 7) / 8), col_chunks), 256, 0, st>>>(f, key.Current(), entry_row, entry_factor);
    if (entries >= kRun * kRun)
      runs_kernel<T, VEC, 1>
          <<<dim3((unsigned)((entries / kRun / kRun + 7) / 8), col_chunks), 256, 0, st>>>(f, key.Current(), entry_row, entry_factor);
  };
  if (grads) {
    if ((e = cudaEventRecord(s.fork, a.st)) != cudaSuccess || (e = cudaStreamWaitEvent(s.side, s.fork, 0)) != cudaSuccess) return e;
    entries_kernel<<<(unsigned)((entries + 255) / 256), 256, 0, s.side>>>(f);
    size_t bytes = s.sort_bytes;
    if ((e = cub::DeviceRadixSort::SortPairs(s.sort_tmp, bytes, key, val, (int)entries, 0, bits_of((uint32_t)a.V), s.side)) !=
        cudaSuccess)
      return e;
    tile_first_kernel<<<(unsigned)(tiles / 256 + 1), 256, 0, s.side>>>(f, key.Current());
    if (sizeof(T) == 4) launch_runs(s.side);
    else if (join_early)
      again_kernel<<<(unsigned)((entries + 255) / 256), 256, 0, s.side>>>(f, key.Current(), val.Current());
    if ((e = cudaEventRecord(s.join, s.side)) != cudaSuccess) return e;
  }
  const int64_t n_w = ((int64_t)a.V + 127) / 128;
  const bool large = n_w >= 32 && (a.n + 127) / 128 * n_w >= 24ll * a.sms;
  const MmaShape high_shape = mma_shape(Pass::kMax, a.D, 1);
  if (kParts == 2 && large) f.high_tiles = high_shape.tiles;
  compact_kernel<<<(unsigned)((a.n + 1023) / 1024), 1024, 0, a.st>>>(f);
  if constexpr (kParts == 2) {
    const int64_t work = std::max((int64_t)a.V, a.n) * a.D / VEC;
    max_kernel<VEC><<<dim3((unsigned)std::min<int64_t>((work + 255) / 256, 8ll * a.sms), 2), 256, 0, a.st>>>(f);
  }
  launch_units<T, VEC>(f);

  MmaArgs m{};
  m.A = s.units_h, m.B = s.units_w, m.scale_a = s.scale_h, m.scale_b = s.scale_w, m.words = s.words, m.V = a.V, m.b = a.b;
  m.row_max = s.row_max, m.col = s.col, m.col_m = s.col_m, m.col_f = s.col_f, m.stat = s.stat, m.out = s.out, m.ld = f.ld;
  m.status = a.target.status;
  // Tiles between additions in fp32.  4096 x 18k, K = 100, lists of 32: dh is 1.0e-6 off
  // with 32 tiles, 5.8e-7 with 16, 3.4e-7 with 8 (7.5e-7 by fp32 products of whole
  // matrices); the call takes as long with any of the three, to 1%.  Where the small
  // products of halves have no sums of their own, half as many tiles.
  const MmaShape stats_shape = mma_shape(Pass::kStats, a.D, kParts), rows_shape = mma_shape(Pass::kRows, a.D, kParts);
  const int out_chunks = (a.D + 255) / 256, run_tiles = kParts == 1 ? 128 : rows_shape.cross ? 16 : 8;
  // Maxima, of large problems of fp32 rows by high halves where that does.
  auto maxima = [&](Pass pass) {
    m.s = stats_shape, m.high = high_shape, m.try_high = kParts == 2 && large, m.run = INT32_MAX;
    return launch_mma(pass, kBf16, kParts, m, a.sms, 1, a.st);
  };
  // Maxima (and sums) over W's first `items` rows, and what is made of them.
  auto stats = [&](Pass pass, int32_t items, int if_redo) {
    f.shape = m.s = stats_shape, f.if_redo = m.if_redo = if_redo, m.V = items, m.run = INT32_MAX;
    const cudaError_t err = pass == Pass::kMax ? maxima(pass) : launch_mma(pass, kBf16, kParts, m, a.sms, 1, a.st);
    m.V = a.V;
    return err;
  };
  auto rows = [&](bool by_ref, int if_redo) {
    f.shape = m.s = rows_shape, f.if_redo = m.if_redo = if_redo, m.run = run_tiles;
    f.up = m.up = kBf16 ? 0.f : kHalfShift;
    m.sums = by_ref ? reinterpret_cast<float*>(s.stat) : nullptr;
    return launch_mma(Pass::kRows, kBf16, kParts, m, a.sms, out_chunks, a.st);
  };
  auto exact = [&](int if_redo) {
    cudaError_t err = stats(Pass::kStats, a.V, if_redo);
    if (err != cudaSuccess) return err;
    loss_kernel<T, VEC><<<by_row, 256, 0, a.st>>>(f);
    if constexpr (kBf16) {
      if (grads) {
        if ((err = rows(false, if_redo)) != cudaSuccess || (join_early && (err = join()) != cudaSuccess)) return err;
        grad_h_kernel<T, VEC, false><<<dim3(by_row, col_chunks), 256, 0, a.st>>>(f);
      }
    }
    return cudaGetLastError();
  };
  // A pass over all scores of bf16 rows for their maxima alone is a fifth of the work.
  // Where it is more than that of the launches that stand by (about 10 us), references
  // from a sixteenth of W do, and the exact passes run only if one of them was too low.
  const bool sampled = kBf16 && large;
  if (grads && (sampled || !kBf16)) {
    f.sample = sampled ? (int32_t)(128 * (n_w / 16)) : a.V;
    if ((e = stats(Pass::kMax, f.sample, 0)) != cudaSuccess) return e;
    reference_kernel<T, VEC><<<by_row, 256, 0, a.st>>>(f);
    if ((e = rows(true, 0)) != cudaSuccess || (join_early && (e = join()) != cudaSuccess)) return e;
    grad_h_kernel<T, VEC, true><<<dim3(by_row, col_chunks), 256, 0, a.st>>>(f);
    if (sampled && (e = exact(1)) != cudaSuccess) return e;
  } else if ((e = exact(0)) != cudaSuccess) {
    return e;
  }
  if (!grads) return cudaSuccess;
  m.if_redo = f.if_redo = 0;

  if (!join_early && (e = join()) != cudaSuccess) return e;
  m.A = s.units_w, m.B = s.units_h, m.scale_a = s.scale_w, m.scale_b = s.scale_h, m.item_top = s.item_top;
  if (!kBf16) {
    m.if_apart = kParts == 1, m.col = kParts == 2 ? s.col_top : s.col;
    if (kParts == 2 && large) {
      m.low = &s.words->low;
      if ((e = maxima(Pass::kMaxCols)) != cudaSuccess) return e;
      m.low = nullptr, m.if_low = 1;
    }
    if ((e = maxima(Pass::kMaxCols)) != cudaSuccess) return e;
    m.s = rows_shape, m.run = run_tiles, m.col = s.col;
  }
  if (sizeof(T) == 2) launch_runs(a.st);  // (wants the rows' sums and the items' references)
  if ((e = launch_mma(Pass::kCols, kBf16, kParts, m, a.sms, out_chunks, a.st)) != cudaSuccess) return e;
  const int per_block = (int64_t)a.V < 64ll * 8 * a.sms ? 16 : (int64_t)a.V < 64ll * 32 * a.sms ? 64 : kItems;
  grad_w_kernel<T, VEC><<<(unsigned)(((int64_t)a.V + per_block - 1) / per_block), 256, 0, a.st>>>(f, per_block, key.Current(),
                                                                                           entry_row, entry_factor);
  return cudaGetLastError();
}

}  // namespace

ManySizes many_sizes(int64_t rows, int64_t V, int32_t D, int32_t dtype, int64_t top, bool backward, int sms) {
  ManySizes z{};
  const int parts = dtype == ESSPT_F32 ? 2 : 1;
  const MmaShape stats = mma_shape(Pass::kStats, D, parts), grads = mma_shape(Pass::kRows, D, parts);
  const int64_t tile_bytes = (int64_t)grads.nk * parts * kUnitBytes;
  auto groups = [](int64_t n, int tiles) { return (n + 128 * tiles - 1) / (128 * tiles); };
  z.units_h = (size_t)((rows + 127) / 128 * tile_bytes);
  z.units_w = (size_t)((V + 127) / 128 * tile_bytes);
  z.stat = (size_t)(groups(rows, stats.tiles) + sms) * 512 * sizeof(float2);
  if (!backward) return z;
  const int64_t slots = std::max(groups(rows, grads.tiles), groups(V, grads.tiles)) + sms;
  z.out = (size_t)slots * grads.tiles * 128 * ((D + 15) / 16 * 16) * sizeof(float);
  cub::DoubleBuffer<uint32_t> none(nullptr, nullptr);
  cub::DeviceRadixSort::SortPairs(nullptr, z.sort, none, none, (int)(rows * top), 0, bits_of((uint32_t)V));
  for (int i = 0, run = kRun; i < 2; ++i, run *= kRun) z.run_sum[i] = (size_t)(rows * top / run + 1) * D * sizeof(float);
  return z;
}

cudaError_t launch_many_rows(const SoftmaxArgs& a, const ManyScratch& s) {
  const bool grads = a.grad_h != nullptr;
  if (a.dtype == ESSPT_BF16) return rows_by<__nv_bfloat16>(4, a, grads) ? run<__nv_bfloat16, 4>(a, s) : run<__nv_bfloat16, 1>(a, s);
  if (a.dtype == ESSPT_F16) return rows_by<__half>(4, a, grads) ? run<__half, 4>(a, s) : run<__half, 1>(a, s);
  return rows_by<float>(4, a, grads) ? run<float, 4>(a, s) : run<float, 1>(a, s);
}

}  // namespace esspt
