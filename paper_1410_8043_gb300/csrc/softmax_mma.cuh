// The tensor-core kernel of the softmax operators: scores of 128 x 128 tiles, and
// what follows from them in one pass, on operands in units (tensor.cuh).
#pragma once

#include "softmax.cuh"
#include "tensor.cuh"

namespace esspt {

// What a pass makes of the scores S = A B^T b / ln 2:
//   kStats  per row of A the maximum and the sum of 2^(S - maximum)
//   kMax    per row of A the maximum (of S c of the columns' RowScale: what the products hold)
//   kMaxCols  A = W, B = H: the maximum of S + col over B's rows, an item's over all blocks
//   kRows   A = H, B = W: sum over B's rows of 2^(S - row_max) B, and of 2^(S - row_max);
//           with RowScale, 2^(S - row_max) c meets the tensor cores, at most one as row_max is kMax's
//   kCols   A = W, B = H: sum over B's rows t of 2^(S - maximum_t) factor_t B
enum class Pass { kStats, kMax, kMaxCols, kRows, kCols };
__host__ __device__ constexpr bool only_scores(Pass pass) {
  return pass == Pass::kStats || pass == Pass::kMax || pass == Pass::kMaxCols;
}
__host__ __device__ constexpr bool items_first(Pass pass) { return pass == Pass::kMaxCols || pass == Pass::kCols; }

constexpr int kUnits = 13;             // units of shared memory
constexpr float kHalfShift = 14.f;     // fp16 probabilities: the largest is kept as 2^14
// Scores this far from zero (in units of log 2) are rounded before the row's maximum is
// taken off.  Below, one fused operation does both, and what is off is the rounding of
// the maximum, 2^-14 at most.  Above, S b less a rounded maximum would be off by half a
// unit of it: by 512 at 10^10, where all of a row's probabilities became zero or infinite.
// Rounded first, the best item's difference is zero, as all passes form the same sums in
// the same order.
constexpr float kHuge = 1024.f;
// Column data of a tile in shared memory lies in slots of its own, by turns.  Where the
// scores alone are wanted (kMaxCols), a tile's stage is free before its columns were
// read: by then at most five more tiles' scores are done, each block of eight warps
// having two of the buffers and taking part in every second tile of a group.
constexpr int kTopSlots = 8;           // slots beyond the stages, for that
constexpr int kMmaThreads = 640;       // a warp that loads, one that multiplies, two spare, two groups of eight

// How a pass uses shared and tensor memory: A's units stay (res) or come with every
// tile of B, for one or two tiles of A at once (tiles); a stage of the ring holds
// stage_units; B is kept from the scores to the sums (keep) or loaded again for them;
// `buffers` tiles of scores are in tensor memory.
//
// Up to two units a row (t), a stage is a tile of B.  Above, stages are units: a tile
// of B is then never waited for as a whole (K = 256, bf16: with two stages of 64 KB a
// tile waited 940 of 3150 cycles); or pairs of units, half as many waits, where two
// tiles of four fit (4096 x 18k, K = 100, fp32: 251 and 238 us for the call).  Two tiles
// of A share B where only the scores are wanted and three units are left for it; with
// sums, a third buffer of scores is worth more than sharing (4001 x 200k, K = 64, bf16:
// 295 and 222 us for the rows pass).
struct MmaShape {
  int nk, steps;       // units and 16-value steps of a row
  int tiles, res, keep;
  int stage_units, stages, buffers;
  int cross;           // sums of products of halves hi lo and lo hi have columns of their own
};
__host__ __device__ constexpr MmaShape mma_shape(Pass pass, int32_t D, int parts) {
  MmaShape s{};
  s.steps = (D + 15) / 16;
  s.nk = (D + 63) / 64;
  const int t = s.nk * parts;
  const bool stats = only_scores(pass);
  s.tiles = stats && 2 * t + 3 <= kUnits ? 2 : 1;
  s.res = s.tiles == 2 || t + (parts == 2 ? 4 : 3) <= kUnits;
  s.keep = s.res && 3 * t <= kUnits;
  s.stage_units = t <= 2 ? t : t == 4 && !stats ? 2 : 1;
  s.stages = (kUnits - (s.res ? s.tiles * t : 0)) / s.stage_units;
  s.buffers = stats ? 4 : t <= 2 ? 3 : 2;
  s.cross = !stats && parts == 2 && s.nk <= 2;
  return s;
}

struct MmaArgs {
  const char *A, *B;
  const RowScale *scale_a, *scale_b;  // fp32 rows
  MmaShape s;
  const ManyWords* words;
  int32_t V;
  float b;
  const float* row_max;  // kRows
  // kCols, fp32 rows: two columns to a float4, (-maximum, -maximum, factor, factor); of
  // 16-bit rows a float to a column, log2 |factor| - maximum with the sign as its lowest bit.
  // kMaxCols: the latter for fp32 rows too.
  const float* col;
  const float *col_m, *col_f;  // kMaxCols, kCols: -maximum and factor by themselves
  uint32_t* item_top;    // kMaxCols out, kCols: ManyScratch
  int if_apart;          // only where weights_apart
  MmaShape high;         // kMax, kMaxCols of fp32 rows: for the high halves alone, where `try_high`
  int try_high;          // and high_halves_do
  uint32_t* low;         // kMaxCols: over B's first tile alone, to find what words->low says
  int if_low;            // only where words->low is set
  float2* stat;          // kStats, kMax out: [slot][4][128], by group and half of the columns
  float* sums;           // kRows out: sums of the probabilities, likewise, or null
  float up;              // kRows: probabilities are taken 2^up times as large
  int if_redo;           // only where words->redo is set
  float* out;            // kRows, kCols: [slot][128][ld]
  int ld;
  int run;               // tiles of B that the tensor core sums up before fp32 does
  uint32_t* status;
};

// Work is the sequence of all (group of A's tiles, tile of B), cut into one even range
// per block, so that no SM waits whatever the two sizes are; block i's part of group g goes to slot i + g, and the slots of a
// group are consecutive.
struct Ranges {
  int64_t groups, n_b, units, blocks;
  __host__ __device__ Ranges(int64_t rows_a, int64_t rows_b, int tiles, int64_t grid) {
    groups = (rows_a + 128 * tiles - 1) / (128 * tiles);
    n_b = (rows_b + 127) / 128;
    units = groups * n_b;
    blocks = grid < units ? grid : units;
  }
  __host__ __device__ int64_t begin(int64_t i) const { return units * i / blocks; }
  __host__ __device__ int64_t block_of(int64_t unit) const { return ((unit + 1) * blocks - 1) / units; }
};

// Scaling of fp32 operands: x 2^shift has its largest value in [2^14, 2^15), and so has
// a row of its own scale.
__device__ __forceinline__ int half_shift_of(uint32_t max_bits) {
  return max_bits == 0u ? 0 : 14 - ((int)(max_bits >> 23) - 127);
}
__device__ __forceinline__ float times_pow2(float x, int e) {
  const int e1 = e / 2;
  return x * __int_as_float((e1 + 127) << 23) * __int_as_float((e - e1 + 127) << 23);
}
// Maxima only decide powers of two that probabilities are taken times, with room for a
// factor of two.  The high halves give them where what they leave out of a score, 2^-10 of
// |h| |w| at most, is below one in units of log 2; a third of the products then.  (2048 x
// 1M, K = 64: a call of 3.66 ms with exact maxima.)
__device__ __forceinline__ bool high_halves_do(const ManyWords& w, float b) {
  const float most = sqrtf(__uint_as_float(w.norm_h)) * sqrtf(__uint_as_float(w.norm_w));
  return w.spread_h == 0u && w.spread_w == 0u &&
         ldexpf(most * (b * kLog2e), -(half_shift_of(w.max_h) + half_shift_of(w.max_w)) - 10) < 1.f;
}
// Log2 of the weight p, relative to the largest weight, that one power of two for all items
// still serves: halves of p in steps of 2^-39 then are 2^-15 of it.
constexpr float kLow = -24.f;
// Whether the rows' weights differ by more than 2^8.
__device__ __forceinline__ bool weights_apart(const ManyWords& w) {
  return w.max_weight != 0u && (int)(w.max_weight >> 23) - (int)((0x7f800000u - w.min_weight) >> 23) > 8;
}
// Floats in their order as whole numbers; 0 is below all.
__device__ __forceinline__ uint32_t top_key(float x) {
  const uint32_t u = __float_as_uint(x);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
// The power of two that an item's terms weight p are multiplied by in the sum over rows.
// fp32 rows, whose result has fp32's range: by the item's own largest term, for what is
// left of an item that is nobody's target may be 2^-40 and less of what a target gets.
// In large problems a tile of rows tells whether any item needs that (`low`; small ones
// set it), else one power for all does, by the largest weight (2048 x 1M, K = 64: the maxima
// of all take 320 us of 3190).  fp16 rows: the result has no such values, and that one
// power does unless the weights differ much, so that ordinary rows' share is small.
template <bool BF16, int PARTS>
__device__ __forceinline__ float item_up(const ManyWords& w, const uint32_t* top, int64_t item) {
  if (BF16) return 0.f;
  if (PARTS == 2 ? w.low == 0u : !weights_apart(w))
    return w.max_weight == 0u ? kHalfShift : kHalfShift - 1.f - (float)((int)(w.max_weight >> 23) - 127);
  const uint32_t key = top[item];
  if (key == 0u) return 0.f;
  const float m = __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
  return fminf(fmaxf(kHalfShift - ceilf(m), -100.f), 100.f);
}

cudaError_t launch_mma(Pass pass, bool bf16, int parts, const MmaArgs& a, int blocks, int out_chunks, cudaStream_t st);

}  // namespace esspt
