// Declarations shared by the softmax operators' translation units (cross entropy
// and distillation over a catalogue; see include/esspt.h for the mathematics).
// Scores are kept in units of log 2 throughout: s2 = s / ln 2.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "esspt.h"

namespace esspt {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr uint32_t kErrTarget = 1u;  // a target or id >= V (status word)
constexpr uint32_t kErrStuck = 2u;   // a wait inside a kernel ran out (never expected)
constexpr int kFewRows = ESSPT_SOFTMAX_FEW_ROWS;

// The target of every row: one item (ids[t], q = 1: logits is null), or a list.
struct TargetArgs {
  const int32_t* ids;    // [n, top]
  const float* logits;   // [n, top], or null: cross entropy
  int32_t top;
  int64_t n;
  int32_t V;
  float b;               // inverse temperature
  float* q;              // [n, top] out (lists only): the entries' shares, 0 where absent
  float* self;           // [n] out (lists only): sum q log q, or kIgnored
  uint32_t* status;
  uint8_t* again;        // [n, top] out, or null: whether the row named the entry's item before
};
// Lists up to this long have their repeats found by the row's warp, entries 32 by 32 with
// those before them, which grows with the square of the length; longer ones by the sorted
// entries, which dh then waits for.  (4001 rows, lists of 64 over 200k items, bf16: calls of
// 575 and 600 us, for the sort runs in the gaps between the passes.)
constexpr int kAgainByWarp = 256;
constexpr float kIgnored = 3.0e38f;  // (sum q log q is never positive)

struct SoftmaxArgs {
  const void *h, *w;
  int64_t h_stride, w_stride, n;
  int32_t V, D, dtype;
  TargetArgs target;
  const float* weight;   // [n] or null
  float b;
  float *loss, *lse;     // [n]
  void *grad_h, *grad_w; // null: forward alone
  cudaStream_t st;
  int sms;
};

// Up to kFewRows rows, and small problems of up to kSmallRows, by scores kept in the
// workspace, in groups of kFewRows rows.
constexpr int kSmallRows = 128;
struct FewScratch {
  float* scores;   // [groups][V][kFewRows]
  float2* part;    // [few_blocks or groups][kFewRows] maximum and sum of a block's items
  float* stat;     // [rows][2] maximum of a row and 1 / sum
  float* dh;       // [few_blocks or groups][kFewRows][D]
  uint32_t* done;  // [groups] blocks of a group that have ended; 0 between calls
};
int few_blocks(int sms);

// Many rows: operands in 16 KB units of 128 rows by 64 16-bit values (tensor.cuh);
// fp32 values in two halves of 11 bits (x = hi + lo, both fp16), so that three products of
// halves give fp32's.  H and W are scaled by a power of two each, and a row that is more
// than 2^8 below its matrix's largest value by a second one of its own (RowScale): a value
// is held to 2^-40 of its row's largest, or to 2^-32, whatever the other rows are.
struct ManyWords {  // (device) what a call's kernels tell each other
  uint32_t max_h, max_w, max_weight;  // largest finite magnitude, as fp32 bits
  uint32_t min_weight;                // smallest but zero, as its distance below infinity
  int32_t rows;                       // rows that are not ignored
  uint32_t negative;                  // whether one of their weights is
  uint32_t redo;                      // a row's reference was too low: the exact passes run
  uint32_t huge;                      // a row's reference is past kHuge
  uint32_t spread_h, spread_w;        // whether any row has a power of its own
  uint32_t norm_h, norm_w;            // (fp32) largest sum of a row's squares, by the matrix's power
  uint32_t low;                       // (fp32) an item's weight p are all below kLow of the largest weight, or may be
};
struct RowScale {  // units hold the row 1 / c times as large as the matrix's power alone says
  float c, log2_c;
};
struct ManyScratch {
  ManyWords* words;
  int32_t *act, *pos;      // [n] the kept rows in order; a row's place among them, or -1
  char *units_h, *units_w;
  RowScale *scale_h, *scale_w;  // (fp32) of the kept rows and of W, up to whole tiles
  float *row_max, *row_sum;  // [n] statistics of the kept rows, in order
  float *col, *col_top, *col_m, *col_f;  // [2 (n up to 128)], [n up to 128] the kept rows as columns of dw: see MmaArgs
  uint32_t* item_top;        // [V] an item's largest log2 of weight p over the rows (top_key); fp32 and fp16
  float* score;              // [n * top] scores of the targets
  float2* stat;              // partial statistics and
  float* out;                // partial gradients by slot (Ranges, softmax_mma.cuh)
  uint32_t *key[2], *val[2]; // [n * top] entries by item
  uint8_t* again;            // [n * top] TargetArgs (lists of 16-bit rows)
  int32_t* tile_first;       // [tiles of W + 1] first entry of a tile's items
  float* run_sum[2];         // [n * top / kRun (^2) + 1][D] sums over whole runs of one item
  void* sort_tmp;
  size_t sort_bytes;
  cudaStream_t side;         // the targets are sorted beside the scores
  cudaEvent_t fork, join;
};
constexpr int kRun = 16;

// Sizes of the above.
struct ManySizes {
  size_t units_h, units_w, stat, out, sort, run_sum[2];  // bytes
};
ManySizes many_sizes(int64_t rows, int64_t V, int32_t D, int32_t dtype, int64_t top, bool backward, int sms);
cudaError_t launch_many_rows(const SoftmaxArgs& a, const ManyScratch& s);

cudaError_t launch_targets(const TargetArgs& a, cudaStream_t st);
// Whether a call of n rows goes by scores kept (launch_few_rows).
bool few_rows(int64_t n, int64_t V, int32_t D, int32_t dtype, bool grads);
int few_groups(int64_t max_rows, int64_t V, int32_t D, int32_t dtype, bool backward);  // most groups of such a call
cudaError_t launch_few_rows(const SoftmaxArgs& a, const FewScratch& s);

}  // namespace esspt
