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
};
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

// Up to kFewRows rows at once, by scores kept in the workspace.
struct FewScratch {
  float* scores;   // [V][kFewRows]
  float2* part;    // [few_blocks][kFewRows] maximum and sum of a block's items
  float* stat;     // [kFewRows][2] maximum of a row and 1 / sum
  float* dh;       // [few_blocks][kFewRows][D]
  float* dw;       // [V][D] running gradient, or null where one group is all
};
int few_blocks(int sms);

cudaError_t launch_targets(const TargetArgs& a, cudaStream_t st);
cudaError_t launch_few_rows(const SoftmaxArgs& a, const FewScratch& s);

}  // namespace esspt
