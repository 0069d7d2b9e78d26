// What the layer norm's translation units share: its arguments, and how rows are spread over threads.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace esspt {

constexpr int kNormThreads = 256;   // of a block whose rows take a warp or less
constexpr int kNormValues = 16;     // of a thread, at most; of a wide row's all have so many
constexpr int kNormWidth = 8192;    // of a row
constexpr int kNormWide = kNormWidth / kNormValues;  // threads of a wide row's block

struct Norm {
  const void *x, *dy;
  int64_t x_stride, dy_stride, n;
  int32_t D;
  int32_t lanes;  // threads of a row: a power of two up to 32, or the block
  float inv_D, eps;
  const void *weight, *bias;
  int weight_f32;  // their type, where it is not the rows'
  void* y;        // dx in the backward pass
  float *mean, *rstd;
  float* part;    // [blocks][2][D] sums for dw and db
  int want_w;     // whether they are asked for
};

// How rows of D values are spread over threads: those of a block and of a row, vectors of a thread (N), and
// blocks of an SM.
struct Spread {
  int threads, lanes, n, resident;
  bool wide;
};
inline Spread spread(int D, int vec, bool back) {
  const int vectors = (D + vec - 1) / vec, most = kNormValues / vec;
  Spread s{kNormThreads, 32, 1, 0, false};
  if (vectors <= 32 * most) {
    while (s.n * 32 < vectors) s.n *= 2;
    while (s.lanes / 2 >= vectors && s.lanes > 1) s.lanes /= 2;
  } else {
    s.n = most;
    s.threads = s.lanes = ((vectors + most - 1) / most + 31) / 32 * 32;
    s.wide = true;
  }
  // by registers: up to 64 with eight values; with 16 up to 80 (vectors of four or eight, forward), 128.  (60000 rows of 1002
  // bf16 values, in pairs, forward: 57 us, with 768 threads 68.)
  s.resident = (s.n * vec <= 8 ? 1024 : vec >= 4 && !back ? 768 : 512) / s.threads;
  return s;
}

// Rows of `bytes`-byte vectors, all of which alignment allows; *blocks: how many were launched, with their sums in a.part.
template <typename T>
cudaError_t launch_norm(Norm& a, bool back, int bytes, int sms, unsigned* blocks, cudaStream_t st);

}  // namespace esspt
