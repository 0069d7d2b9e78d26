// What the handles of the operators on rows share: where errors are kept, alignment.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>
#include <stdio.h>

#include "esspt.h"

namespace esspt {

struct Errors {
  char text[256] = "";
  esspt_status fail(esspt_status code, const char* why) {
    snprintf(text, sizeof(text), "%s", why);
    return code;
  }
  esspt_status cuda(cudaError_t e, const char* where) {
    snprintf(text, sizeof(text), "%s: %s", where, cudaGetErrorString(e));
    return ESSPT_ECUDA;
  }
};

#define ESSPT_CUDA(errors, call)                             \
  do {                                                       \
    cudaError_t e_ = (call);                                 \
    if (e_ != cudaSuccess) return (errors).cuda(e_, #call);  \
  } while (0)

inline bool misaligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }
inline size_t size_of(int dtype) { return dtype == ESSPT_F32 ? 4 : 2; }
inline size_t up256(size_t bytes) { return (bytes + 255) & ~size_t(255); }

// Bytes of the vectors that rows of `width` values can be read in, whose addresses and
// distances are those: the largest of 16, 8, 4 and 2 that divides all of them.
inline int vector_bytes(int64_t width, size_t size, uintptr_t addresses_and_strides) {
  const uintptr_t all = (uintptr_t)(width * size) | addresses_and_strides | 16;
  return (int)(all & (~all + 1));
}

}  // namespace esspt
