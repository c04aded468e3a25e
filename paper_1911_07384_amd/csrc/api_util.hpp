// Argument checks and status conversion shared by the C ABI's translation units.
#pragma once

#include "../../include/fp16train.h"

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace fp16k {

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

inline bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  if (!a || !b || na == 0 || nb == 0) return false;
  const uintptr_t pa = (uintptr_t)a, pb = (uintptr_t)b;
  return pa < pb + nb && pb < pa + na;
}

inline size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }

inline fp16_status hip_status(hipError_t e) { return e == hipSuccess ? FP16_OK : FP16_ERR_HIP; }

#define TRY(expr)                                  \
  do {                                             \
    const hipError_t e_ = (expr);                  \
    if (e_ != hipSuccess) return FP16_ERR_HIP;     \
  } while (0)

}  // namespace fp16k
