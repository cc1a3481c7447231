// checks.h -- what the argument checks behind the C ABI share (host side).
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/fastbfp.h"

namespace fastbfp {

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

inline int status_of(hipError_t e) { return e == hipSuccess ? BFP_OK : BFP_E_HIP; }

// Whether the `an` bytes at a and the `bn` bytes at b share any (null: nothing there).
inline bool overlap(const void* a, uint64_t an, const void* b, uint64_t bn) {
  const uint64_t p = reinterpret_cast<uintptr_t>(a), q = reinterpret_cast<uintptr_t>(b);
  return a && b && (p < q ? q - p < an && bn > 0 : p - q < bn && an > 0);
}

}  // namespace fastbfp
