// Host-side argument checks shared by the C ABI's source files.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/mbscan.h"

namespace mbscan {

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

struct Range {
    uintptr_t lo, hi;
};
inline Range range_of(const void *p, int64_t bytes) {   // a null pointer is an empty range
    uintptr_t a = reinterpret_cast<uintptr_t>(p);
    return Range{a, p ? a + (uintptr_t)(bytes > 0 ? bytes : 0) : a};
}
inline bool overlap(Range a, Range b) { return a.lo < b.hi && b.lo < a.hi && a.lo != a.hi && b.lo != b.hi; }

// Products of sizes must stay far from int64 overflow and inside the
// 32-bit element counts the kernels assume for token tensors.
constexpr int64_t kMaxTokens = (int64_t)1 << 31;

inline mb_status from_cuda(cudaError_t e) { return e == cudaSuccess ? MB_OK : MB_ERR_CUDA; }

}  // namespace mbscan
