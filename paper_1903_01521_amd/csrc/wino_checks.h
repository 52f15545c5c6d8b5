// Argument checks shared by the C-ABI's source files.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "wino.h"

namespace wino {

constexpr int64_t kMaxElems = (int64_t)1 << 40;      // per tensor, well inside size_t

// Checked product of non-negative int64 values; false on overflow past kMaxElems.
inline bool mul_ok(int64_t a, int64_t b, int64_t* out) {
    if (a < 0 || b < 0) return false;
    if (a != 0 && b > kMaxElems / a) return false;
    *out = a * b;
    return *out <= kMaxElems;
}

inline bool overlap(const void* a, size_t na, const void* b, size_t nb) {
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return x < y + nb && y < x + na;
}

inline size_t round_up(size_t v, size_t a) { return (v + a - 1) / a * a; }
inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
inline int hip_status(hipError_t e) { return e == hipSuccess ? WINO_OK : WINO_ERR_HIP; }

}  // namespace wino
