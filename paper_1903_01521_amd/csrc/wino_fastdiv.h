// Division by a number fixed at launch.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace wino {

// Division of n < 2^31 by a fixed d >= 1 as ((mulhi(n, m) + n) >> l), with
// l = ceil(log2 d) and m = floor(2^32 (2^l - d) / d) + 1 (Granlund and
// Montgomery's round-up method; mulhi(n, m) + n < 2^32 for such n).
struct FastDiv {
    uint32_t m;
    int l;
};

inline FastDiv make_fastdiv(uint32_t d) {
    FastDiv f;
    f.l = 0;
    while ((1ull << f.l) < d) ++f.l;
    f.m = (uint32_t)(((1ull << 32) * ((1ull << f.l) - d)) / d + 1);
    return f;
}

__device__ __forceinline__ uint32_t fdiv(uint32_t n, FastDiv d) { return (__umulhi(n, d.m) + n) >> d.l; }

}  // namespace wino
