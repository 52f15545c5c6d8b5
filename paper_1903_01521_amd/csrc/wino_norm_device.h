// Device helpers of the norm, the checkpoint and the weight gradient.
#pragma once

#include <math.h>

#include "wino_norm.h"

namespace wino {

constexpr float kCodes = 127.0f;
constexpr float kFlat = 0x1p-100f;            // half ranges below this: the channel is kept as its centre

template <typename T, int V>
struct alignas(sizeof(T) * V) Raw {
    T v[V];
};

// The channel's part of the norm, and the checkpoint's.  Every step is rounded:
// the sign of z, which decides ReLU's gradient, is then the same in the forward
// and the backward pass.
struct Affine {
    float mean, rstd, gamma, beta;
    __device__ __forceinline__ float norm(float x) const {
#pragma clang fp contract(off)
        return (x - mean) * rstd;
    }
    __device__ __forceinline__ float z(float n) const {
#pragma clang fp contract(off)
        return n * gamma + beta;
    }
};

__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.0f + __expf(-z)); }

template <Act ACT>
__device__ __forceinline__ float act_of(float z) {
    if constexpr (ACT == Act::Relu) return z < 0.0f ? 0.0f : z;        // NaN stays
    if constexpr (ACT == Act::Silu) return z * sigmoid(z);
    return z;
}

template <Act ACT>
__device__ __forceinline__ float dact(float z, float dy) {
    if constexpr (ACT == Act::Relu) return z > 0.0f ? dy : 0.0f;
    if constexpr (ACT == Act::Silu) {
        const float s = sigmoid(z);
        return dy * (s * (1.0f + z * (1.0f - s)));
    }
    return dy;
}

// Checkpoint row of a channel from its range: centre, step and 1 / step.
struct Row {
    float centre, step, inverse;
};
__device__ __forceinline__ Row row_of(float lo, float hi) {
#pragma clang fp contract(off)
    const float half = 0.5f * hi - 0.5f * lo;
    Row r;
    r.centre = 0.5f * lo + 0.5f * hi;
    r.step = half < kFlat ? 0.0f : half / kCodes;
    r.inverse = half < kFlat ? 0.0f : kCodes / half;
    return r;
}
__device__ __forceinline__ int8_t code_of(float x, const Row& r) {
#pragma clang fp contract(off)
    const float q = rintf((x - r.centre) * r.inverse);
    return (int8_t)(int)fminf(fmaxf(q, -kCodes), kCodes);
}
__device__ __forceinline__ float value_of(int8_t code, float centre, float step) {
#pragma clang fp contract(off)
    return (float)code * step + centre;
}

}  // namespace wino
