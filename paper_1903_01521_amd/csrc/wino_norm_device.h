// Device helpers of the norm, the checkpoint and the weight gradient.
#pragma once

#include <math.h>

#include <type_traits>

#include "wino_fastdiv.h"
#include "wino_norm.h"

namespace wino {

constexpr float kCodes = 127.0f;
constexpr float kFlat = 0x1p-100f;            // half ranges below this: the channel is kept as its centre

template <typename T, int V>
struct alignas(sizeof(T) * V) Raw {
    T v[V];
};

// A result that is not read again here goes past the caches' normal order, so that
// what is read again stays there (norm, N = 64, 256 channels at 56x56, in three
// launches: 133 us, with this and get() 106).
template <typename T, int V>
__device__ __forceinline__ void put(T* p, const Raw<T, V>& o) {
    if constexpr (sizeof(T) * V >= 4) {
        typedef uint32_t V4 __attribute__((ext_vector_type(sizeof(T) * V / 4)));
        __builtin_nontemporal_store(__builtin_bit_cast(V4, o), (V4*)p);
        return;
    }
    *(Raw<T, V>*)p = o;
}

// V values as loaded, in registers of their own: pin() keeps the compiler from
// also keeping them converted, from one use to the next.
template <typename T, int V>
struct Held {
    static constexpr int kBytes = sizeof(T) * V, kWords = (kBytes + 3) / 4;
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const T* p) {
        if constexpr (kBytes == 1) w[0] = *(const uint8_t*)p;
        else if constexpr (kBytes == 2) w[0] = *(const uint16_t*)p;
        else {
            const Raw<uint32_t, kWords> r = *(const Raw<uint32_t, kWords>*)p;
#pragma unroll
            for (int i = 0; i < kWords; ++i) w[i] = r.v[i];
        }
    }
    // the last read of these values
    __device__ __forceinline__ void get(const T* p) {
        if constexpr (kBytes >= 4) {
            typedef uint32_t V4 __attribute__((ext_vector_type(kWords)));
            const V4 r = __builtin_nontemporal_load((const V4*)p);
#pragma unroll
            for (int i = 0; i < kWords; ++i) w[i] = r[i];
        } else {
            load(p);
        }
    }
    __device__ __forceinline__ void pin() {
#pragma unroll
        for (int i = 0; i < kWords; ++i) asm volatile("" : "+v"(w[i]));
    }
    __device__ __forceinline__ float value(int j) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[j]);
        else if constexpr (sizeof(T) == 1) return (float)(int8_t)(w[j / 4] >> (j % 4 * 8));
        else if constexpr (std::is_same<T, _Float16>::value)
            return (float)__builtin_bit_cast(_Float16, (uint16_t)(w[j / 2] >> (j % 2 * 16)));
        else return __uint_as_float(j % 2 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16);
    }
};

__device__ __forceinline__ float rstd_of(float var, float eps) { return 1.0f / sqrtf(var + eps); }
__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.0f + __expf(-z)); }

// The activation's argument z and its normalised value n from a stored value v, x
// itself or a code, for one channel.  The mean is subtracted first, so that a mean far
// from zero costs no bits: of x itself, and of a checkpoint's centre.  SiLU of a code:
// one fused operation on folded constants.  ReLU or none: every step of the definition
// is rounded, so that the sign of z, which decides ReLU's gradient, is the same in both
// passes.
template <bool SILU, bool X8>
struct Norm {
    float scale, shift, gamma, beta, mean, rstd, centre, step;
    __device__ __forceinline__ void set(const float* stats, float g, float b, const float* row) {
        mean = stats[0];
        rstd = stats[1];
        gamma = g;
        beta = b;
        centre = X8 ? row[0] : 0.0f;
        step = X8 ? row[1] : 1.0f;
        if constexpr (SILU && X8) {
            scale = rstd * step;
            shift = (centre - mean) * rstd;
        }
    }
    __device__ __forceinline__ float n(float v) const {
#pragma clang fp contract(off)
        if constexpr (SILU && X8) return fmaf(v, scale, shift);
        const float x = X8 ? v * step + centre : v;
        return (x - mean) * rstd;
    }
    __device__ __forceinline__ float z(float n) const {
#pragma clang fp contract(off)
        if constexpr (SILU) return fmaf(n, gamma, beta);
        return n * gamma + beta;
    }
};

// y of z
template <bool SILU>
__device__ __forceinline__ float act_of(float z, bool relu) {
    if constexpr (SILU) return z * sigmoid(z);
    return relu && z < 0.0f ? 0.0f : z;                                // NaN stays
}

// dz of z and dy
template <bool SILU>
__device__ __forceinline__ float act_grad(float z, float dy, bool relu) {
    if constexpr (SILU) {
        const float s = sigmoid(z);
        return dy * fmaf(z * s, 1.0f - s, s);
    }
    return !relu || z > 0.0f ? dy : 0.0f;
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
// The code is the low byte: adding 1.5 * 2^23 rounds to an integer, ties to even.  The
// centre's rounding takes one end of a range of a few units in its last place past 127
// (three units: to 169), hence the limits, which keep NaN.
__device__ __forceinline__ uint32_t code_bits(float x, float centre, float inverse) {
#pragma clang fp contract(off)
    const float q = __builtin_elementwise_maximum(__builtin_elementwise_minimum((x - centre) * inverse, kCodes), -kCodes);
    return __float_as_uint(q + 12582912.0f);
}
template <int V>
__device__ __forceinline__ void store_codes(int8_t* p, const uint32_t (&b)[V]) {
    if constexpr (V == 1) *p = (int8_t)b[0];
    else {
        const uint32_t lo = __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(b[3], b[2], 0x04000c0cu);
        *(uint32_t*)p = lo | hi;
    }
}
__device__ __forceinline__ float value_of(float code, float centre, float step) {
#pragma clang fp contract(off)
    return code * step + centre;
}

}  // namespace wino
