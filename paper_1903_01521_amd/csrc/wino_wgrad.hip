// Weight gradient of the 3x3 stride-1 layer on channel-last tensors:
//   dg[k][c][r][s] = sum over n, i, j of a[n][i + r - pad][j + s - pad][c] dy[n][i][j][k]
// with a the layer's input, read as zero outside the image: x, a checkpoint's
// values, or act(norm(either)) formed on load.
#include <math.h>

#include <type_traits>

#include "wino_norm_device.h"
#include "wino_wgrad.h"

namespace wino {

namespace {

// a at (n, pixel, c)
template <typename T, bool X8, bool NORM>
__device__ __forceinline__ float a_value(const WgradArgs& a, const WgradShape& s, int n, int64_t pixel, int c) {
    const size_t at = ((size_t)n * s.H * s.W + pixel) * s.C + c;
    float v;
    if constexpr (X8) {
        const float* r = a.rows + ((size_t)n * s.C + c) * 2;
        v = value_of((float)a.codes[at], r[0], r[1]);
    } else {
        v = (float)((const T*)a.x)[at];
    }
    if constexpr (NORM) {
        const float* st = a.stats + ((size_t)n * s.G + c / s.D) * 2;
        Norm<false, false> f;
        f.set(st, a.gamma ? a.gamma[c] : 1.0f, a.beta ? a.beta[c] : 0.0f, nullptr);
        const float z = f.z(f.n(v));
        v = s.act == Act::Silu ? act_of<true>(z, false) : act_of<false>(z, s.act == Act::Relu);
    }
    return v;
}

// 16 channels x 16 filters a workgroup, a thread a pair; rows of the batch
// [r0, r1) by slice; part [slices][9][C][K].
template <typename T, bool X8, bool NORM>
__global__ __launch_bounds__(256) void k_wgrad(WgradArgs a, WgradShape s, float* part, int slices) {
    __shared__ float la[3][18][16], ld[16][16];
    const int kt = (s.K + 15) / 16, ct = (s.C + 15) / 16;
    const int slice = blockIdx.x / (kt * ct), tile = blockIdx.x % (kt * ct);
    const int c0 = tile / kt * 16, k0 = tile % kt * 16;
    const int lo = threadIdx.x & 15, hi = threadIdx.x >> 4;
    const int64_t all = (int64_t)s.N * s.Ho, r0 = all * slice / slices, r1 = all * (slice + 1) / slices;
    float acc[9] = {};
    for (int64_t row = r0; row < r1; ++row) {
        const int n = (int)(row / s.Ho), i = (int)(row % s.Ho);
        for (int j0 = 0; j0 < s.Wo; j0 += 16) {
            __syncthreads();
            for (int e = threadIdx.x; e < 3 * 18 * 16; e += 256) {
                const int c = c0 + e % 16, col = j0 + e / 16 % 18 - s.pad, y = i + e / (16 * 18) - s.pad;
                const bool in = c < s.C && col >= 0 && col < s.W && y >= 0 && y < s.H;
                la[e / (16 * 18)][e / 16 % 18][e % 16] =
                    in ? a_value<T, X8, NORM>(a, s, n, (int64_t)y * s.W + col, c) : 0.0f;
            }
            const int j = j0 + hi, k = k0 + lo;
            ld[hi][lo] = j < s.Wo && k < s.K
                             ? (float)((const T*)a.dy)[(((size_t)n * s.Ho + i) * s.Wo + j) * s.K + k]
                             : 0.0f;
            __syncthreads();
            for (int p = 0; p < 16; ++p) {
                const float d = ld[p][lo];
#pragma unroll
                for (int t = 0; t < 9; ++t) acc[t] += la[t / 3][p + t % 3][hi] * d;
            }
        }
    }
    const int c = c0 + hi, k = k0 + lo;
    if (c < s.C && k < s.K)
        for (int t = 0; t < 9; ++t) part[(((size_t)slice * 9 + t) * s.C + c) * s.K + k] = acc[t];
}

// dg = the slices' sum, to [K][C][3][3].
__global__ __launch_bounds__(256) void k_wgrad_sum(const float* __restrict__ part, float* __restrict__ dg, int C, int K,
                                                   int slices) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, all = (int64_t)9 * C * K;
    if (i >= all) return;
    const int64_t kc = i / 9, t = i % 9, k = kc / C, c = kc % C;
    float v = 0.0f;
    for (int sl = 0; sl < slices; ++sl) v += part[(((size_t)sl * 9 + t) * C + c) * K + k];
    dg[i] = v;
}

int slices_of(const WgradShape& s) {
    const int64_t tiles = (int64_t)((s.K + 15) / 16) * ((s.C + 15) / 16), rows = (int64_t)s.N * s.Ho;
    int64_t n = tiles >= 2048 ? 1 : 2048 / tiles;
    return (int)(n < rows ? n : rows);
}

}  // namespace

size_t wgrad_workspace(const WgradShape& s) { return (size_t)slices_of(s) * 9 * s.C * s.K * sizeof(float); }

hipError_t launch_wgrad(const WgradArgs& a, const WgradShape& s, void* ws, hipStream_t st) {
    const int slices = slices_of(s);
    const unsigned grid = (unsigned)slices * ((s.K + 15) / 16) * ((s.C + 15) / 16);
    auto go = [&](auto t) {
        typedef decltype(t) T;
        if (s.x8 && s.norm) k_wgrad<T, true, true><<<grid, 256, 0, st>>>(a, s, (float*)ws, slices);
        else if (s.x8) k_wgrad<T, true, false><<<grid, 256, 0, st>>>(a, s, (float*)ws, slices);
        else if (s.norm) k_wgrad<T, false, true><<<grid, 256, 0, st>>>(a, s, (float*)ws, slices);
        else k_wgrad<T, false, false><<<grid, 256, 0, st>>>(a, s, (float*)ws, slices);
    };
    if (s.io == Io::F32) go(float());
    else if (s.io == Io::F16) go(_Float16());
    else go(__bf16());
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t all = (int64_t)9 * s.C * s.K;
    k_wgrad_sum<<<(unsigned)((all + 255) / 256), 256, 0, st>>>((const float*)ws, a.dg, s.C, s.K, slices);
    return hipGetLastError();
}

}  // namespace wino
