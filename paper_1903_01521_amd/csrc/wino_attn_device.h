// Device side of the attention kernels: operands of eight values, tiles in LDS, the
// kernels themselves as templates over the element type and the head's width.
//
// All products run on 32x32 matrix-core tiles.  A lane l of a wave holds column
// l % 32 of a result and, with h = l / 32, its rows 8 b + 4 h + i (b, i < 4).  Scores
// are formed transposed, keys down and rows across (or, for dk and dv, rows down and
// keys across), so that the sums of a softmax run inside a lane and its partner
// l ^ 32, a row's largest score, sum and factors are one register of that lane, and
// the result is the next product's right operand as it is: a sum does not depend on the
// order of its terms, so the left operand is read in the order in which the lanes hold
// theirs, 16 terms as {4 h + i} and {8 + 4 h + i}.
#pragma once

#include <math.h>

#include <type_traits>

#include "wino_attn.h"
#include "wino_fastdiv.h"

namespace wino {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4v __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

// x of this lane and of lane ^ 32
__device__ __forceinline__ void halves(float x, float& a, float& b) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    a = __uint_as_float(r[0]);
    b = __uint_as_float(r[1]);
}
__device__ __forceinline__ float max_halves(float x) {
    float a, b;
    halves(x, a, b);
    return fmaxf(a, b);
}
__device__ __forceinline__ float add_halves(float x) {
    float a, b;
    halves(x, a, b);
    return a + b;
}

// ---------------------------------------------------------------- operands
// Eight values of a lane: 16 terms of a product, eight each in the wave's halves.

template <typename T>
struct Frag {
    typedef T V __attribute__((ext_vector_type(8)));
    V v;
};
template <>
struct Frag<float> {
    float v[8];
};

__device__ __forceinline__ f32x16 mma(const Frag<__bf16>& a, const Frag<__bf16>& b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v, b.v, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma(const Frag<_Float16>& a, const Frag<_Float16>& b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a.v, b.v, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma(const Frag<float>& a, const Frag<float>& b, f32x16 c) {
#pragma unroll
    for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[j], b.v[j], c, 0, 0, 0);
    return c;
}

// Values 8 at .. 8 at + 7 of a result as an operand, rounded once to T.
template <typename T>
__device__ __forceinline__ Frag<T> pack(const f32x16& s, int at) {
    Frag<T> f;
#pragma unroll
    for (int j = 0; j < 8; ++j) f.v[j] = (T)s[8 * at + j];
    return f;
}

// ---------------------------------------------------------------- tiles in LDS
// Rows of W = 16 D16 values (up to a power of two), in 16-byte chunks whose place is
// xored with bits of the row, so that 16 rows' chunk of the same number lie in
// different banks (read(), a row for each lane) and four rows' 64 bytes too (turned(),
// the transposing read of four rows by 16 columns).

template <typename T, int D16>
struct Tile {
    static constexpr int kP2 = D16 <= 2 ? 2 : D16 <= 4 ? 4 : 8;
    static constexpr int kRow = kP2 * 16 * (int)sizeof(T);          // bytes
    static constexpr int kChunks = D16 * (int)sizeof(T);            // used 16-byte chunks of a row
    static constexpr int kEach = 16 / (int)sizeof(T);               // values of a chunk

    __device__ static __forceinline__ int twist(int row) {
        if constexpr (kRow == 64) return (row >> 2) & 3;
        else if constexpr (kRow == 128) return ((row & 2) << 1) | ((row >> 2) & 3);
        else return ((row & 3) << 2) | ((row >> 2) & 3);
    }
    __device__ static __forceinline__ int at(int row, int chunk) { return row * kRow + ((chunk ^ twist(row)) << 4); }

    // values 16 c + 8 h .. + 7 of row `row`
    __device__ static __forceinline__ Frag<T> read(const char* t, int row, int c, int h) {
        Frag<T> f;
        if constexpr (sizeof(T) == 2) {
            f.v = __builtin_bit_cast(typename Frag<T>::V, *(const uint4*)(t + at(row, 2 * c + h)));
        } else {
            const f32x4v a = *(const f32x4v*)(t + at(row, 4 * c + 2 * h));
            const f32x4v b = *(const f32x4v*)(t + at(row, 4 * c + 2 * h + 1));
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                f.v[j] = a[j];
                f.v[4 + j] = b[j];
            }
        }
        return f;
    }
    // column 32 db + lane % 32 of rows r + {4 h + i} and r + 8 + {4 h + i} (turned), or of
    // rows r + 8 h .. + 7, read()'s order of terms (turned8); r a multiple of 16
    __device__ static __forceinline__ Frag<T> turned(const char* t, int r, int db, int lane) {
        return turned_by<4, 8>(t, r, db, lane);
    }
    __device__ static __forceinline__ Frag<T> turned8(const char* t, int r, int db, int lane) {
        return turned_by<8, 4>(t, r, db, lane);
    }
    template <int HALF, int NEXT>
    __device__ static __forceinline__ Frag<T> turned_by(const char* t, int r, int db, int lane) {
        Frag<T> f;
        const int h = lane >> 5;
        if constexpr (sizeof(T) == 2) {
            const int row = r + HALF * h + ((lane >> 2) & 3), chunk = 4 * db + ((lane >> 3) & 2) + ((lane >> 1) & 1);
            const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(t + at(row, chunk) + (lane & 1) * 8));
            const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(t + at(row + NEXT, chunk) + (lane & 1) * 8));
            typedef short s16x8 __attribute__((ext_vector_type(8)));
            f.v = __builtin_bit_cast(typename Frag<T>::V, (s16x8)__builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            const int c = 32 * db + (lane & 31);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int row = r + HALF * h + (j & 3) + NEXT * (j >> 2);
                f.v[j] = *(const float*)(t + at(row, c >> 2) + (c & 3) * 4);
            }
        }
        return f;
    }
};

// ---------------------------------------------------------------- global memory

// Values d .. d + each - 1 of a vector of D values at p; those past D are zero.  vec:
// p and D allow whole 16-byte words.
template <typename T>
__device__ __forceinline__ uint4 load_chunk(const T* p, int d, int D, bool vec) {
    constexpr int kEach = 16 / (int)sizeof(T);
    if (vec) return d < D ? *(const uint4*)(p + d) : make_uint4(0, 0, 0, 0);
    T v[kEach];
#pragma unroll
    for (int j = 0; j < kEach; ++j) v[j] = d + j < D ? p[d + j] : (T)0.0f;
    uint4 r;
    __builtin_memcpy(&r, v, 16);
    return r;
}

// Values 16 c + 8 h .. + 7 of the vector at p; zeros where p is null.
template <typename T>
__device__ __forceinline__ Frag<T> load_frag(const T* p, int c, int h, int D, bool vec) {
    uint4 r[sizeof(T) / 2];
    constexpr int kEach = 16 / (int)sizeof(T);
#pragma unroll
    for (int j = 0; j < (int)sizeof(T) / 2; ++j)
        r[j] = p ? load_chunk(p, 16 * c + 8 * h + j * kEach, D, vec) : make_uint4(0, 0, 0, 0);
    Frag<T> f;
    __builtin_memcpy(&f.v, r, sizeof(r));
    return f;
}

// Four neighbouring values of a result to p + d, those below D.
template <typename T>
__device__ __forceinline__ void store4(T* p, int d, int D, bool vec, float a, float b, float c, float e) {
    const T v[4] = {(T)a, (T)b, (T)c, (T)e};
    if (vec) {
        if (d < D) __builtin_memcpy(__builtin_assume_aligned(p + d, 4 * sizeof(T)), v, sizeof(v));
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (d + j < D) p[d + j] = v[j];
}

// A tile of `R` rows on its way: loaded to registers while the one before is worked on.
template <typename T, int D16, int R, int NT>
struct Moving {
    using Tl = Tile<T, D16>;
    static constexpr int kAll = R * Tl::kChunks, kMine = (kAll + NT - 1) / NT;
    uint4 w[kMine];
    // ptr(row): the row's vector, or null for zeros
    template <typename F>
    __device__ __forceinline__ void load(F ptr, int D, bool vec) {
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const int idx = threadIdx.x + i * NT, row = idx / Tl::kChunks, ch = idx % Tl::kChunks;
            const T* p = kAll % NT == 0 || idx < kAll ? ptr(row) : nullptr;
            w[i] = p ? load_chunk(p, ch * Tl::kEach, D, vec) : make_uint4(0, 0, 0, 0);
        }
    }
    __device__ __forceinline__ void store(char* t) const {
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const int idx = threadIdx.x + i * NT, row = idx / Tl::kChunks, ch = idx % Tl::kChunks;
            if (kAll % NT == 0 || idx < kAll) *(uint4*)(t + Tl::at(row, ch)) = w[i];
        }
    }
};

// ---------------------------------------------------------------- work

// Workgroups that share an image's keys (or rows) follow each other on one XCD, whose
// L2 then holds them: workgroup ids go round the eight XCDs.  Item of `all`, or -1.
__device__ __forceinline__ int64_t item_of(int64_t all) {
    const int64_t each = (all + 7) / 8, i = (int64_t)(blockIdx.x & 7) * each + (blockIdx.x >> 3);
    return (blockIdx.x >> 3) < each && i < all ? i : -1;
}

struct AttnK {
    AttnShape s;
    AttnArgs a;
    AttnBwd b;
    int64_t items, tiles;                    // of this launch; item = (pair * tiles + tile) * splits + split
    int splits;
    float *delta, *part, *part2, *stat;
    bool vec;
    FastDiv rep;                             // by s.rep; rows are below 2^31
};

// token and head of row `row` of a pair
struct RowAt {
    int64_t tok;                             // n * Lq + t
    int t, head;
};
__device__ __forceinline__ RowAt row_at(const AttnK& g, int n, int hk, int64_t row) {
    const int t = (int)fdiv((uint32_t)row, g.rep);
    return {(int64_t)n * g.s.Lq + t, t, hk * g.s.rep + (int)row - t * g.s.rep};
}

// keys of image n
__device__ __forceinline__ int keys_of(const int* klen, int n, int Lk) {
    return klen ? min(max(klen[n], 0), Lk) : Lk;
}

// part `split` of `n` in whole steps of `step`
__device__ __forceinline__ void part_of(int64_t n, int step, int split, int splits, int64_t& lo, int64_t& hi) {
    const int64_t each = ((n + step - 1) / step + splits - 1) / splits * step;
    lo = min(each * split, n);
    hi = min(lo + each, n);
}

// ---------------------------------------------------------------- forward
// One pass over the keys with a running maximum and sum.  The maximum moves, and what
// is summed is scaled, only where it grows by more than 2^8: exponentials stay below
// 2^8, and most tiles skip the scaling.  kFew: the NW waves share 32 rows and take 32
// keys of a tile each, and join at the end (single tokens: memory bound).

template <typename T, int D16, bool kFew>
struct FwdCut {
    static constexpr int kWaves = kFew && sizeof(T) == 4 ? 2 : 4;
    static constexpr int kKeys = kFew ? 32 * kWaves : 64;
    static constexpr int kRows = kFew ? 32 : 32 * kWaves;
    static constexpr int kThreads = 64 * kWaves;
};

template <typename T, int D16, bool kFew>
__global__ __launch_bounds__((FwdCut<T, D16, kFew>::kThreads)) void k_attn(AttnK g) {
    using Cut = FwdCut<T, D16, kFew>;
    using Tl = Tile<T, D16>;
    constexpr int NT = Cut::kThreads, KT = Cut::kKeys, KB = kFew ? 1 : KT / 32, DB = (D16 + 1) / 2;
    __shared__ alignas(16) char sk[KT * Tl::kRow];
    __shared__ alignas(16) char sv[KT * Tl::kRow];
    __shared__ alignas(16) float bias[KT];
    const AttnShape& s = g.s;
    const int64_t item = item_of(g.items);
    if (item < 0) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5;
    const int split = (int)(item % g.splits);
    const int64_t tile = item / g.splits % g.tiles, pair = item / g.splits / g.tiles;
    const int n = (int)(pair / s.Hk), hk = (int)(pair % s.Hk);
    const int64_t row = tile * Cut::kRows + (kFew ? 0 : wave * 32) + (lane & 31);
    const bool live = row < s.rows;
    const RowAt me = row_at(g, n, hk, row);
    const T* q = live ? (const T*)g.a.q + me.tok * s.ldq + (int64_t)me.head * s.D : nullptr;
    Frag<T> fq[D16];
#pragma unroll
    for (int c = 0; c < D16; ++c) fq[c] = load_frag(q, c, h, s.D, g.vec);

    int64_t lo, hi;
    const int len = keys_of(g.a.klen, n, s.Lk);
    part_of(len, KT, split, g.splits, lo, hi);
    const T* kbase = (const T*)g.a.k + (int64_t)n * s.Lk * s.ldk + (int64_t)hk * s.D;
    const T* vbase = (const T*)g.a.v + (int64_t)n * s.Lk * s.ldv + (int64_t)hk * s.D;
    const uint8_t* mask = g.a.mask ? g.a.mask + (int64_t)n * s.Lk : nullptr;

    Moving<T, D16, KT, NT> mk, mv;
    float mb = 0.0f;
    auto load = [&](int64_t k0) {
        auto kept = [&](int r) { return k0 + r < hi && (!mask || mask[k0 + r]); };
        mk.load([&](int r) { return kept(r) ? kbase + (k0 + r) * s.ldk : nullptr; }, s.D, g.vec);
        mv.load([&](int r) { return kept(r) ? vbase + (k0 + r) * s.ldv : nullptr; }, s.D, g.vec);
        if (threadIdx.x < KT) mb = kept(threadIdx.x) ? 0.0f : -INFINITY;
    };

    const float c2 = s.scale * kLog2e, slack = fminf(8.0f / c2, 0x1p127f);
    float top = -INFINITY, sum = 0.0f;
    f32x16 o[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) o[d] = f32x16{};
    if (lo < hi) load(lo);
    for (int64_t k0 = lo; k0 < hi; k0 += KT) {
        __syncthreads();
        mk.store(sk);
        mv.store(sv);
        if (threadIdx.x < KT) bias[threadIdx.x] = mb;
        __syncthreads();
        const bool whole = !mask && k0 + KT <= hi;
        if (k0 + KT < hi) load(k0 + KT);
        const int kb0 = kFew ? wave : 0;
        f32x16 p[KB];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            p[kb] = f32x16{};
#pragma unroll
            for (int c = 0; c < D16; ++c) p[kb] = mma(Tl::read(sk, (kb0 + kb) * 32 + (lane & 31), c, h), fq[c], p[kb]);
        }
        if (!whole) {
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    const f32x4v m = *(const f32x4v*)&bias[(kb0 + kb) * 32 + 8 * b + 4 * h];
#pragma unroll
                    for (int i = 0; i < 4; ++i) p[kb][4 * b + i] += m[i];
                }
        }
        float mx = p[0][0];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i) mx = fmaxf(mx, p[kb][i]);
        mx = max_halves(mx);
        if (__any(mx > top + slack)) {
            const float to = fmaxf(top, mx), a = to == top ? 1.0f : __builtin_amdgcn_exp2f((top - to) * c2);
            top = to;
            sum *= a;
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] *= a;
        }
        const float off = top == -INFINITY ? 0.0f : -top * c2;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                p[kb][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[kb][i], c2, off));
                sum += p[kb][i];
            }
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const Frag<T> f = pack<T>(p[kb], e);
#pragma unroll
                for (int d = 0; d < DB; ++d) o[d] = mma(Tl::turned(sv, (kb0 + kb) * 32 + 16 * e, d, lane), f, o[d]);
            }
    }
    sum = add_halves(sum);
    if constexpr (kFew) {
        // the waves' sums over their keys, by way of LDS: sk holds a wave's 32 rows at a time
        __shared__ float st[Cut::kWaves][32][2];
        static_assert(sizeof(sk) >= 32 * 32 * sizeof(float));
        if (h == 0) {
            st[wave][lane][0] = top;
            st[wave][lane][1] = sum;
        }
        __syncthreads();
        float all = -INFINITY;
#pragma unroll
        for (int w = 0; w < Cut::kWaves; ++w) all = fmaxf(all, st[w][lane & 31][0]);
        sum = 0.0f;
        const float base = all == -INFINITY ? 0.0f : all;
#pragma unroll
        for (int w = 0; w < Cut::kWaves; ++w)
            sum += st[w][lane & 31][1] * __builtin_amdgcn_exp2f((st[w][lane & 31][0] - base) * c2);
        const float a = __builtin_amdgcn_exp2f((top - base) * c2);
        top = all;
        float* x = (float*)sk;
#pragma unroll
        for (int d = 0; d < DB; ++d)
            for (int w = 0; w < Cut::kWaves; ++w) {
                if (wave == w) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int e = (8 * (i >> 2) + 4 * h + (i & 3)) * 32 + (lane & 31);
                        x[e] = (w ? x[e] : 0.0f) + o[d][i] * a;
                    }
                }
                __syncthreads();
                if (w == Cut::kWaves - 1 && wave == 0) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[d][i] = x[(8 * (i >> 2) + 4 * h + (i & 3)) * 32 + (lane & 31)];
                }
                __syncthreads();
            }
        if (wave) return;
    }
    if (!live) return;
    if (g.splits > 1) {
        const int64_t id = ((int64_t)split * s.N * s.Hk + pair) * s.rows + row;
        float* part = g.part + id * s.D;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int b = 0; b < 4; ++b)
                store4(part, 32 * d + 8 * b + 4 * h, s.D, (s.D & 3) == 0, o[d][4 * b], o[d][4 * b + 1], o[d][4 * b + 2],
                       o[d][4 * b + 3]);
        if (h == 0) {
            g.stat[id * 2] = top;
            g.stat[id * 2 + 1] = sum;
        }
        return;
    }
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    T* y = (T*)g.a.y + (me.tok * s.Hq + me.head) * s.D;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int b = 0; b < 4; ++b)
            store4(y, 32 * d + 8 * b + 4 * h, s.D, g.vec, o[d][4 * b] * inv, o[d][4 * b + 1] * inv, o[d][4 * b + 2] * inv,
                   o[d][4 * b + 3] * inv);
    if (g.a.lse && h == 0)
        g.a.lse[((int64_t)n * s.Hq + me.head) * s.Lq + me.t] =
            sum == 0.0f ? -INFINITY : __builtin_fmaf(top, s.scale, __builtin_amdgcn_logf(sum) * kLn2);
}

// The parts of a row: y = sum w o / sum w l with w = 2^(top - the largest top).  A
// workgroup's 256 threads are 256 / D rows; each thread one value of a row.
template <typename T>
__global__ __launch_bounds__(256) void k_attn_join(AttnK g) {
    const AttnShape& s = g.s;
    const int per = 256 / s.D, r = threadIdx.x / s.D, d = threadIdx.x % s.D;
    const int64_t all = (int64_t)s.N * s.Hk * s.rows, id = (int64_t)blockIdx.x * per + r;
    if (r >= per || id >= all) return;
    const float c2 = s.scale * kLog2e;
    float top = -INFINITY, sum = 0.0f, o = 0.0f;
    for (int i = 0; i < g.splits; ++i) top = fmaxf(top, g.stat[(i * all + id) * 2]);
    const float base = top == -INFINITY ? 0.0f : top;
    for (int i = 0; i < g.splits; ++i) {
        const int64_t at = i * all + id;
        const float w = __builtin_amdgcn_exp2f((g.stat[at * 2] - base) * c2);
        sum = __builtin_fmaf(g.stat[at * 2 + 1], w, sum);
        o = __builtin_fmaf(g.part[at * s.D + d], w, o);
    }
    const int64_t pair = id / s.rows, row = id % s.rows;
    const int n = (int)(pair / s.Hk), head = (int)(pair % s.Hk) * s.rep + (int)(row % s.rep);
    const int64_t t = row / s.rep;
    ((T*)g.a.y)[(((int64_t)n * s.Lq + t) * s.Hq + head) * s.D + d] = (T)(sum == 0.0f ? 0.0f : o / sum);
    if (g.a.lse && d == 0)
        g.a.lse[((int64_t)n * s.Hq + head) * s.Lq + t] =
            sum == 0.0f ? -INFINITY : __builtin_fmaf(top, s.scale, __builtin_amdgcn_logf(sum) * kLn2);
}

// ---------------------------------------------------------------- backward
// With P = exp(S - lse), dP = dy v^T, delta = sum dy y and dS = P (dP - delta):
// dq = scale dS k, dk = scale dS^T q, dv = P^T dy.  Two launches, over rows and over
// keys, each forming S and dP again, so that every sum has one owner and a fixed
// order; the first also leaves delta for the second.
//
// fp16 operands: P is held 2^12 times as large (a row's share of 2^-24 keeps its bits),
// dS times a power of two for each column of the result, which falls, with what is
// summed, where a larger dS than fp16 holds comes by.

constexpr float kPUp = 4096.0f;

// dS of a lane's column to operands' range: s *= up; up falls first if it must.
template <int NB, int DB>
__device__ __forceinline__ void keep_range(const f32x16 (&ds)[NB], float& up, f32x16 (&acc)[DB]) {
    float mx = 0.0f;
#pragma unroll
    for (int k = 0; k < NB; ++k)
#pragma unroll
        for (int i = 0; i < 16; ++i) mx = fmaxf(mx, fabsf(ds[k][i]));
    mx = max_halves(mx);
    if (__any(mx * up > 0x1p15f)) {
        // 2^14 over the power of two at or below mx
        const int e = (int)((__float_as_uint(mx) >> 23) & 255) - 127;
        const float to = fminf(up, __uint_as_float((uint32_t)(min(max(14 - e, -126), 100) + 127) << 23));
        const float a = to / up;
        up = to;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[d][i] *= a;
    }
}

// dq of 128 rows, and delta.
template <typename T, int D16>
__global__ __launch_bounds__(256) void k_attn_dq(AttnK g) {
    using Tl = Tile<T, D16>;
    constexpr int NT = 256, KT = 64, KB = 2, DB = (D16 + 1) / 2;
    constexpr bool kHalf = std::is_same_v<T, _Float16>;
    __shared__ alignas(16) char sk[KT * Tl::kRow];
    __shared__ alignas(16) char sv[KT * Tl::kRow];
    __shared__ alignas(16) float bias[KT];
    const AttnShape& s = g.s;
    const int64_t item = item_of(g.items);
    if (item < 0) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5;
    const int split = (int)(item % g.splits);
    const int64_t tile = item / g.splits % g.tiles, pair = item / g.splits / g.tiles;
    const int n = (int)(pair / s.Hk), hk = (int)(pair % s.Hk);
    const int64_t row = tile * 128 + wave * 32 + (lane & 31);
    const bool live = row < s.rows;
    const RowAt me = row_at(g, n, hk, row);
    const int64_t stat = ((int64_t)n * s.Hq + me.head) * s.Lq + me.t, dense = (me.tok * s.Hq + me.head) * s.D;
    const T* q = live ? (const T*)g.b.q + me.tok * s.ldq + (int64_t)me.head * s.D : nullptr;
    const T* dy = live ? (const T*)g.b.dy + dense : nullptr;
    const T* y = live ? (const T*)g.b.y + dense : nullptr;
    Frag<T> fq[D16], fo[D16];
    float delta = 0.0f;
#pragma unroll
    for (int c = 0; c < D16; ++c) {
        fq[c] = load_frag(q, c, h, s.D, g.vec);
        fo[c] = load_frag(dy, c, h, s.D, g.vec);
        const Frag<T> fy = load_frag(y, c, h, s.D, g.vec);
#pragma unroll
        for (int j = 0; j < 8; ++j) delta = __builtin_fmaf((float)fo[c].v[j], (float)fy.v[j], delta);
    }
    delta = add_halves(delta);
    if (live && h == 0 && split == 0) g.delta[stat] = delta;
    const float lse = live ? g.b.lse[stat] : -INFINITY;
    const float off = lse == -INFINITY ? -INFINITY : -lse * kLog2e;

    int64_t lo, hi;
    const int len = keys_of(g.b.klen, n, s.Lk);
    part_of(len, KT, split, g.splits, lo, hi);
    const T* kbase = (const T*)g.b.k + (int64_t)n * s.Lk * s.ldk + (int64_t)hk * s.D;
    const T* vbase = (const T*)g.b.v + (int64_t)n * s.Lk * s.ldv + (int64_t)hk * s.D;
    const uint8_t* mask = g.b.mask ? g.b.mask + (int64_t)n * s.Lk : nullptr;
    Moving<T, D16, KT, NT> mk, mv;
    float mb = 0.0f;
    auto load = [&](int64_t k0) {
        auto kept = [&](int r) { return k0 + r < hi && (!mask || mask[k0 + r]); };
        mk.load([&](int r) { return kept(r) ? kbase + (k0 + r) * s.ldk : nullptr; }, s.D, g.vec);
        mv.load([&](int r) { return kept(r) ? vbase + (k0 + r) * s.ldv : nullptr; }, s.D, g.vec);
        if (threadIdx.x < KT) mb = kept(threadIdx.x) ? 0.0f : -INFINITY;
    };

    const float c2 = s.scale * kLog2e;
    float up = kHalf ? 0x1p100f : 1.0f;
    f32x16 acc[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) acc[d] = f32x16{};
    if (lo < hi) load(lo);
    for (int64_t k0 = lo; k0 < hi; k0 += KT) {
        __syncthreads();
        mk.store(sk);
        mv.store(sv);
        if (threadIdx.x < KT) bias[threadIdx.x] = mb;
        __syncthreads();
        const bool whole = !mask && k0 + KT <= hi;
        if (k0 + KT < hi) load(k0 + KT);
        f32x16 ds[KB];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            f32x16 p{}, dp{};
#pragma unroll
            for (int c = 0; c < D16; ++c) {
                p = mma(Tl::read(sk, kb * 32 + (lane & 31), c, h), fq[c], p);
                dp = mma(Tl::read(sv, kb * 32 + (lane & 31), c, h), fo[c], dp);
            }
            if (!whole) {
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    const f32x4v m = *(const f32x4v*)&bias[kb * 32 + 8 * b + 4 * h];
#pragma unroll
                    for (int i = 0; i < 4; ++i) p[4 * b + i] += m[i];
                }
            }
#pragma unroll
            for (int i = 0; i < 16; ++i)
                ds[kb][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[i], c2, off)) * (dp[i] - delta);
        }
        if constexpr (kHalf) {
            keep_range(ds, up, acc);
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int i = 0; i < 16; ++i) ds[kb][i] *= up;
        }
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const Frag<T> f = pack<T>(ds[kb], e);
#pragma unroll
                for (int d = 0; d < DB; ++d) acc[d] = mma(Tl::turned(sk, kb * 32 + 16 * e, d, lane), f, acc[d]);
            }
    }
    if (!live) return;
    const float f = s.scale / up;
    if (g.splits > 1) {
        float* part = g.part + (((int64_t)split * s.N * s.Hk + pair) * s.rows + row) * s.D;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int b = 0; b < 4; ++b)
                store4(part, 32 * d + 8 * b + 4 * h, s.D, (s.D & 3) == 0, acc[d][4 * b] * f, acc[d][4 * b + 1] * f,
                       acc[d][4 * b + 2] * f, acc[d][4 * b + 3] * f);
        return;
    }
    T* dq = (T*)g.b.dq + me.tok * s.ldq + (int64_t)me.head * s.D;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int b = 0; b < 4; ++b)
            store4(dq, 32 * d + 8 * b + 4 * h, s.D, g.vec, acc[d][4 * b] * f, acc[d][4 * b + 1] * f, acc[d][4 * b + 2] * f,
                   acc[d][4 * b + 3] * f);
}

// dk and dv of 128 keys: a wave owns 32 of them and walks the pair's rows.  Keys that
// are left out are columns of their own, so what they hold goes nowhere.
template <typename T, int D16>
__global__ __launch_bounds__(256) void k_attn_dkv(AttnK g) {
    using Tl = Tile<T, D16>;
    constexpr int NT = 256, RT = 32, DB = (D16 + 1) / 2;
    constexpr bool kHalf = std::is_same_v<T, _Float16>;
    __shared__ alignas(16) char sq[RT * Tl::kRow];
    __shared__ alignas(16) char so[RT * Tl::kRow];
    __shared__ alignas(16) float offs[RT], deltas[RT];
    const AttnShape& s = g.s;
    const int64_t item = item_of(g.items);
    if (item < 0) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5;
    const int split = (int)(item % g.splits);
    const int64_t tile = item / g.splits % g.tiles, pair = item / g.splits / g.tiles;
    const int n = (int)(pair / s.Hk), hk = (int)(pair % s.Hk);
    const int len = keys_of(g.b.klen, n, s.Lk);
    const int64_t key = tile * 128 + wave * 32 + (lane & 31);
    const bool kept = key < len && (!g.b.mask || g.b.mask[(int64_t)n * s.Lk + key]);
    const int64_t tok = (int64_t)n * s.Lk + key;
    const T* k = kept ? (const T*)g.b.k + tok * s.ldk + (int64_t)hk * s.D : nullptr;
    const T* v = kept ? (const T*)g.b.v + tok * s.ldv + (int64_t)hk * s.D : nullptr;
    Frag<T> fk[D16], fv[D16];
#pragma unroll
    for (int c = 0; c < D16; ++c) {
        fk[c] = load_frag(k, c, h, s.D, g.vec);
        fv[c] = load_frag(v, c, h, s.D, g.vec);
    }
    int64_t lo, hi;
    part_of(tile * 128 < len ? s.rows : 0, RT, split, g.splits, lo, hi);
    Moving<T, D16, RT, NT> mq, mo;
    float moff = 0.0f, mdel = 0.0f;
    auto load = [&](int64_t r0) {
        mq.load([&](int r) {
            const RowAt x = row_at(g, n, hk, r0 + r);
            return r0 + r < hi ? (const T*)g.b.q + x.tok * s.ldq + (int64_t)x.head * s.D : nullptr;
        }, s.D, g.vec);
        mo.load([&](int r) {
            const RowAt x = row_at(g, n, hk, r0 + r);
            return r0 + r < hi ? (const T*)g.b.dy + (x.tok * s.Hq + x.head) * s.D : nullptr;
        }, s.D, g.vec);
        if (threadIdx.x < RT) {
            const bool in = r0 + threadIdx.x < hi;
            const RowAt x = row_at(g, n, hk, r0 + threadIdx.x);
            const int64_t at = in ? ((int64_t)n * s.Hq + x.head) * s.Lq + x.t : 0;
            const float l = in ? g.b.lse[at] : -INFINITY;
            moff = l == -INFINITY ? -INFINITY : -l * kLog2e;
            mdel = in ? g.delta[at] : 0.0f;
        }
    };

    const float c2 = s.scale * kLog2e;
    float up = kHalf ? 0x1p100f : 1.0f;
    f32x16 ak[DB], av[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) ak[d] = av[d] = f32x16{};
    if (lo < hi) load(lo);
    for (int64_t r0 = lo; r0 < hi; r0 += RT) {
        __syncthreads();
        mq.store(sq);
        mo.store(so);
        if (threadIdx.x < RT) {
            offs[threadIdx.x] = moff;
            deltas[threadIdx.x] = mdel;
        }
        __syncthreads();
        if (r0 + RT < hi) load(r0 + RT);
        f32x16 p{}, ds[1] = {f32x16{}};
#pragma unroll
        for (int c = 0; c < D16; ++c) {
            p = mma(Tl::read(sq, lane & 31, c, h), fk[c], p);
            ds[0] = mma(Tl::read(so, lane & 31, c, h), fv[c], ds[0]);
        }
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const f32x4v o4 = *(const f32x4v*)&offs[8 * b + 4 * h], d4 = *(const f32x4v*)&deltas[8 * b + 4 * h];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(p[4 * b + i], c2, o4[i]));
                ds[0][4 * b + i] = x * (ds[0][4 * b + i] - d4[i]);
                p[4 * b + i] = kHalf ? x * kPUp : x;
            }
        }
        if constexpr (kHalf) {
            keep_range(ds, up, ak);
#pragma unroll
            for (int i = 0; i < 16; ++i) ds[0][i] *= up;
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const Frag<T> fp = pack<T>(p, e), fd = pack<T>(ds[0], e);
#pragma unroll
            for (int d = 0; d < DB; ++d) {
                av[d] = mma(Tl::turned(so, 16 * e, d, lane), fp, av[d]);
                ak[d] = mma(Tl::turned(sq, 16 * e, d, lane), fd, ak[d]);
            }
        }
    }
    if (key >= s.Lk) return;
    const float f = s.scale / up, fvv = kHalf ? 1.0f / kPUp : 1.0f;
    auto put = [&](auto* dk, auto* dv, bool vec) {
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                float x[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x[i] = kept ? ak[d][4 * b + i] * f : 0.0f;
                    x[4 + i] = kept ? av[d][4 * b + i] * fvv : 0.0f;
                }
                store4(dk, 32 * d + 8 * b + 4 * h, s.D, vec, x[0], x[1], x[2], x[3]);
                store4(dv, 32 * d + 8 * b + 4 * h, s.D, vec, x[4], x[5], x[6], x[7]);
            }
    };
    if (g.splits > 1) {
        const int64_t id = (((int64_t)split * s.N * s.Hk + pair) * s.Lk + key) * s.D;
        put(g.part + id, g.part2 + id, (s.D & 3) == 0);
    } else {
        put((T*)g.b.dk + tok * s.ldk + (int64_t)hk * s.D, (T*)g.b.dv + tok * s.ldv + (int64_t)hk * s.D, g.vec);
    }
}

// Sum of `splits` partial gradients [pairs][rows][D], to tokens ld elements apart.
struct AttnSum {
    const float *a, *b;                      // b: a second tensor, or null
    void *x, *y;
    int64_t pairs, rows;
    int Hk, rep, L, D, ldx, ldy, splits;
};
template <typename T>
__global__ __launch_bounds__(256) void k_attn_sum(AttnSum g) {
    const int64_t all = g.pairs * g.rows * g.D, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= all) return;
    const float* p = blockIdx.y ? g.b : g.a;
    float sum = 0.0f;
    for (int k = 0; k < g.splits; ++k) sum += p[k * all + i];
    const int d = (int)(i % g.D);
    const int64_t id = i / g.D, pair = id / g.rows, row = id % g.rows;
    const int64_t tok = pair / g.Hk * g.L + row / g.rep;
    const int head = (int)(pair % g.Hk) * g.rep + (int)(row % g.rep);
    ((T*)(blockIdx.y ? g.y : g.x))[tok * (blockIdx.y ? g.ldy : g.ldx) + (int64_t)head * g.D + d] = (T)sum;
}

// ---------------------------------------------------------------- launches

inline unsigned grid_of(int64_t items) { return (unsigned)((items + 7) / 8 * 8); }

template <typename T, int D16>
hipError_t attn_run(const AttnK& g, const AttnPlan& p, bool backward, hipStream_t st) {
    AttnK a = g;
    const AttnShape& s = g.s;
    const int64_t pairs = (int64_t)s.N * s.Hk;
    a.tiles = p.rows.tiles;
    a.splits = p.rows.splits;
    a.items = pairs * a.tiles * a.splits;
    if (!backward) {
        if (p.few)
            k_attn<T, D16, true><<<grid_of(a.items), FwdCut<T, D16, true>::kThreads, 0, st>>>(a);
        else
            k_attn<T, D16, false><<<grid_of(a.items), FwdCut<T, D16, false>::kThreads, 0, st>>>(a);
        if (a.splits > 1) {
            const int per = 256 / s.D;
            k_attn_join<T><<<(unsigned)((pairs * s.rows + per - 1) / per), 256, 0, st>>>(a);
        }
        return hipGetLastError();
    }
    k_attn_dq<T, D16><<<grid_of(a.items), 256, 0, st>>>(a);
    if (a.splits > 1) {
        const AttnSum m{a.part, nullptr, a.b.dq, nullptr, pairs, s.rows, s.Hk, s.rep, s.Lq, s.D, s.ldq, 0, a.splits};
        k_attn_sum<T><<<(unsigned)((pairs * s.rows * s.D + 255) / 256), 256, 0, st>>>(m);
    }
    a.tiles = p.keys.tiles;
    a.splits = p.keys.splits;
    a.items = pairs * a.tiles * a.splits;
    a.part2 = a.part + (size_t)a.splits * pairs * s.Lk * s.D;
    k_attn_dkv<T, D16><<<grid_of(a.items), 256, 0, st>>>(a);
    if (a.splits > 1) {
        const AttnSum m{a.part, a.part2, a.b.dk, a.b.dv, pairs, s.Lk, s.Hk, 1, s.Lk, s.D, s.ldk, s.ldv, a.splits};
        k_attn_sum<T><<<dim3((unsigned)((pairs * s.Lk * s.D + 255) / 256), 2), 256, 0, st>>>(m);
    }
    return hipGetLastError();
}

template <typename T>
hipError_t attn_run_any(const AttnK& g, const AttnPlan& p, bool backward, hipStream_t st) {
    const int d16 = (g.s.D + 15) / 16;
    if (d16 <= 2) return attn_run<T, 2>(g, p, backward, st);
    if (d16 == 3) return attn_run<T, 3>(g, p, backward, st);
    if (d16 == 4) return attn_run<T, 4>(g, p, backward, st);
    if (d16 <= 6) return attn_run<T, 6>(g, p, backward, st);
    return attn_run<T, 8>(g, p, backward, st);
}

hipError_t attn_f32(const AttnK& g, const AttnPlan& p, bool backward, hipStream_t st);
hipError_t attn_f16(const AttnK& g, const AttnPlan& p, bool backward, hipStream_t st);
hipError_t attn_bf16(const AttnK& g, const AttnPlan& p, bool backward, hipStream_t st);

}  // namespace wino
