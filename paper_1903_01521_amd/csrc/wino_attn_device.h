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

// fp32 operands are three bf16 terms each, h + m + l, eight significand bits a term (their
// split is exact down to 2^-110), and a product is the sum of the six largest of nine,
// 2.67 times the fp32 matrix rate; what is dropped is below 2^-20 of the product.  A value
// that is not finite makes its sums NaN.

template <typename T>
struct Frag {
    typedef T V __attribute__((ext_vector_type(8)));
    V v;
};
typedef __bf16 b16x8 __attribute__((ext_vector_type(8)));
template <>
struct Frag<float> {
    b16x8 h, m, l;
};

__device__ __forceinline__ f32x16 mma(const Frag<_Float16>& a, const Frag<_Float16>& b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a.v, b.v, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma(b16x8 a, b16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma(const Frag<__bf16>& a, const Frag<__bf16>& b, f32x16 c) { return mma(a.v, b.v, c); }
__device__ __forceinline__ f32x16 mma(const Frag<float>& a, const Frag<float>& b, f32x16 c) {
    c = mma(a.l, b.h, c);
    c = mma(a.h, b.l, c);
    c = mma(a.m, b.m, c);
    c = mma(a.m, b.h, c);
    c = mma(a.h, b.m, c);
    return mma(a.h, b.h, c);
}

// The terms of two values, a word of each: h and m cut off towards zero, l what is left.
__device__ __forceinline__ void split_two(float a, float b, uint32_t& h, uint32_t& m, uint32_t& l) {
    constexpr uint32_t kHigh = 0xffff0000u, kTake = 0x07060302u;
    const uint32_t ab = __float_as_uint(a), bb = __float_as_uint(b);
    const float a1 = a - __uint_as_float(ab & kHigh), b1 = b - __uint_as_float(bb & kHigh);
    const uint32_t a1b = __float_as_uint(a1), b1b = __float_as_uint(b1);
    const float a2 = a1 - __uint_as_float(a1b & kHigh), b2 = b1 - __uint_as_float(b1b & kHigh);
    h = __builtin_amdgcn_perm(bb, ab, kTake);
    m = __builtin_amdgcn_perm(b1b, a1b, kTake);
    l = __builtin_amdgcn_perm(__float_as_uint(b2), __float_as_uint(a2), kTake);
}

// Eight values as an operand, rounded once to T.
template <typename T>
__device__ __forceinline__ Frag<T> frag_of(const float (&x)[8]) {
    Frag<T> f;
    if constexpr (sizeof(T) == 4) {
        uint32_t h[4], m[4], l[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) split_two(x[2 * j], x[2 * j + 1], h[j], m[j], l[j]);
        __builtin_memcpy(&f.h, h, 16);
        __builtin_memcpy(&f.m, m, 16);
        __builtin_memcpy(&f.l, l, 16);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) f.v[j] = (T)x[j];
    }
    return f;
}

// Values 8 at .. 8 at + 7 of a result as an operand.
template <typename T>
__device__ __forceinline__ Frag<T> pack(const f32x16& s, int at) {
    float x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = s[8 * at + j];
    return frag_of<T>(x);
}

// c + the sum of an operand's eight values as they are rounded (16-bit types).
__device__ __forceinline__ float sum_of(const Frag<_Float16>& f, float c) {
    typedef _Float16 V2 __attribute__((ext_vector_type(2)));
    const V2 one = {(_Float16)1.0f, (_Float16)1.0f};
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_fdot2(V2{f.v[2 * j], f.v[2 * j + 1]}, one, c, false);
    return c;
}
__device__ __forceinline__ float sum_of(const Frag<__bf16>& f, float c) {
    typedef __bf16 V2 __attribute__((ext_vector_type(2)));
    const V2 one = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_fdot2_f32_bf16(V2{f.v[2 * j], f.v[2 * j + 1]}, one, c, false);
    return c;
}

// ---------------------------------------------------------------- tiles in LDS
// R rows of W = 16 D16 16-bit values (up to a power of two), in 16-byte chunks whose place
// is xored with bits of the row, so that 16 rows' chunk of the same number lie in
// different banks (read(), a row for each lane) and four rows' 64 bytes too (turned(),
// the transposing read of four rows by 16 columns).  fp32 tiles are three such planes.

template <typename T, int D16, int R>
struct Tile {
    static constexpr int kP2 = D16 <= 2 ? 2 : D16 <= 4 ? 4 : 8;
    static constexpr int kRow = kP2 * 32;                           // bytes
    static constexpr int kPlane = R * kRow;
    static constexpr int kBytes = kPlane * (sizeof(T) == 4 ? 3 : 1);
    static constexpr int kChunks = D16 * (int)sizeof(T);            // 16-byte chunks of a row in memory
    static constexpr int kEach = 16 / (int)sizeof(T);               // values of a chunk

    __device__ static __forceinline__ int twist(int row) {
        if constexpr (kRow == 64) return (row >> 2) & 3;
        else if constexpr (kRow == 128) return ((row & 2) << 1) | ((row >> 2) & 3);
        else return ((row & 3) << 2) | ((row >> 2) & 3);
    }
    __device__ static __forceinline__ int at(int row, int chunk) { return row * kRow + ((chunk ^ twist(row)) << 4); }

    // a chunk of memory, to its place
    __device__ static __forceinline__ void store(char* t, int row, int ch, uint4 w) {
        if constexpr (sizeof(T) == 2) {
            *(uint4*)(t + at(row, ch)) = w;
        } else {
            uint2 h, m, l;
            split_two(__uint_as_float(w.x), __uint_as_float(w.y), h.x, m.x, l.x);
            split_two(__uint_as_float(w.z), __uint_as_float(w.w), h.y, m.y, l.y);
            char* p = t + at(row, ch >> 1) + (ch & 1) * 8;
            *(uint2*)p = h;
            *(uint2*)(p + kPlane) = m;
            *(uint2*)(p + 2 * kPlane) = l;
        }
    }

    // values 16 c + 8 h .. + 7 of row `row`
    __device__ static __forceinline__ Frag<T> read(const char* t, int row, int c, int h) {
        Frag<T> f;
        const char* p = t + at(row, 2 * c + h);
        if constexpr (sizeof(T) == 2) {
            f.v = *(const typename Frag<T>::V*)p;
        } else {
            f.h = *(const b16x8*)p;
            f.m = *(const b16x8*)(p + kPlane);
            f.l = *(const b16x8*)(p + 2 * kPlane);
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
        const int row = r + HALF * (lane >> 5) + ((lane >> 2) & 3);
        const int chunk = 4 * db + ((lane >> 3) & 2) + ((lane >> 1) & 1), low = (lane & 1) * 8;
        const char *p = t + at(row, chunk) + low, *q = t + at(row + NEXT, chunk) + low;
        auto two = [&](int plane) {
            const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + plane * kPlane));
            const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(q + plane * kPlane));
            typedef short s16x8 __attribute__((ext_vector_type(8)));
            return (s16x8)__builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
        };
        if constexpr (sizeof(T) == 2) {
            f.v = __builtin_bit_cast(typename Frag<T>::V, two(0));
        } else {
            f.h = __builtin_bit_cast(b16x8, two(0));
            f.m = __builtin_bit_cast(b16x8, two(1));
            f.l = __builtin_bit_cast(b16x8, two(2));
        }
        return f;
    }
};

// ---------------------------------------------------------------- global memory

// Values d .. d + each - 1 of a vector of D values at p; those past D are zero.  vec:
// p and D allow whole 16-byte words; else a load of 16 bytes on any address (a value at a time
// cost 432 tokens of 700 channels by 2000 units, backward, 170 us), and the end one by one.
template <typename T>
__device__ __forceinline__ uint4 load_chunk(const T* p, int d, int D, bool vec) {
    constexpr int kEach = 16 / (int)sizeof(T);
    if (vec) return d < D ? *(const uint4*)(p + d) : make_uint4(0, 0, 0, 0);
    uint4 r = make_uint4(0, 0, 0, 0);
    if (d + kEach <= D) {
        __builtin_memcpy(&r, p + d, 16);
    } else if (d < D) {
        T v[kEach];
#pragma unroll
        for (int j = 0; j < kEach; ++j) v[j] = d + j < D ? p[d + j] : (T)0.0f;
        __builtin_memcpy(&r, v, 16);
    }
    return r;
}

// Values 16 c + 8 h .. + 7 of the vector at p; zeros where p is null.
template <typename T>
struct Eight {
    T v[8];
    __device__ __forceinline__ Eight(const T* p, int c, int h, int D, bool vec) {
        constexpr int kEach = 16 / (int)sizeof(T);
        uint4 r[sizeof(T) / 2];
#pragma unroll
        for (int j = 0; j < (int)sizeof(T) / 2; ++j)
            r[j] = p ? load_chunk(p, 16 * c + 8 * h + j * kEach, D, vec) : make_uint4(0, 0, 0, 0);
        __builtin_memcpy(v, r, sizeof(r));
    }
    __device__ __forceinline__ Frag<T> frag() const {
        Frag<T> f;
        if constexpr (sizeof(T) == 4) f = frag_of<float>(v);
        else __builtin_memcpy(&f.v, v, 16);
        return f;
    }
};
template <typename T>
__device__ __forceinline__ Frag<T> load_frag(const T* p, int c, int h, int D, bool vec) {
    return Eight<T>(p, c, h, D, vec).frag();
}

// Four neighbouring values of a result to p + d, those below D.
template <typename T>
__device__ __forceinline__ void store4(T* p, int d, int D, bool vec, float a, float b, float c, float e) {
    const T v[4] = {(T)a, (T)b, (T)c, (T)e};
    if (vec) {
        if (d < D) __builtin_memcpy(__builtin_assume_aligned(p + d, 4 * sizeof(T)), v, sizeof(v));
        return;
    }
    if (d + 4 <= D) {
        __builtin_memcpy(p + d, v, sizeof(v));
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (d + j < D) p[d + j] = v[j];
}

// A tile of `R` rows on its way: loaded to registers while the one before is worked on.
template <typename T, int D16, int R, int NT>
struct Moving {
    using Tl = Tile<T, D16, R>;
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
            if (kAll % NT == 0 || idx < kAll) Tl::store(t, row, ch, w[i]);
        }
    }
};

// `bytes` at p, zeros behind them, as loads take it
typedef uint32_t Buffer __attribute__((ext_vector_type(4)));
__device__ __forceinline__ Buffer buffer_of(const void* p, uint32_t bytes) {
    const uint64_t at = (uint64_t)p;
    return Buffer{(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)at),
                  (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(at >> 32)) & 0xffffu,
                  (uint32_t)__builtin_amdgcn_readfirstlane(bytes), 0x00020000u};
}

// A tile of R rows from memory straight to LDS, 16 bytes a lane, whose place is fixed there:
// a lane takes the chunk that belongs to it.  Offsets past 2^31 read zeros, as do rows past
// the buffer's end; they are the same for every tile.  (In place of Moving: 64 keys of 64
// channels a step cost 80 of 285 vector instructions and 16 registers less.)
template <typename Tl, int R, int NT>
struct Direct {
    static constexpr int kRowChunks = Tl::kRow / 16, kN = R * kRowChunks / NT;
    static_assert(R * kRowChunks % NT == 0);
    uint32_t off[kN];
    // offset(row, chunk) in bytes; the chunk is one past the row's values: none
    template <typename F>
    __device__ __forceinline__ void init(int used, F offset) {
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            const int at = threadIdx.x + i * NT, row = at / kRowChunks, chunk = (at % kRowChunks) ^ Tl::twist(row);
            off[i] = chunk < used ? offset(row, chunk) : 0x80000000u;
        }
    }
    // to the tile at t; bytes: of the buffer at p
    __device__ __forceinline__ void issue(char* t, const void* p, uint32_t bytes) const {
        issue_at(place(t), buffer_of(p, bytes), 0);
    }
    // this wave's part of the tile at t
    __device__ static __forceinline__ uint32_t place(char* t) {
        const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)t;
        return __builtin_amdgcn_readfirstlane(lds + (threadIdx.x >> 6) * 1024);
    }
    // at: bytes from the buffer's start.  In assembly: the compiler would wait for every load to
    // LDS before it reads any of LDS, the other copies' tiles too.  What waits for them is ready().
    __device__ __forceinline__ void issue_at(uint32_t lds, const Buffer& r, uint32_t at) const {
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"          // m0 on the clobber list
#pragma unroll
        for (int i = 0; i < kN; ++i)
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(lds + i * NT * 16),
                         "v"(off[i]), "s"(r), "s"(at)
                         : "memory", "m0");
#pragma clang diagnostic pop
    }
    // the same, of each row `used` chunks
    __device__ __forceinline__ Direct part(int used) const {
        Direct d;
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            const int at = threadIdx.x + i * NT, row = at / kRowChunks;
            d.off[i] = ((at % kRowChunks) ^ Tl::twist(row)) < used ? off[i] : 0x80000000u;
        }
        return d;
    }
};
// 64 floats (or bytes, each a word of LDS) at p, `left` of them and zeros behind, to LDS by one wave.
template <typename V>
__device__ __forceinline__ void load_words(void* t, const V* p, int64_t left) {
    const Buffer r = buffer_of(p, (uint32_t)(left < 64 ? left : 64) * (uint32_t)sizeof(V));
    const uint32_t lds = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)(char*)t);
    const uint32_t off = (threadIdx.x & 63) * (uint32_t)sizeof(V);
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
    if constexpr (sizeof(V) == 4)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(lds), "v"(off), "s"(r)
                     : "memory", "m0");
    else
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_ubyte %1, %2, 0 offen lds" ::"s"(lds), "v"(off), "s"(r)
                     : "memory", "m0");
#pragma clang diagnostic pop
}
// This wave's loads to LDS have arrived, but the last n, and its own LDS accesses are
// done; then so are those of the workgroup's other waves.
template <int n>
__device__ __forceinline__ void ready() {
    static_assert(n < 64);
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(n) : "memory");
}

// Before a loop with such loads: whatever was loaded to registers is there, or the compiler's
// wait for it, inside the loop, would wait for the tiles in every step.
__device__ __forceinline__ void settled() { __builtin_amdgcn_s_waitcnt(0x0F70); }

// ---------------------------------------------------------------- work

struct AttnK {
    AttnShape s;
    AttnArgs a;
    AttnBwd b;
    int64_t tiles;                           // of a pair in this launch, each in `splits` parts
    int splits;
    bool by_xcd;
    FastDiv per_pair, per_tile;              // by tiles * splits, by splits
    // backward, of each pair's rows in turn: delta, the exponent's offset -lse log2 e (fp16: + 12), and (fp32)
    // 1 over the sum of P
    float *delta, *offset, *share;
    float *part, *part2, *stat;
    bool vec;
    FastDiv rep, heads;                      // by s.rep (rows are below 2^31), by s.Hk
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

// A workgroup's (image, key head) pair, tile and part.  Workgroup ids go round the eight
// XCDs; with by_xcd all workgroups of a pair are on one, whose L2 then holds the pair's
// keys (or rows), and the pairs go round, so that images of different lengths spread (16
// images of 0 to 2048 keys, 8 heads: 248 us with runs of pairs on an XCD).  Without, for few pairs, an
// XCD would be left with less: workgroups as they come.
struct Work {
    int n, hk, split;
    int64_t pair, tile;
    bool none;
};
__device__ __forceinline__ Work work_of(const AttnK& g) {
    const uint32_t id = blockIdx.x, per = (uint32_t)(g.tiles * g.splits), j = g.by_xcd ? id >> 3 : id;
    const uint32_t p = fdiv(j, g.per_pair), at = j - p * per, tile = fdiv(at, g.per_tile);
    Work w;
    w.pair = g.by_xcd ? p * 8 + (id & 7) : p;
    w.none = w.pair >= (int64_t)g.s.N * g.s.Hk;
    w.n = (int)fdiv((uint32_t)w.pair, g.heads);
    w.hk = (int)w.pair - w.n * g.s.Hk;
    w.tile = tile;
    w.split = (int)(at - tile * (uint32_t)g.splits);
    return w;
}

// keys of image n
__device__ __forceinline__ int keys_of(const int* klen, int n, int Lk) {
    return klen ? min(max(klen[n], 0), Lk) : Lk;
}

// part `split` of n < 2^31 in whole steps of `step`
__device__ __forceinline__ void part_of(int64_t n, int step, int split, int splits, int64_t& lo, int64_t& hi) {
    const int64_t each = (int64_t)(((uint32_t)((n + step - 1) / step) + (uint32_t)splits - 1) / (uint32_t)splits) * step;
    lo = min(each * split, n);
    hi = min(lo + each, n);
}

// Waves a SIMD that a kernel's registers are held to.  With two (256 registers a wave) no
// result lies in accumulation registers, from where every step would have to copy it; heads
// wider than 16 `most` would spill.
template <typename T, int D16>
constexpr int waves_of(int most) {
    return sizeof(T) == 2 && D16 <= most ? 2 : 1;
}

// Copies of the tiles in LDS: with two, a step has one barrier, and the next tile is
// stored while slower waves still read this one.  fp32 tiles are too large.
template <typename T>
constexpr int kCopies = sizeof(T) == 2 ? 2 : 1;

// How vectors lie in memory: anywhere; in whole 16-byte words; so, and rows of a tile within
// 2^31 bytes, in 16 bits, straight to LDS.
enum { kAnywhere, kWords, kStraight };

// The keys' and values' tiles of a walk over keys up to hi.
template <typename T, int D16, int KT, int NT, int kHow>
struct KeyTiles {                            // by way of registers: any address and type
    Moving<T, D16, KT, NT> mk, mv;
    float mb;
    const AttnShape* s;
    const T *kbase, *vbase;
    const uint8_t* mask;
    int64_t hi;
    __device__ __forceinline__ void init(const AttnShape& s_, const T* k, const T* v, const uint8_t* mask_,
                                         int64_t hi_, float*) {
        s = &s_; kbase = k; vbase = v; mask = mask_; hi = hi_;
        mb = 0.0f;
    }
    __device__ __forceinline__ void load(int64_t k0) {
        auto kept = [&](int r) { return k0 + r < hi && (!mask || mask[k0 + r]); };
        mk.load([&](int r) { return kept(r) ? kbase + (k0 + r) * s->ldk : nullptr; }, s->D, kHow == kWords);
        mv.load([&](int r) { return kept(r) ? vbase + (k0 + r) * s->ldv : nullptr; }, s->D, kHow == kWords);
        if (threadIdx.x < KT) mb = kept(threadIdx.x) ? 0.0f : -INFINITY;
    }
    __device__ __forceinline__ void first(char*, char*, int64_t k0) { load(k0); }
    // the tile at k0 to LDS, the next one on its way
    __device__ __forceinline__ void step(char* sk, char* sv, float* bias, char*, char*, int64_t k0) {
        if (kCopies<T> == 1) __syncthreads();
        mk.store(sk);
        mv.store(sv);
        if (threadIdx.x < KT) bias[threadIdx.x] = mb;
        __syncthreads();
        if (k0 + KT < hi) load(k0 + KT);
    }
    // x[e] .. x[e + 3] are the scores of the tile's keys at + 4 h .. + 3: -infinity for those that are left
    // out (a sum with -infinity would leave NaN where the row holds what is not finite)
    __device__ __forceinline__ void leave_out(const float* bias, int at, int h, f32x16& x, int e) const {
        const f32x4v m = *(const f32x4v*)&bias[at + 4 * h];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[e + i] = m[i] == 0.0f ? x[e + i] : -INFINITY;
    }
};
template <typename T, int D16, int KT, int NT>
struct KeyTiles<T, D16, KT, NT, kStraight> {      // straight to LDS: 16-bit, 16-byte words
    using Tl = Tile<T, D16, KT>;
    Direct<Tl, KT, NT> dk, dv;
    const T *kbase, *vbase;
    const uint8_t* mask;
    int64_t hi;
    int ldk, ldv, D;
    uint64_t bits, coming;                   // keys kept of the tile at work and of the one on its way
    float* marks;                            // a word of LDS for each key's byte, of two tiles in turn
    __device__ __forceinline__ void init(const AttnShape& s, const T* k, const T* v, const uint8_t* mask_, int64_t hi_,
                                         float* marks_) {
        kbase = k; vbase = v; mask = mask_; hi = hi_; ldk = s.ldk; ldv = s.ldv; D = s.D;
        bits = coming = 0;
        marks = marks_;
        dk.init(D / 8, [&](int row, int chunk) { return (uint32_t)row * (uint32_t)s.ldk * 2 + chunk * 16; });
        dv.init(D / 8, [&](int row, int chunk) { return (uint32_t)row * (uint32_t)s.ldv * 2 + chunk * 16; });
    }
    // the mask of the tile at k0 on its way, to LDS too: a wait for a register of the loop's next
    // step would be one for the tiles
    __device__ __forceinline__ void look(int64_t k0) const {
        if (k0 < hi && __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) == 0) load_words(marks + (k0 / KT & 1) * 64, mask + k0, hi - k0);
    }
    // keys that are left out are not read: their places get zeros
    __device__ __forceinline__ void some(const Direct<Tl, KT, NT>& d, char* t, const void* p, uint32_t bytes) const {
        Direct<Tl, KT, NT> x;
#pragma unroll
        for (int i = 0; i < x.kN; ++i)
            x.off[i] = coming >> ((threadIdx.x + i * NT) / x.kRowChunks) & 1 ? d.off[i] : 0x80000000u;
        x.issue(t, p, bytes);
    }
    __device__ __forceinline__ void issue(char* sk, char* sv, int64_t k0) {
        const int64_t left = hi - k0;
        const uint32_t last = (uint32_t)(left < KT ? left : KT) - 1;
        const uint32_t bk = (last * (uint32_t)ldk + (uint32_t)D) * 2, bv = (last * (uint32_t)ldv + (uint32_t)D) * 2;
        if (mask) {
            const uint32_t mark = __float_as_uint(marks[(k0 / KT & 1) * 64 + (threadIdx.x & 63)]);
            coming = __ballot(mark != 0);
            some(dk, sk, kbase + k0 * ldk, bk);
            some(dv, sv, vbase + k0 * ldv, bv);
            look(k0 + KT);
        } else {
            coming = left < 64 ? ((uint64_t)1 << left) - 1 : ~(uint64_t)0;
            dk.issue(sk, kbase + k0 * ldk, bk);
            dv.issue(sv, vbase + k0 * ldv, bv);
        }
    }
    __device__ __forceinline__ void first(char* sk, char* sv, int64_t k0) {
        if (mask) {
            look(k0);
            ready<0>();
        }
        issue(sk, sv, k0);
    }
    __device__ __forceinline__ void step(char*, char*, float*, char* nk, char* nv, int64_t k0) {
        ready<0>();
        bits = coming;
        if (k0 + KT < hi) issue(nk, nv, k0 + KT);
    }
    __device__ __forceinline__ void leave_out(const float*, int at, int h, f32x16& x, int e) const {
        const uint32_t b = (uint32_t)((h ? bits >> 4 : bits) >> at);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[e + i] = b >> i & 1 ? x[e + i] : -INFINITY;
    }
};

// ---------------------------------------------------------------- forward
// One pass over the keys with a running maximum and sum, bound by vector instructions: of a
// score register's 33 cycles the exponential takes 16, its argument, the sum, the maximum
// and the rounding 13 (16 images of 3136 tokens to 0..2048 keys, 8 heads of 64, bf16: 142 to 152 us,
// 0.69 to 0.74 PFLOP/s).  The maximum moves, and what is summed is scaled, only where it grows by
// more than 2^8: exponentials stay below 2^8, and most tiles skip the scaling.  fp16 exponentials are
// held 2^7 times as large, below 2^15, and lose what is below 2^-32 of a row's largest (2^-25 without; of
// 65536 keys of 2^-17 each, half a row's weight, every one would be off by as much as 2^-8).  kFew: one
// wave has 32 rows and takes 32 keys a step (single tokens, memory bound: four such workgroups a CU, each
// with its own start and end.  One of four waves, 128 keys a step, a CU took 77 us for 32 tokens to
// 0..4096 keys, 8 heads of 128, bf16, in place of 64).

template <typename T>
constexpr float kExpUp = std::is_same_v<T, _Float16> ? 7.0f : 0.0f;

template <typename T, int D16, bool kFew>
struct FwdCut {
    static constexpr int kWaves = kFew ? 1 : 4;
    static constexpr int kKeys = kFew ? 32 : 64;
    static constexpr int kRows = 32 * kWaves;
    static constexpr int kThreads = 64 * kWaves;
};

template <typename T, int D16, bool kFew, int kHow>
__global__ __launch_bounds__((FwdCut<T, D16, kFew>::kThreads), (waves_of<T, D16>(kFew && kHow != kStraight ? 6 : 8)))
void k_attn(AttnK g) {
    using Cut = FwdCut<T, D16, kFew>;
    constexpr bool kDirect = kHow == kStraight, kVec = kHow != kAnywhere;
    constexpr int NT = Cut::kThreads, KT = Cut::kKeys, KB = kFew ? 1 : KT / 32, DB = (D16 + 1) / 2;
    using Tl = Tile<T, D16, KT>;
    __shared__ alignas(16) char tk[kCopies<T>][Tl::kBytes];
    __shared__ alignas(16) char tv[kCopies<T>][Tl::kBytes];
    __shared__ alignas(16) float biases[kCopies<T>][kDirect ? 64 : KT];
    const AttnShape& s = g.s;
    const Work wk = work_of(g);
    if (wk.none) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5;
    const int split = wk.split, n = wk.n, hk = wk.hk;
    const int64_t tile = wk.tile, pair = wk.pair;
    const int64_t row = tile * Cut::kRows + wave * 32 + (lane & 31);
    const bool live = row < s.rows;
    const RowAt me = row_at(g, n, hk, row);
    const T* q = live ? (const T*)g.a.q + me.tok * s.ldq + (int64_t)me.head * s.D : nullptr;
    Frag<T> fq[D16];
#pragma unroll
    for (int c = 0; c < D16; ++c) fq[c] = load_frag(q, c, h, s.D, kVec);

    int64_t lo, hi;
    const int len = keys_of(g.a.klen, n, s.Lk);
    part_of(len, KT, split, g.splits, lo, hi);
    const T* kbase = (const T*)g.a.k + (int64_t)n * s.Lk * s.ldk + (int64_t)hk * s.D;
    const T* vbase = (const T*)g.a.v + (int64_t)n * s.Lk * s.ldv + (int64_t)hk * s.D;
    const uint8_t* mask = g.a.mask ? g.a.mask + (int64_t)n * s.Lk : nullptr;

    KeyTiles<T, D16, KT, NT, kHow> in;
    in.init(s, kbase, vbase, mask, hi, biases[0]);

    const float c2 = s.scale * kLog2e, slack = fminf(8.0f / c2, 0x1p127f);
    float top = -INFINITY, sum = 0.0f;
    f32x16 o[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) o[d] = f32x16{};
    if (lo < hi) in.first(tk[0], tv[0], lo);
    if (kDirect) settled();
    int copy = 0;
    for (int64_t k0 = lo; k0 < hi; k0 += KT) {
        const char *sk = tk[copy], *sv = tv[copy];
        const float* bias = biases[copy];
        const int next = kCopies<T> == 1 ? 0 : copy ^ 1;
        in.step(tk[copy], tv[copy], biases[copy], tk[next], tv[next], k0);
        copy = next;
        const bool whole = !mask && k0 + KT <= hi;
        f32x16 p[KB];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            p[kb] = f32x16{};
#pragma unroll
            for (int c = 0; c < D16; ++c) p[kb] = mma(Tl::read(sk, kb * 32 + (lane & 31), c, h), fq[c], p[kb]);
        }
        if (!whole) {
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int b = 0; b < 4; ++b) in.leave_out(bias, kb * 32 + 8 * b, h, p[kb], 4 * b);
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
        const float off = top == -INFINITY ? 0.0f : kExpUp<T> - top * c2;
        // a step's sum of its own: one addition to the running one, whose roundings all go one way where
        // keys weigh alike (65536 of them, one by one: off by 3e-4)
        float part = 0.0f;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                p[kb][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[kb][i], c2, off));
                part += p[kb][i];
            }
        sum += part;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const Frag<T> f = pack<T>(p[kb], e);
#pragma unroll
                for (int d = 0; d < DB; ++d) o[d] = mma(Tl::turned(sv, kb * 32 + 16 * e, d, lane), f, o[d]);
            }
    }
    sum = add_halves(sum);
    if (!live) return;
    if (g.splits > 1) {
        const int64_t id = ((int64_t)split * s.N * s.Hk + pair) * s.rows + row;
        float* part = g.part + id * s.D;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int b = 0; b < 4; ++b)
                store4(part, 32 * d + 8 * b + 4 * h, s.D, kVec || (s.D & 3) == 0, o[d][4 * b], o[d][4 * b + 1], o[d][4 * b + 2],
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
            store4(y, 32 * d + 8 * b + 4 * h, s.D, kVec, o[d][4 * b] * inv, o[d][4 * b + 1] * inv, o[d][4 * b + 2] * inv,
                   o[d][4 * b + 3] * inv);
    if (g.a.lse && h == 0)
        g.a.lse[((int64_t)n * s.Hq + me.head) * s.Lq + me.t] =
            sum == 0.0f ? -INFINITY : __builtin_fmaf(top, s.scale, (__builtin_amdgcn_logf(sum) - kExpUp<T>) * kLn2);
}

// The parts of a row: y = sum w o / sum w l with w = 2^(top - the largest top).  A lane has
// the weight of one part, a wave every kWaves-th part; kWaves 4 for a row of many parts (64 of
// them one after the other took 40 us).
template <typename T, int kWaves>
__global__ __launch_bounds__(256) void k_attn_join(AttnK g) {
    const AttnShape& s = g.s;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t all = (int64_t)s.N * s.Hk * s.rows, id = (int64_t)blockIdx.x * (4 / kWaves) + wave / kWaves;
    if (id >= all) return;                   // of all the row's waves
    const float c2 = s.scale * kLog2e;
    float top = lane < g.splits ? g.stat[(lane * all + id) * 2] : -INFINITY;
    float sum = lane < g.splits ? g.stat[(lane * all + id) * 2 + 1] : 0.0f;
    const float mine = top;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
    const float w = __builtin_amdgcn_exp2f((mine - (top == -INFINITY ? 0.0f : top)) * c2);
    sum *= w;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d, 64);
    float o[2] = {0.0f, 0.0f};
    const int last = g.splits - 1;
    for (int i0 = wave % kWaves; i0 <= last; i0 += 8 * kWaves) {
        float v[8][2];                       // eight parts' values on their way together
#pragma unroll
        for (int u = 0; u < 8; ++u)
#pragma unroll
            for (int e = 0; e < 2; ++e)
                v[u][e] = lane + 64 * e < s.D ? g.part[(min(i0 + u * kWaves, last) * all + id) * s.D + lane + 64 * e] : 0.0f;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int i = i0 + u * kWaves;
            if (i > last) break;
            const float wi = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), i));
            o[0] = __builtin_fmaf(v[u][0], wi, o[0]);
            o[1] = __builtin_fmaf(v[u][1], wi, o[1]);
        }
    }
    if constexpr (kWaves == 4) {
        __shared__ float x[3][2][64];
        if (wave) {
            x[wave - 1][0][lane] = o[0];
            x[wave - 1][1][lane] = o[1];
        }
        __syncthreads();
        if (wave) return;
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            o[0] += x[i][0][lane];
            o[1] += x[i][1][lane];
        }
    }
    // with parts there are fewer than 2^31 rows
    const uint32_t pair = (uint32_t)id / (uint32_t)s.rows, n = fdiv(pair, g.heads), row = (uint32_t)id - pair * (uint32_t)s.rows;
    const int64_t t = fdiv(row, g.rep);
    const int head = (int)(pair - n * s.Hk) * s.rep + (int)(row - (uint32_t)t * s.rep);
    T* y = (T*)g.a.y + (((int64_t)n * s.Lq + t) * s.Hq + head) * s.D;
#pragma unroll
    for (int e = 0; e < 2; ++e)
        if (lane + 64 * e < s.D) y[lane + 64 * e] = (T)(sum == 0.0f ? 0.0f : o[e] / sum);
    if (g.a.lse && lane == 0)
        g.a.lse[((int64_t)n * s.Hq + head) * s.Lq + t] =
            sum == 0.0f ? -INFINITY : __builtin_fmaf(top, s.scale, (__builtin_amdgcn_logf(sum) - kExpUp<T>) * kLn2);
}

// ---------------------------------------------------------------- backward
// With P = exp(S - lse), dP = dy v^T, delta = sum dy y and dS = P (dP - delta):
// dq = scale dS k, dk = scale dS^T q, dv = P^T dy.  Two launches, over rows and over
// keys, each forming S and dP again, so that every sum has one owner and a fixed
// order; the first also leaves delta for the second.
//
// y of 16-bit tensors is rounded, which moves delta by up to 2^-9 |dy| |y|: where one key
// has most of a row, dS is the small difference of dP and delta and loses most of its bits
// (gradients of a head of 64, 1024 keys, scores of deviation 2: 3.0e-3 off instead of 2.3e-3;
// sharper rows far more).  With dS' formed from that delta, e = sum dS' is what it lacks:
// delta + e is exact, and dq = scale (sum dS' k - e sum P k), one more product.  There e is
// summed from dS' as rounded, so that what keys have in common, which dS (its sum is zero)
// does not see, takes no part in the rounding either.
//
// fp32: lse's own rounding, and that of its product with log2 e, move all of a row's P by some
// 2^-21; the first launch sums P and both divide by it.
//
// fp16 operands: P is held 2^12 times as large (a row's share of 2^-24 keeps its bits; so is
// dS, and the offset that the first launch leaves says it), and dS times a power of two for
// each column of the result, which falls, with what is summed, where a larger dS than fp16
// holds comes by.

constexpr float kPUp = 4096.0f, kPUpLog = 12.0f;

// Lets up fall where a lane's column of dS times up would pass fp16's range, and what is
// summed with it.
template <int NB, int DB>
__device__ __forceinline__ void keep_range(const f32x16 (&ds)[NB], float& up, f32x16 (&acc)[DB], float& round) {
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
        round *= a;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[d][i] *= a;
    }
}

// 1 over a row's sum of P; 0 for a row without keys.
__device__ __forceinline__ float share_of(float sum) { return sum == 0.0f ? 0.0f : 1.0f / sum; }

// dq of 128 rows, and delta.
template <typename T, int D16, int kHow>
__global__ __launch_bounds__(256, (waves_of<T, D16>(4))) void k_attn_dq(AttnK g) {
    constexpr bool kDirect = kHow == kStraight, kVec = kHow != kAnywhere;
    constexpr int NT = 256, KT = 64, KB = 2, DB = (D16 + 1) / 2;
    constexpr bool kHalf = std::is_same_v<T, _Float16>, kFix = sizeof(T) == 2;
    using Tl = Tile<T, D16, KT>;
    __shared__ alignas(16) char tk[kCopies<T>][Tl::kBytes];
    __shared__ alignas(16) char tv[kCopies<T>][Tl::kBytes];
    __shared__ alignas(16) float biases[kCopies<T>][kDirect ? 64 : KT];
    const AttnShape& s = g.s;
    const Work wk = work_of(g);
    if (wk.none) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5;
    const int split = wk.split, n = wk.n, hk = wk.hk;
    const int64_t tile = wk.tile, pair = wk.pair;
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
        fq[c] = load_frag(q, c, h, s.D, kVec);
        const Eight<T> ed(dy, c, h, s.D, kVec), ey(y, c, h, s.D, kVec);
        fo[c] = ed.frag();
#pragma unroll
        for (int j = 0; j < 8; ++j) delta = __builtin_fmaf((float)ed.v[j], (float)ey.v[j], delta);
    }
    delta = add_halves(delta);
    const float lse = live ? g.b.lse[stat] : -INFINITY;
    // of fp16's P, 2^12 times as large
    const float off = lse == -INFINITY ? -INFINITY : (kHalf ? kPUpLog : 0.0f) - lse * kLog2e;

    int64_t lo, hi;
    const int len = keys_of(g.b.klen, n, s.Lk);
    part_of(len, KT, split, g.splits, lo, hi);
    const T* kbase = (const T*)g.b.k + (int64_t)n * s.Lk * s.ldk + (int64_t)hk * s.D;
    const T* vbase = (const T*)g.b.v + (int64_t)n * s.Lk * s.ldv + (int64_t)hk * s.D;
    const uint8_t* mask = g.b.mask ? g.b.mask + (int64_t)n * s.Lk : nullptr;
    KeyTiles<T, D16, KT, NT, kHow> in;
    in.init(s, kbase, vbase, mask, hi, biases[0]);

    const float c2 = s.scale * kLog2e;
    float up = kHalf ? 0x1p100f : 1.0f, lack = 0.0f, round = 0.0f;
    f32x16 acc[DB], mean[DB];                // mean: sum P k
#pragma unroll
    for (int d = 0; d < DB; ++d) acc[d] = mean[d] = f32x16{};
    if (lo < hi) in.first(tk[0], tv[0], lo);
    if (kDirect) settled();
    int copy = 0;
    for (int64_t k0 = lo; k0 < hi; k0 += KT) {
        const char *sk = tk[copy], *sv = tv[copy];
        const float* bias = biases[copy];
        const int next = kCopies<T> == 1 ? 0 : copy ^ 1;
        in.step(tk[copy], tv[copy], biases[copy], tk[next], tv[next], k0);
        copy = next;
        const bool whole = !mask && k0 + KT <= hi;
        f32x16 ds[KB], ps[KB];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            f32x16 p{}, dp{};
            float part = 0.0f;
#pragma unroll
            for (int c = 0; c < D16; ++c) {
                p = mma(Tl::read(sk, kb * 32 + (lane & 31), c, h), fq[c], p);
                dp = mma(Tl::read(sv, kb * 32 + (lane & 31), c, h), fo[c], dp);
            }
            if (!whole) {
#pragma unroll
                for (int b = 0; b < 4; ++b) in.leave_out(bias, kb * 32 + 8 * b, h, p, 4 * b);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(p[i], c2, off));
                ds[kb][i] = x * (dp[i] - delta);
                if constexpr (kFix) {
                    part += ds[kb][i];
                    ps[kb][i] = x;
                } else {
                    part += x;
                }
            }
            lack += part;
        }
        if constexpr (kHalf) {
            keep_range(ds, up, acc, round);
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
                Frag<T> fp;
                if constexpr (kFix) {
                    fp = pack<T>(ps[kb], e);
                    round = sum_of(f, round);
                }
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    const Frag<T> t = Tl::turned(sk, kb * 32 + 16 * e, d, lane);
                    acc[d] = mma(t, f, acc[d]);
                    if constexpr (kFix) mean[d] = mma(t, fp, mean[d]);
                }
            }
    }
    constexpr float kDown = kHalf ? 1.0f / kPUp : 1.0f;
    lack = add_halves(lack) * kDown;
    round = add_halves(round) * kDown / up;
    if (!live) return;
    if (lse == -INFINITY) {
        // a row without keys: dy that is not finite by their zeros
        delta = lack = round = 0.0f;
#pragma unroll
        for (int d = 0; d < DB; ++d) acc[d] = mean[d] = f32x16{};
    }
    const float share = kFix || g.splits > 1 ? 1.0f : share_of(lack);
    const float f = s.scale * share * kDown / up, fm = s.scale * kDown;
    if (g.splits > 1) {
        // parts: what dq and the sums P k are so far, and what delta lacks
        const int64_t id = ((int64_t)split * s.N * s.Hk + pair) * s.rows + row;
        float *part = g.part + id * s.D, *part2 = g.part2 + id * s.D;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                store4(part, 32 * d + 8 * b + 4 * h, s.D, kVec || (s.D & 3) == 0, acc[d][4 * b] * f, acc[d][4 * b + 1] * f,
                       acc[d][4 * b + 2] * f, acc[d][4 * b + 3] * f);
                if constexpr (kFix)
                    store4(part2, 32 * d + 8 * b + 4 * h, s.D, kVec || (s.D & 3) == 0, mean[d][4 * b] * fm,
                           mean[d][4 * b + 1] * fm, mean[d][4 * b + 2] * fm, mean[d][4 * b + 3] * fm);
            }
        if (h == 0) {
            g.stat[id * 2] = lack;
            g.stat[id * 2 + 1] = round;
            if (split == 0) {
                g.delta[pair * s.rows + row] = delta;
                g.offset[pair * s.rows + row] = off;
            }
        }
        return;
    }
    if (h == 0) {
        const int64_t at = pair * s.rows + row;
        g.delta[at] = kFix ? delta + lack : delta;
        g.offset[at] = off;
        if constexpr (!kFix) g.share[at] = share;
    }
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            acc[d][i] *= f;
            if constexpr (kFix) acc[d][i] -= round * (mean[d][i] * fm);
        }
    T* dq = (T*)g.b.dq + me.tok * s.ldq + (int64_t)me.head * s.D;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int b = 0; b < 4; ++b)
            store4(dq, 32 * d + 8 * b + 4 * h, s.D, kVec, acc[d][4 * b], acc[d][4 * b + 1], acc[d][4 * b + 2],
                   acc[d][4 * b + 3]);
}

// dq of rows whose keys were taken in parts, and their delta.
template <typename T>
__global__ __launch_bounds__(256) void k_attn_dq_join(AttnK g) {
    const AttnShape& s = g.s;
    // with parts there are fewer than 2^31 values
    const int64_t rows = (int64_t)s.N * s.Hk * s.rows, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t id = (uint32_t)i / (uint32_t)s.D;
    if (id >= rows) return;
    const int d = (int)(i - id * s.D);
    float sum = 0.0f, mean = 0.0f, lack = 0.0f, round = 0.0f;
#pragma unroll 8
    for (int k = 0; k < g.splits; ++k) {
        const int64_t at = k * rows + id;
        sum += g.part[at * s.D + d];
        lack += g.stat[at * 2];
        if constexpr (sizeof(T) == 2) {
            mean += g.part2[at * s.D + d];
            round += g.stat[at * 2 + 1];
        }
    }
    const int64_t pair = (uint32_t)id / (uint32_t)s.rows, row = id - pair * s.rows;
    const int n = (int)fdiv((uint32_t)pair, g.heads);
    const RowAt me = row_at(g, n, (int)(pair - (int64_t)n * s.Hk), row);
    T* dq = (T*)g.b.dq + me.tok * s.ldq + (int64_t)me.head * s.D;
    if constexpr (sizeof(T) == 2) {
        dq[d] = (T)(sum - round * mean);
        if (d == 0) g.delta[id] += lack;
    } else {
        dq[d] = sum * share_of(lack);
        if (d == 0) g.share[id] = share_of(lack);
    }
}

// The rows' tiles, of q and dy, of a walk over a pair's rows up to hi.
template <typename T, int D16, int RT, int NT, int kHow>
struct RowTiles {
    Moving<T, D16, RT, NT> mq, mo;
    const AttnK* g;
    int n, hk;
    int64_t hi;
    __device__ __forceinline__ void init(const AttnK& g_, int n_, int hk_, int64_t hi_) {
        g = &g_; n = n_; hk = hk_; hi = hi_;
    }
    __device__ __forceinline__ void load(int64_t r0, char*, char*) {
        const AttnShape& s = g->s;
        mq.load([&](int r) {
            const RowAt x = row_at(*g, n, hk, r0 + r);
            return r0 + r < hi ? (const T*)g->b.q + x.tok * s.ldq + (int64_t)x.head * s.D : nullptr;
        }, s.D, kHow == kWords);
        mo.load([&](int r) {
            const RowAt x = row_at(*g, n, hk, r0 + r);
            return r0 + r < hi ? (const T*)g->b.dy + (x.tok * s.Hq + x.head) * s.D : nullptr;
        }, s.D, kHow == kWords);
    }
    __device__ __forceinline__ void store(char* sq, char* so) const {
        mq.store(sq);
        mo.store(so);
    }
};
// Straight to LDS.  rep divides a tile's rows: its tokens are whole, and offsets the same in
// every tile.
template <typename T, int D16, int RT, int NT>
struct RowTiles<T, D16, RT, NT, kStraight> {
    using Tl = Tile<T, D16, RT>;
    Direct<Tl, RT, NT> mq, mo;
    const T *q, *dy;
    FastDiv rep;
    int64_t hi;
    uint32_t ldq, ldo, row;
    __device__ __forceinline__ void init(const AttnK& g, int n, int hk, int64_t hi_) {
        const AttnShape& s = g.s;
        const RowAt x = row_at(g, n, hk, 0);
        hi = hi_;
        rep = g.rep;
        ldq = s.ldq;
        ldo = s.Hq * s.D;
        row = s.rep * s.D;
        q = (const T*)g.b.q + x.tok * s.ldq + (int64_t)x.head * s.D;
        dy = (const T*)g.b.dy + (x.tok * s.Hq + x.head) * s.D;
        auto place = [&](Direct<Tl, RT, NT>& m, uint32_t ld) {
            m.init(s.D / 8, [&](int r, int chunk) {
                const uint32_t t = fdiv((uint32_t)r, g.rep);
                return (t * ld + ((uint32_t)r - t * s.rep) * s.D) * 2 + chunk * 16;
            });
        };
        place(mq, ldq);
        place(mo, ldo);
    }
    __device__ __forceinline__ void load(int64_t r0, char* sq, char* so) {
        const int64_t left = hi - r0, t = fdiv((uint32_t)r0, rep);
        const uint32_t last = fdiv((uint32_t)(left < RT ? left : RT), rep) - 1;
        mq.issue(sq, q + t * ldq, (last * ldq + row) * 2);
        mo.issue(so, dy + t * ldo, (last * ldo + row) * 2);
    }
    __device__ __forceinline__ void store(char*, char*) const {}
};

// dk and dv of 64 keys: a wave owns 32 of them and every other 32 of the pair's rows, and
// the two waves of 32 keys join at the end (128 keys a workgroup, a wave to 32: half as many
// workgroups, each twice as long, one wave a SIMD where lengths are ragged, 288 us in place
// of 225 for 16 images of 3136 by 0 to 1024 tokens, 8 and 4 heads of 64, bf16).  Keys that are
// left out are columns of their own, so what they hold goes nowhere.  Heads of 64 are held to the
// registers of three workgroups a CU: of ragged images no more than 544 of 1024 have keys, and
// with two a CU the last 32 ran alone (217 us and 190; 512 that all have keys 2% slower; fp16, whose
// powers of two would spill, 18%: two).
constexpr int kOwnKeys = 64;
template <typename T, int D16, int kHow>
__global__ __launch_bounds__(256, (kHow == kStraight && D16 == 4 && !std::is_same_v<T, _Float16>
                                       ? 3 : waves_of<T, D16>(kHow == kStraight ? 6 : 4)))
void k_attn_dkv(AttnK g) {
    constexpr bool kDirect = kHow == kStraight, kVec = kHow != kAnywhere;
    constexpr int NT = 256, RT = 64, DB = (D16 + 1) / 2, CP = kCopies<T>;
    constexpr bool kHalf = std::is_same_v<T, _Float16>, kShare = sizeof(T) == 4;
    using Tl = Tile<T, D16, RT>;
    __shared__ alignas(16) char tq[CP][Tl::kBytes];
    __shared__ alignas(16) char to[CP][Tl::kBytes];
    __shared__ alignas(16) float toff[CP][RT], tdel[CP][RT], tshare[CP][kShare ? RT : 4];
    const AttnShape& s = g.s;
    const Work wk = work_of(g);
    if (wk.none) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    const int split = wk.split, n = wk.n, hk = wk.hk;
    const int64_t tile = wk.tile, pair = wk.pair;
    const int len = keys_of(g.b.klen, n, s.Lk);
    const int64_t key = tile * kOwnKeys + (wave & 1) * 32 + (lane & 31);
    const int mine = (wave >> 1) * 32;       // of a tile's rows
    const bool kept = key < len && (!g.b.mask || g.b.mask[(int64_t)n * s.Lk + key]);
    const int64_t tok = (int64_t)n * s.Lk + key;
    const T* k = kept ? (const T*)g.b.k + tok * s.ldk + (int64_t)hk * s.D : nullptr;
    const T* v = kept ? (const T*)g.b.v + tok * s.ldv + (int64_t)hk * s.D : nullptr;
    Frag<T> fk[D16], fv[D16];
#pragma unroll
    for (int c = 0; c < D16; ++c) {
        fk[c] = load_frag(k, c, h, s.D, kVec);
        fv[c] = load_frag(v, c, h, s.D, kVec);
    }
    int64_t lo, hi;
    part_of(tile * kOwnKeys < len ? s.rows : 0, RT, split, g.splits, lo, hi);
    RowTiles<T, D16, RT, NT, kHow> in;
    in.init(g, n, hk, hi);
    float moff = 0.0f, mdel = 0.0f, mshare = 0.0f;
    // rows past hi: P = 1, but their q and dy are zeros
    auto load = [&](int64_t r0, char* sq, char* so, float* offs, float* deltas) {
        in.load(r0, sq, so);
        const int64_t at = pair * s.rows + r0;
        if constexpr (kDirect) {
            if (wave == 0) load_words(offs, g.offset + at, hi - r0);
            if (wave == 1) load_words(deltas, g.delta + at, hi - r0);
        } else if (threadIdx.x < RT) {
            const bool inside = r0 + threadIdx.x < hi;
            moff = inside ? g.offset[at + threadIdx.x] : 0.0f;
            mdel = inside ? g.delta[at + threadIdx.x] : 0.0f;
            if constexpr (kShare) mshare = inside ? g.share[at + threadIdx.x] : 0.0f;
        }
    };

    const float c2 = s.scale * kLog2e;
    float up = kHalf ? 0x1p100f : 1.0f, none = 0.0f;
    f32x16 ak[DB], av[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) ak[d] = av[d] = f32x16{};
    if (lo < hi) load(lo, tq[0], to[0], toff[0], tdel[0]);
    if (kDirect) settled();
    int copy = 0;
    for (int64_t r0 = lo; r0 < hi; r0 += RT) {
        char *sq = tq[copy], *so = to[copy];
        float *offs = toff[copy], *deltas = tdel[copy], *shares = tshare[copy];
        if (CP == 1) __syncthreads();
        else copy ^= 1;
        in.store(sq, so);
        if (!kDirect && threadIdx.x < RT) {
            offs[threadIdx.x] = moff;
            deltas[threadIdx.x] = mdel;
            if constexpr (kShare) shares[threadIdx.x] = mshare;
        }
        if constexpr (kDirect) ready<0>();
        else __syncthreads();
        if (r0 + RT < hi) load(r0 + RT, tq[copy], to[copy], toff[copy], tdel[copy]);
        f32x16 p{}, ds[1] = {f32x16{}};
#pragma unroll
        for (int c = 0; c < D16; ++c) {
            p = mma(Tl::read(sq, mine + (lane & 31), c, h), fk[c], p);
            ds[0] = mma(Tl::read(so, mine + (lane & 31), c, h), fv[c], ds[0]);
        }
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int at = mine + 8 * b + 4 * h;
            const f32x4v o4 = *(const f32x4v*)&offs[at], d4 = *(const f32x4v*)&deltas[at];
            f32x4v s4{};
            if constexpr (kShare) s4 = *(const f32x4v*)&shares[at];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float x = __builtin_amdgcn_exp2f(__builtin_fmaf(p[4 * b + i], c2, o4[i]));
                if constexpr (kShare) x *= s4[i];
                ds[0][4 * b + i] = x * (ds[0][4 * b + i] - d4[i]);
                p[4 * b + i] = x;
            }
        }
        if constexpr (kHalf) {
            keep_range(ds, up, ak, none);
#pragma unroll
            for (int i = 0; i < 16; ++i) ds[0][i] *= up;
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const Frag<T> fp = pack<T>(p, e), fd = pack<T>(ds[0], e);
#pragma unroll
            for (int d = 0; d < DB; ++d) {
                av[d] = mma(Tl::turned(so, mine + 16 * e, d, lane), fp, av[d]);
                ak[d] = mma(Tl::turned(sq, mine + 16 * e, d, lane), fd, ak[d]);
            }
        }
    }
    const float fvv = kHalf ? 1.0f / kPUp : 1.0f, f = s.scale * fvv / up;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            ak[d][i] *= f;
            av[d][i] *= fvv;
        }
    // the second half of the rows, by way of LDS, 32 channels at a time
    static_assert(sizeof(tq) >= 2 * 16 * 64 * sizeof(float));
    float *xk = (float*)tq[0] + (wave & 1) * 1024, *xv = (float*)to[0] + (wave & 1) * 1024;
#pragma unroll
    for (int d = 0; d < DB; ++d) {
        __syncthreads();
        if (mine) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                xk[i * 64 + lane] = ak[d][i];
                xv[i * 64 + lane] = av[d][i];
            }
        }
        __syncthreads();
        if (!mine) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                ak[d][i] += xk[i * 64 + lane];
                av[d][i] += xv[i * 64 + lane];
            }
        }
    }
    if (mine || key >= s.Lk) return;
    auto put = [&](auto* dk, auto* dv, bool vec) {
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                float x[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x[i] = kept ? ak[d][4 * b + i] : 0.0f;
                    x[4 + i] = kept ? av[d][4 * b + i] : 0.0f;
                }
                store4(dk, 32 * d + 8 * b + 4 * h, s.D, vec, x[0], x[1], x[2], x[3]);
                store4(dv, 32 * d + 8 * b + 4 * h, s.D, vec, x[4], x[5], x[6], x[7]);
            }
    };
    if (g.splits > 1) {
        const int64_t id = (((int64_t)split * s.N * s.Hk + pair) * s.Lk + key) * s.D;
        put(g.part + id, g.part2 + id, kVec || (s.D & 3) == 0);
    } else {
        put((T*)g.b.dk + tok * s.ldk + (int64_t)hk * s.D, (T*)g.b.dv + tok * s.ldv + (int64_t)hk * s.D, kVec);
    }
}

// dk (blockIdx.y 0) or dv of keys whose rows were taken in parts.
template <typename T>
__global__ __launch_bounds__(256) void k_attn_sum(AttnK g) {
    const AttnShape& s = g.s;
    const int64_t all = (int64_t)s.N * s.Hk * s.Lk * s.D, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= all) return;
    const float* p = blockIdx.y ? g.part2 : g.part;
    float sum = 0.0f;
#pragma unroll 8
    for (int k = 0; k < g.splits; ++k) sum += p[k * all + i];
    // with parts there are fewer than 2^31 values
    const int64_t id = (uint32_t)i / (uint32_t)s.D, pair = (uint32_t)id / (uint32_t)s.Lk, n = fdiv((uint32_t)pair, g.heads);
    const int64_t tok = n * s.Lk + (id - pair * s.Lk);
    T* x = (T*)(blockIdx.y ? g.b.dv : g.b.dk) + tok * (blockIdx.y ? s.ldv : s.ldk);
    x[(pair - n * s.Hk) * s.D + (i - id * s.D)] = (T)sum;
}

// ---------------------------------------------------------------- launches

// Sets a launch's cut; the number of its workgroups (below 2^31: attn_plan).
inline unsigned cut(AttnK& a, const AttnCut& c) {
    const int64_t pairs = (int64_t)a.s.N * a.s.Hk;
    a.tiles = c.tiles;
    a.splits = c.splits;
    a.per_pair = make_fastdiv((uint32_t)(c.tiles * c.splits));
    a.per_tile = make_fastdiv((uint32_t)c.splits);
    a.by_xcd = pairs % 8 == 0 || pairs >= 64;
    return (unsigned)((a.by_xcd ? (pairs + 7) / 8 * 8 : pairs) * c.tiles * c.splits);
}

template <typename T, int D16, int kHow>
hipError_t attn_run_by(const AttnK& g, const AttnPlan& p, bool backward, hipStream_t st) {
    AttnK a = g;
    const AttnShape& s = g.s;
    const int64_t pairs = (int64_t)s.N * s.Hk;
    unsigned blocks = cut(a, p.rows);
    if (!backward) {
        if (p.few)
            k_attn<T, D16, true, kHow><<<blocks, FwdCut<T, D16, true>::kThreads, 0, st>>>(a);
        else
            k_attn<T, D16, false, kHow><<<blocks, FwdCut<T, D16, false>::kThreads, 0, st>>>(a);
        if (a.splits > 1) {
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
            // one part a wave at a time
            if (a.splits > 8) k_attn_join<T, 4><<<(unsigned)(pairs * s.rows), 256, 0, st>>>(a);
            else k_attn_join<T, 1><<<(unsigned)((pairs * s.rows + 3) / 4), 256, 0, st>>>(a);
        }
        return hipGetLastError();
    }
    a.part2 = a.part + (size_t)a.splits * pairs * s.rows * s.D;
    k_attn_dq<T, D16, kHow><<<blocks, 256, 0, st>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (a.splits > 1) {
        k_attn_dq_join<T><<<(unsigned)((pairs * s.rows * s.D + 255) / 256), 256, 0, st>>>(a);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    blocks = cut(a, p.keys);
    a.part2 = a.part + (size_t)a.splits * pairs * s.Lk * s.D;
    // straight to LDS tokens are whole in a tile of 64 rows
    if (kHow == kStraight && 64 % s.rep) k_attn_dkv<T, D16, kWords><<<blocks, 256, 0, st>>>(a);
    else k_attn_dkv<T, D16, kHow><<<blocks, 256, 0, st>>>(a);
    e = hipGetLastError();
    if (e != hipSuccess || a.splits == 1) return e;
    k_attn_sum<T><<<dim3((unsigned)((pairs * s.Lk * s.D + 255) / 256), 2), 256, 0, st>>>(a);
    return hipGetLastError();
}

// vec: vectors of whole 16-byte words.  16-bit tiles of them go straight to LDS where the rows
// of a tile, 64 of them, are within 2^31 bytes.
template <typename T, int D16>
hipError_t attn_run(const AttnK& g, const AttnPlan& p, bool backward, hipStream_t st) {
    constexpr int kMost = 1 << 22;
    const AttnShape& s = g.s;
    if constexpr (sizeof(T) == 4) {
        if (g.vec) return attn_run_by<T, D16, kWords>(g, p, backward, st);
    } else if (g.vec && s.ldq <= kMost && s.ldk <= kMost && s.ldv <= kMost && s.Hq * s.D <= kMost) {
        return attn_run_by<T, D16, kStraight>(g, p, backward, st);
    }
    return attn_run_by<T, D16, kAnywhere>(g, p, backward, st);
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
