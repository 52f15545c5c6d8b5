// The gated layer of channel-last tensors, y = act(zg) * zu with zg = x w0^T + b0 and
// zu = x w1^T + b1, and its backward pass
//   dzg = dy zu act'(zg), dzu = dy act(zg), dx = dzg w0 + dzu w1, dw = dz^T x, db = sum dz.
//
// Matrix products on 32x32 matrix-core tiles, their operands staged through LDS: the left
// operand's index runs down a lane's registers and is the output's contiguous one, the right
// operand's runs over the lanes.  Forward, half a workgroup's left rows are units' gates, half their values, so
// that both of a unit meet in one lane and neither leaves it.  Backward is three products:
// zg and zu once more, ending in dz (kept in the tensors' type, as any gradient between two
// layers; fp16: times a power of two), then dx from dz and w, and dw from dz and x, the sum over
// tokens in parts.
//
// 6272 tokens of 512 channels by 2048 units, bf16, forward: 40 us, 0.65 PFLOP/s; 200704 of 256
// by 1024, backward: 957 to 990 us, of which dz's way through memory, 2.4 GB, is 400 at 6.2 TB/s; fp16:
// 1032, and 1574 where dz is formed again.
#include "wino_attn_device.h"
#include "wino_checks.h"
#include "wino_gated.h"
#include "wino_norm_device.h"

namespace wino {

namespace {

__host__ __device__ inline int64_t tiles_of(int64_t n, int each) { return (n + each - 1) / each; }

struct GatedK {
    GatedArgs a;
    int64_t M;
    int C, K;
    Act act;
    bool vec;
    void* dz;                                // [M][2 K]
    float *dbias, *part;                     // [token tiles][2 K]; [splits][2 K][C]
    float *tops, *ups;                       // fp16: each tile's largest |dz|; dz's power of two, and 1 over it
    int items, tiles;                        // below 2^24; tiles: of the faster axis
    int splits;
};

// How a workgroup's four waves share a tile: WA by WB of them, each AB by BB blocks of 32
// by 32 results.  A block's step reads AB + BB operands from LDS for AB * BB products, and a
// tile's step kA + kB rows of 64 bytes from L2, so wide tiles need the least of both; narrow ones
// fill the card where results are few (figures at cut_of).
template <int AB_, int BB_, int WA_, int WB_>
struct Shape {
    static constexpr int AB = AB_, BB = BB_, WA = WA_, WB = WB_;
    static constexpr int kA = 32 * AB * WA, kB = 32 * BB * WB;      // indices of a tile
};
using Wide = Shape<4, 2, 1, 4>;              // 128 x 256
using Square = Shape<2, 2, 2, 2>;            // 128 x 128
using Narrow = Shape<2, 1, 1, 4>;            // 64 x 128
using Small = Shape<1, 1, 2, 2>;             // 64 x 64

constexpr int kBk = 32;                      // terms of a step

// A matrix in memory, [index][sum], or [sum][index] (T_): `rows` rows of `cols` values, ld
// apart.  Rows from `split` on lie `jump` further.
template <typename T>
struct Source {
    const T* p;
    int64_t rows;
    int cols, ld, split, jump;
};

// One operand's tile of I indices by kBk terms.
template <typename T, int I, bool T_, bool kDirect>
struct Side {
    typedef T Value;
    static constexpr int kRows = T_ ? kBk : I;
    // rows of more than 128 values in halves of 128, each a tile
    static constexpr int kCols = T_ ? (I < 128 ? I : 128) : kBk, kParts = T_ ? I / kCols : 1;
    using Tl = Tile<T, kCols / 16, kRows>;
    static constexpr int kBytes = Tl::kBytes * kParts, kLoads = 0;
    Source<T> s;
    bool vec;
    Moving<T, kCols / 16, kRows, 256> m[kParts];

    __device__ __forceinline__ void init(const Source<T>& s_, bool vec_) {
        s = s_;
        vec = vec_;
    }
    int64_t k;
    __device__ __forceinline__ void begin(int64_t k_) { k = k_; }
    __device__ __forceinline__ void load(char*, int left) {
#pragma unroll
        for (int i = 0; i < kParts; ++i)
            m[i].load([&](int r) {
                if constexpr (T_) {
                    return r < left ? s.p + (k + r) * s.ld + i * kCols : nullptr;
                } else {
                    const int64_t row = r + (r >= s.split ? s.jump : 0);
                    return row < s.rows ? s.p + row * s.ld + k : nullptr;
                }
            }, T_ ? s.cols - i * kCols : left, vec);
        k += kBk;
    }
    __device__ __forceinline__ void store(char* t) const {
#pragma unroll
        for (int i = 0; i < kParts; ++i) m[i].store(t + i * Tl::kBytes);
    }
    // terms 16 c .. of indices 32 blk ..
    __device__ static __forceinline__ Frag<T> read(const char* t, int blk, int c, int lane) {
        if constexpr (T_) return Tl::turned8(t + blk / (kCols / 32) * Tl::kBytes, 16 * c, blk % (kCols / 32), lane);
        else return Tl::read(t, 32 * blk + (lane & 31), c, lane >> 5);
    }
};
// fp32 as it is in memory: R rows of W values.  Operands are split as they are read: 22
// vector instructions for eight values, beside the 6 products of 32 cycles each that they
// enter, and the tile is on its way while two others are worked on.
template <int R, int W>
struct Whole {
    static constexpr int kRow = W * 4, kBytes = R * kRow;
    __device__ static __forceinline__ int twist(int row) { return kRow == 128 ? ((row & 2) << 1) | ((row >> 2) & 3) : 0; }
    __device__ static __forceinline__ int at(int row, int chunk) { return row * kRow + ((chunk ^ twist(row)) << 4); }
    __device__ static __forceinline__ Frag<float> read(const char* t, int row, int c, int h) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const f32x4v v = *(const f32x4v*)(t + at(row, 4 * c + 2 * h + e));
#pragma unroll
            for (int i = 0; i < 4; ++i) x[4 * e + i] = v[i];
        }
        return frag_of<float>(x);
    }
    // column 32 db + lane % 32 of rows r + 8 h .. + 7
    __device__ static __forceinline__ Frag<float> turned8(const char* t, int r, int db, int lane) {
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            x[i] = *(const float*)(t + (r + 8 * (lane >> 5) + i) * kRow + (32 * db + (lane & 31)) * 4);
        return frag_of<float>(x);
    }
};

// Straight to LDS: values in whole 16-byte words, a tile within 2^31 bytes.
template <typename T, int I, bool T_>
struct Side<T, I, T_, true> {
    typedef T Value;
    static constexpr int kRows = T_ ? kBk : I;
    static constexpr int kCols = T_ ? (I < 128 ? I : 128) : kBk, kParts = T_ ? I / kCols : 1;
    using Tl = std::conditional_t<sizeof(T) == 4, Whole<kRows, kCols>, Tile<T, kCols / 16, kRows>>;
    using Dir = Direct<Tl, kRows, 256>;
    static constexpr int kBytes = Tl::kBytes * kParts, kEach = 16 / (int)sizeof(T), kSize = sizeof(T);
    static constexpr int kLoads = Dir::kN * kParts;                 // of a lane, a tile
    Source<T> s;
    Dir d[kParts];
    Buffer r;                                // of the next tile's rows (T_), or of all of them
    uint32_t at, all, step;                  // bytes to its first term (not T_); of its buffer, and to the one after it (T_)
    __device__ __forceinline__ void init(const Source<T>& s_, bool) {
        s = s_;
#pragma unroll
        for (int i = 0; i < kParts; ++i)
            d[i].init(T_ ? (s.cols - i * kCols + kEach - 1) / kEach : 1 << 20, [&](int r, int chunk) {
                const uint32_t row = (uint32_t)r + (!T_ && r >= s.split ? (uint32_t)s.jump : 0u);
                return row * (uint32_t)s.ld * kSize + chunk * 16 + i * kCols * kSize;
            });
    }
    // the next load's terms are k ..
    __device__ __forceinline__ void begin(int64_t k) {
        if constexpr (T_) {
            all = ((kBk - 1) * (uint32_t)s.ld + (uint32_t)s.cols) * kSize;
            step = kBk * (uint32_t)s.ld * kSize;
            r = buffer_of(s.p + k * s.ld, all);
        } else {
            const int64_t bytes = ((s.rows - 1) * s.ld + s.cols) * kSize;
            r = buffer_of(s.p, bytes < 0x7fffffff ? (uint32_t)bytes : 0x7fffffffu);
            at = (uint32_t)k * kSize;
        }
    }
    // the tile of the next kBk terms, `left` of them there; to LDS at t
    __device__ __forceinline__ void load(char* t, int left) {
        if constexpr (T_) {
            r[2] = left >= kBk ? all : ((uint32_t)(left - 1) * (uint32_t)s.ld + (uint32_t)s.cols) * kSize;
#pragma unroll
            for (int i = 0; i < kParts; ++i) d[i].issue_at(Dir::place(t + i * Tl::kBytes), r, 0);
            const uint64_t p = ((uint64_t)r[1] << 32 | r[0]) + step;
            r[0] = (uint32_t)p;
            r[1] = (uint32_t)(p >> 32);
        } else {
            if (left >= kBk) d[0].issue_at(Dir::place(t), r, at);
            else d[0].part((left + kEach - 1) / kEach).issue_at(Dir::place(t), r, at);
            at += kBk * kSize;
        }
    }
    __device__ __forceinline__ void store(char*) const {}
    // terms 16 c .. of indices 32 blk ..
    __device__ static __forceinline__ Frag<T> read(const char* t, int blk, int c, int lane) {
        if constexpr (T_) return Tl::turned8(t + blk / (kCols / 32) * Tl::kBytes, 16 * c, blk % (kCols / 32), lane);
        else return Tl::read(t, 32 * blk + (lane & 31), c, lane >> 5);
    }
};

// Copies of the tiles that lie in LDS straight from memory; of fp32's squares two, for two
// workgroups a CU.
template <typename T, typename S>
constexpr int copies_of() {
    return sizeof(T) == 4 && S::AB * S::BB == 4 ? 2 : 3;
}

// acc[i][j] = products of the wave's left block i and right block j, over the terms lo .. hi.
// Left block i of wave column wa: i * WA + wa.  after(i, t), straight to LDS alone: issues
// kAfter loads to a copy t whose tiles are done with, as the last steps begin (i 0 and 1);
// they have arrived when their reader is ready().
struct Nothing {
    static constexpr int kAfter = 0;
    __device__ __forceinline__ void operator()(int, char*) const {}
};
template <typename S, typename A, typename B, typename F = Nothing>
__device__ __forceinline__ void product(f32x16 (&acc)[S::AB][S::BB], A& a, B& b, char* lds, int64_t lo, int64_t hi,
                                        bool direct, const F& after = F()) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wa = wave % S::WA, wb = wave / S::WA;
    constexpr int kBoth = A::kBytes + B::kBytes;
#pragma unroll
    for (int i = 0; i < S::AB; ++i)
#pragma unroll
        for (int j = 0; j < S::BB; ++j) acc[i][j] = f32x16{};
    a.begin(lo);
    b.begin(lo);
    int left = (int)(hi - lo);               // terms from this step's on
    // the tiles of the next step, `n` terms there
    auto load = [&](int copy, int n) {
        a.load(lds + copy * kBoth, n);
        b.load(lds + copy * kBoth + A::kBytes, n);
    };
    decltype(A::read(lds, 0, 0, 0)) fa[2][S::AB];
    decltype(B::read(lds, 0, 0, 0)) fb[2][S::BB];
    auto read = [&](const char* t, int c) {
#pragma unroll
        for (int i = 0; i < S::AB; ++i) fa[c][i] = A::read(t, i * S::WA + wa, c, lane);
#pragma unroll
        for (int j = 0; j < S::BB; ++j) fb[c][j] = B::read(t + A::kBytes, wb * S::BB + j, c, lane);
    };
    auto multiply = [&](int c) {
#pragma unroll
        for (int i = 0; i < S::AB; ++i)
#pragma unroll
            for (int j = 0; j < S::BB; ++j) acc[i][j] = mma(fa[c][i], fb[c][j], acc[i][j]);
    };
    static_assert(kBk == 32);
    // straight to LDS: one step ahead in two copies, two steps in three
    constexpr int N = copies_of<typename A::Value, S>();
    int copy = 0;
    if (left > 0) load(0, left);
    if (direct && N == 3) {
        // Half a step's products run while the other half's operands are on their way, and the
        // wait for the next tile is between the halves: its first operands, read right after,
        // have the second half's products to arrive in.  A tile is done with once its step's wait
        // is passed.
        constexpr int kLoads = A::kLoads + B::kLoads;
        const bool one = left <= kBk;
        if (!one) {
            load(1, left - kBk);
            ready<kLoads>();
        } else {
            ready<0>();
        }
        read(lds, 0);
        for (; left > 0; left -= kBk) {
            const char* t = lds + copy * kBoth;
            const int before = copy == 0 ? 2 : copy - 1;
            copy = copy == 2 ? 0 : copy + 1;
            read(t, 1);
            if (left > 2 * kBk) {
                load(before, left - 2 * kBk);
            } else if (F::kAfter > 0) {
                const bool last = left <= kBk;
                if (!last || one) after(0, lds + before * kBoth);
                if (last) after(1, lds + (one ? copy : before) * kBoth);
            }
            __builtin_amdgcn_sched_barrier(0);
            multiply(0);
            __builtin_amdgcn_sched_barrier(0);
            if (left > kBk) {
                if (left > 2 * kBk) ready<kLoads>();
                else ready<F::kAfter>();
                read(lds + copy * kBoth, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
            multiply(1);
        }
        if (F::kAfter > 0) ready<0>();
        else __syncthreads();                // the tiles' LDS is free
        return;
    }
    for (; left > 0; left -= kBk) {
        char* t = lds + copy * kBoth;
        if (direct) {
            ready<0>();
            copy ^= 1;
            if (left > kBk) load(copy, left - kBk);
        } else {
            __syncthreads();
            a.store(t);
            b.store(t + A::kBytes);
            __syncthreads();
            if (left > kBk) load(0, left - kBk);
        }
#pragma unroll
        for (int c = 0; c < kBk / 16; ++c) {
            read(t, c);
            multiply(c);
        }
    }
    __syncthreads();                         // the tiles' LDS is free
}

// A wave's 32 rows by 64 columns on their way between a lane's order (a row; columns 32 w
// + 8 b + 4 h + i) and memory's (16 bytes a lane, whole rows in turn), by way of LDS.
template <typename O>
struct Rows64 {
    static constexpr int kEach = 16 / (int)sizeof(O), kRow = 64 * (int)sizeof(O) + 16, kBytes = 32 * kRow;
    static constexpr int kLanes = 64 / kEach;                       // of a row
    char* t;                                                        // the wave's own kBytes
    // four values of the lane's row, to columns c .. c + 3
    __device__ __forceinline__ void put4(int c, float a, float b, float d, float e) const {
        const O v[4] = {(O)a, (O)b, (O)d, (O)e};
        __builtin_memcpy(__builtin_assume_aligned(t + (threadIdx.x & 31) * kRow + c * (int)sizeof(O), 8), v, sizeof(v));
    }
    __device__ __forceinline__ void get4(int c, float (&v)[4]) const {
        O o[4];
        __builtin_memcpy(o, __builtin_assume_aligned(t + (threadIdx.x & 31) * kRow + c * (int)sizeof(O), 8), sizeof(o));
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = (float)o[i];
    }
    // rows r < rows, columns c < cols (of 64), to or from p + r * ld + c
    template <bool kStore>
    __device__ __forceinline__ void move(std::conditional_t<kStore, O, const O>* p, int64_t ld, int rows, int cols,
                                         bool vec) const {
        const int lane = threadIdx.x & 63, c = lane % kLanes * kEach;
#pragma unroll
        for (int r0 = 0; r0 < 32; r0 += 64 / kLanes) {
            const int r = r0 + lane / kLanes;
            char* q = t + r * kRow + c * (int)sizeof(O);
            if (r >= rows) continue;
            if (vec || c + kEach <= cols) {
                if (c >= cols) continue;
                // 16 bytes on any address
                if constexpr (kStore) __builtin_memcpy(p + r * ld + c, __builtin_assume_aligned(q, 16), 16);
                else __builtin_memcpy(__builtin_assume_aligned(q, 16), p + r * ld + c, 16);
            } else {
                for (int i = 0; i < kEach; ++i) {
                    if (c + i >= cols) break;
                    if constexpr (kStore) p[r * ld + c + i] = ((const O*)q)[i];
                    else ((O*)q)[i] = p[r * ld + c + i];
                }
            }
        }
    }
};
// LDS of one wave is read as it was written.
__device__ __forceinline__ void wave_sync() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); __builtin_amdgcn_wave_barrier(); }

// The sum of each of 16 values over the 32 lanes of a half: value 8 b4 + 4 b3 + 2 b2 + b1 of
// lane bits b.  Each exchange halves the values.
__device__ __forceinline__ float sum16(float (&v)[16]) {
    const int lane = threadIdx.x;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v[i]), __float_as_uint(v[i + 8]), false, false);
        v[i] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    auto fold = [&](auto dpp, int bit, int n) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (i >= n) break;
            const float keep = lane & bit ? v[i + n] : v[i], give = lane & bit ? v[i] : v[i + n];
            v[i] = keep + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(give), decltype(dpp)::value, 15, 15, true));
        }
    };
    fold(std::integral_constant<int, 0x128>(), 8, 4);       // row_ror:8
    fold(std::integral_constant<int, 0x141>(), 4, 2);       // row_half_mirror
    fold(std::integral_constant<int, 0x4e>(), 2, 1);        // quad_perm 2 3 0 1
    return v[0] + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v[0]), 0xb1, 15, 15, true));
}

// Workgroups that share a tile's tokens follow each other on one XCD, whose L2 then holds
// them: workgroup ids go round the eight XCDs.  Item of `all`, or -1.
__device__ __forceinline__ int item_of(int all) {
    const int each = (all + 7) / 8, i = (int)(blockIdx.x & 7) * each + (int)(blockIdx.x >> 3);
    return (int)(blockIdx.x >> 3) < each && i < all ? i : -1;
}
inline unsigned grid_of(int64_t items) { return (unsigned)((items + 7) / 8 * 8); }

__device__ __forceinline__ float sigmoid(float z) {
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-z * kLog2e));
}
__device__ __forceinline__ float gate(float z, Act act) {
    return act == Act::Relu ? (z > 0.0f ? z : z == z ? 0.0f : z) : act == Act::Silu ? z * sigmoid(z) : z;
}
// act(z) and its slope (ReLU: 0 at z <= 0)
__device__ __forceinline__ void gate_slope(float z, Act act, float& v, float& d) {
    if (act == Act::Silu) {
        const float s = sigmoid(z);
        v = z * s;
        d = s * (1.0f + z * (1.0f - s));
    } else if (act == Act::Relu) {
        v = gate(z, act);
        d = z > 0.0f ? 1.0f : 0.0f;
    } else {
        v = z;
        d = 1.0f;
    }
}

template <typename S, typename A, typename B>
constexpr int lds_of(bool direct, int rows_bytes) {
    const int tiles = (A::kBytes + B::kBytes) * (direct ? copies_of<typename A::Value, S>() : 1), rows = 4 * rows_bytes;
    return tiles > rows ? tiles : rows;
}

// dy of 128 tokens (32 of each wave) by 64 units, straight to LDS while a wide tile's last
// steps run: read afterwards, it held up every workgroup twice (200704 tokens of 256 channels by
// 1024 units: 620 us).
template <typename T>
struct DyTiles {
    using Tl = Tile<T, 4, 128>;
    using Dir = Direct<Tl, 128, 256>;
    static constexpr int kAfter = Dir::kN;
    Dir d;
    const T* p;
    int64_t left;
    int K, cols;
    char** at;
    __device__ __forceinline__ DyTiles(const T* p_, int64_t left_, int K_, int cols_, char** at_)
        : p(p_), left(left_), K(K_), cols(cols_), at(at_) {
        d.init((cols + 7) / 8, [&](int r, int chunk) { return (uint32_t)(r / 32 * 64 + r % 32) * (uint32_t)K * 2 + chunk * 16; });
    }
    __device__ __forceinline__ void operator()(int i, char* t) const {
        at[i] = t;
        const int64_t n = left - 32 * i;             // tokens from this block's first on
        d.issue(t, p + (int64_t)32 * i * K, n > 0 ? (uint32_t)((n - 1) * K + cols) * 2 : 0);
    }
};

// fp16's dz is held times a power of two: of 2^6, and where the call's largest would then be past
// fp16's range, or below 2^-2 (from where 2^-12 of it has all its bits), formed again times one that
// brings the largest to 2^13 or more.  Infinities and NaN are no part of it.
constexpr float kFirstUp = 64.0f;
constexpr int kFirstUpLog = 6;
// top: the largest times the first power of two
__device__ __forceinline__ float up_of(float top) {
    if (top == 0.0f || (top >= 0.25f && top <= 65504.0f)) return kFirstUp;
    const int e = (int)(__float_as_uint(top) >> 23) - 127;          // of a subnormal -127
    return __uint_as_float((uint32_t)(min(kFirstUpLog + 13 - e, 126) + 127) << 23);
}

// The sum, or the largest, of a wave's 64 values (the largest: of numbers from 0 on).
template <bool kMax = false>
__device__ __forceinline__ float join64(float x) {
    auto two = [](float a, float b) { return kMax ? fmaxf(a, b) : a + b; };
#define WINO_ROTATED(ctrl) __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), ctrl, 15, 15, true))
    x = two(x, WINO_ROTATED(0x128));         // row_ror:8, 4, 2, 1
    x = two(x, WINO_ROTATED(0x124));
    x = two(x, WINO_ROTATED(0x122));
    x = two(x, WINO_ROTATED(0x121));
#undef WINO_ROTATED
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = two(__uint_as_float(r[0]), __uint_as_float(r[1]));
    float a, b;
    halves(x, a, b);
    return two(a, b);
}

// y of a tile's tokens and units (its left rows are their gates, then their values, so that
// both of a unit meet in one lane), or dz of them, the tile's sums of it and (fp16) its largest;
// kAgain: dz alone, times `up`.
template <typename T, typename S, bool BACK, bool kDirect, bool kAgain>
__device__ __forceinline__ void gated_tile(const GatedK& g, int item, float up) {
    constexpr bool kHalf = BACK && std::is_same_v<T, _Float16>;
    constexpr int kUnits = S::kA / 2, UB = S::AB / 2;
    using A = Side<T, S::kA, false, kDirect>;
    using B = Side<T, S::kB, false, kDirect>;
    using Rows = Rows64<T>;
    __shared__ alignas(16) char lds[lds_of<S, A, B>(kDirect, Rows::kBytes)];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    const int mt = (uint32_t)item / (uint32_t)g.tiles, u0 = (item - mt * g.tiles) * kUnits, K = g.K;
    const int64_t m0 = (int64_t)mt * S::kB;
    constexpr bool kAhead = BACK && kDirect && S::AB == 4 && sizeof(T) == 2;
    // loaded once: a load between stores would wait for them
    __shared__ alignas(16) float bias[2 * kUnits];
    if (threadIdx.x < 2 * kUnits) {
        const int u = u0 + threadIdx.x % kUnits;
        bias[threadIdx.x] = g.a.bias && u < K ? g.a.bias[threadIdx.x / kUnits * K + u] : 0.0f;
    }
    char* dys[2] = {lds, lds};
    f32x16 acc[S::AB][S::BB];                            // gates, then values, by blocks of 32 tokens
    {
        A a;
        B b;
        a.init({(const T*)g.a.w + (int64_t)u0 * g.C, 2 * (int64_t)K - u0, g.C, g.C, kUnits, K - kUnits}, g.vec);
        b.init({(const T*)g.a.x + m0 * g.C, g.M - m0 < S::kB ? g.M - m0 : S::kB, g.C, g.C, S::kB, 0}, g.vec);
        if constexpr (kAhead) {
            const DyTiles<T> dy((const T*)g.a.dy + m0 * K + u0, g.M - m0 < S::kB ? g.M - m0 : S::kB, K,
                                K - u0 < kUnits ? K - u0 : kUnits, dys);
            product<S>(acc, a, b, lds, 0, g.C, true, dy);
        } else {
            product<S>(acc, a, b, lds, 0, g.C, kDirect);
        }
    }
    // a wave's 32 tokens by 64 columns at a time: its units' gates, or their values; where dy
    // is there already, in the copy that the last step read
    char* free = lds;
    if constexpr (kAhead) {
        constexpr int kBoth = A::kBytes + B::kBytes;
        static_assert(kBoth >= 4 * Rows::kBytes && kBoth >= DyTiles<T>::Tl::kBytes);
        free = lds + (tiles_of(g.C, kBk) - 1) % 3 * kBoth;
    }
    const Rows rows{free + wave * Rows::kBytes};
    const int wa = wave % S::WA, wb = wave / S::WA;
    static_assert(S::AB == 2 || S::WA == 1);   // a wave's units are next to each other
    // unit of (block i, b, i): blocks of a wave's units are 32 (i WA + wa)
    const int cols = 32 * UB, ub = u0 + 32 * wa;
    const int have = K - ub < cols ? K - ub : cols;     // may be negative
    float db[2][UB][16], top = 0.0f;
    if constexpr (BACK) {
#pragma unroll
        for (int w = 0; w < 2; ++w)
#pragma unroll
            for (int i = 0; i < UB; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) db[w][i][e] = 0.0f;
    }
#pragma unroll
    for (int j = 0; j < S::BB; ++j) {
        const int64_t m = m0 + (wb * S::BB + j) * 32;
        const int left = (int)(g.M - m < 32 ? g.M - m : 32);
        if (left <= 0) continue;
        if constexpr (BACK && !kAhead) {
            rows.template move<false>((const T*)g.a.dy + m * K + ub, K, left, have, g.vec);
            wave_sync();
        }
        float og[UB][16], ou[UB][16];
#pragma unroll
        for (int i = 0; i < UB; ++i)
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const int c = 32 * i + 8 * b + 4 * h;
                const f32x4v bg = *(const f32x4v*)&bias[32 * wa + c], bu = *(const f32x4v*)&bias[kUnits + 32 * wa + c];
                float dy[4];
                if constexpr (kAhead) {
                    using D = typename DyTiles<T>::Tl;
                    T o[4];
                    __builtin_memcpy(o, __builtin_assume_aligned(dys[j] + D::at(wb * 32 + (lane & 31), c >> 3) + 8 * h, 8), 8);
#pragma unroll
                    for (int e = 0; e < 4; ++e) dy[e] = (float)o[e];
                } else if constexpr (BACK) {
                    rows.get4(c, dy);
                    // past the tokens LDS holds what was there
                    if (left < 32 && (lane & 31) >= left) dy[0] = dy[1] = dy[2] = dy[3] = 0.0f;
                }
                if constexpr (kHalf && !kAgain) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) dy[e] *= kFirstUp;
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float zg = acc[i][j][4 * b + e] + bg[e], zu = acc[UB + i][j][4 * b + e] + bu[e];
                    if constexpr (BACK) {
                        float v, d;
                        gate_slope(zg, g.act, v, d);
                        og[i][4 * b + e] = dy[e] * zu * d;
                        ou[i][4 * b + e] = dy[e] * v;
                        db[0][i][4 * b + e] += og[i][4 * b + e];
                        db[1][i][4 * b + e] += ou[i][4 * b + e];
                    } else {
                        og[i][4 * b + e] = gate(zg, g.act) * zu;
                    }
                }
            }
        if constexpr (kHalf && !kAgain) {
            float mx = 0.0f;
#pragma unroll
            for (int i = 0; i < UB; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) mx = fmaxf(mx, fmaxf(fabsf(og[i][e]), fabsf(ou[i][e])));
            // what is past the units is any value
            if (have < cols || __any(!(mx < INFINITY))) {
                mx = 0.0f;
#pragma unroll
                for (int i = 0; i < UB; ++i)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const float a = fabsf(og[i][e]), b = fabsf(ou[i][e]);
                        const bool in = 32 * i + 8 * (e >> 2) + 4 * h + (e & 3) < have;
                        if (in && a < INFINITY) mx = fmaxf(mx, a);
                        if (in && b < INFINITY) mx = fmaxf(mx, b);
                    }
            }
            top = fmaxf(top, mx);
        }
        auto out = [&](const float (&o)[UB][16], T* p, int64_t ld) {
            wave_sync();
            const float f = kAgain ? up : 1.0f;
#pragma unroll
            for (int i = 0; i < UB; ++i)
#pragma unroll
                for (int b = 0; b < 4; ++b)
                    rows.put4(32 * i + 8 * b + 4 * h, o[i][4 * b] * f, o[i][4 * b + 1] * f, o[i][4 * b + 2] * f,
                              o[i][4 * b + 3] * f);
            wave_sync();
            rows.template move<true>(p, ld, left, have, g.vec);
        };
        if constexpr (BACK) {
            T* dz = (T*)g.dz + m * 2 * K + ub;
            out(og, dz, 2 * (int64_t)K);
            out(ou, dz + K, 2 * (int64_t)K);
            wave_sync();
        } else {
            out(og, (T*)g.a.y + m * K + ub, K);
            wave_sync();
        }
    }
    if constexpr (BACK && !kAgain) {
        if (!kHalf && !g.a.dbias) return;
        // over the lanes, then over the waves that have these units
        __shared__ float sums[S::WB][2][kUnits], largest[4];
#pragma unroll
        for (int w = 0; w < 2; ++w)
#pragma unroll
            for (int i = 0; i < UB; ++i) {
                const float v = sum16(db[w][i]);
                // value 8 b4 + 4 b3 + 2 b2 + b1: row 8 (value / 4) + 4 h + value % 4 of the block
                const int val = (lane >> 4 & 1) * 8 + (lane >> 3 & 1) * 4 + (lane >> 2 & 1) * 2 + (lane >> 1 & 1);
                if (!(lane & 1)) sums[wb][w][32 * (i * S::WA + wa) + 8 * (val >> 2) + 4 * h + (val & 3)] = v;
            }
        if constexpr (kHalf) {
            top = join64<true>(top);
            if (lane == 0) largest[wave] = top;
        }
        __syncthreads();
        if (kHalf && threadIdx.x == 0) g.tops[item] = fmaxf(fmaxf(largest[0], largest[1]), fmaxf(largest[2], largest[3]));
        if (g.a.dbias && threadIdx.x < 2 * kUnits) {
            const int w = threadIdx.x / kUnits, u = threadIdx.x % kUnits;
            float v = 0.0f;
#pragma unroll
            for (int i = 0; i < S::WB; ++i) v += sums[i][w][u];
            if (u0 + u < K) g.dbias[(int64_t)mt * 2 * K + (int64_t)w * K + u0 + u] = kHalf ? v * (1.0f / kFirstUp) : v;
        }
    }
}

template <typename T, typename S, bool BACK, bool kDirect>
__global__ __launch_bounds__(256, 2) void k_gated(GatedK g) {
    const int item = item_of(g.items);
    if (item >= 0) gated_tile<T, S, BACK, kDirect, false>(g, item, kFirstUp);
}

// dz's power of two from its tiles' largest; dz again where it is not the first one.
template <typename S, bool kDirect>
__global__ __launch_bounds__(256, 2) void k_gated_again(GatedK g) {
    __shared__ float largest[4];
    float top = 0.0f;
    for (int i0 = threadIdx.x; i0 < g.items; i0 += 16 * 256) {
        float v[16];                                     // on their way together (12544 one by one took 20 us)
#pragma unroll
        for (int j = 0; j < 16; ++j) v[j] = i0 + 256 * j < g.items ? g.tops[i0 + 256 * j] : 0.0f;
#pragma unroll
        for (int j = 0; j < 16; ++j) top = fmaxf(top, v[j]);
    }
    top = join64<true>(top);
    if ((threadIdx.x & 63) == 0) largest[threadIdx.x >> 6] = top;
    __syncthreads();
    const float up = up_of(fmaxf(fmaxf(largest[0], largest[1]), fmaxf(largest[2], largest[3])));
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        g.ups[0] = up;
        g.ups[1] = 1.0f / up;
    }
    if (up == kFirstUp) return;                          // of every workgroup
    for (int item = blockIdx.x; item < g.items; item += gridDim.x) {
        gated_tile<_Float16, S, true, kDirect, true>(g, item, up);
        __syncthreads();                                 // the tile's LDS is free
    }
}

// A few tokens: a wave for each unit, its lanes along the channels, eight at a time.  All
// there is to do is to read the weights once (in tiles of 32 units 2048 of them are 64
// workgroups: one token of 512 channels 9.1 us).
constexpr int kFewTokens = 8;

template <typename T, int MT>
__global__ __launch_bounds__(256) void k_gated_few(GatedK g) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t u = (int64_t)blockIdx.x * 4 + wave;
    if (u >= g.K) return;
    const int C = g.C, M = (int)g.M;
    const T *w0 = (const T*)g.a.w + u * C, *w1 = w0 + (int64_t)g.K * C, *x = (const T*)g.a.x;
    float z[2][MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) z[0][m] = z[1][m] = 0.0f;
    for (int c = lane * 8; c < C; c += 512) {
        const Eight<T> a(w0 + c, 0, 0, C - c, g.vec), b(w1 + c, 0, 0, C - c, g.vec);
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const Eight<T> v(m < M ? x + (int64_t)m * C + c : nullptr, 0, 0, C - c, g.vec);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                z[0][m] = __builtin_fmaf((float)a.v[i], (float)v.v[i], z[0][m]);
                z[1][m] = __builtin_fmaf((float)b.v[i], (float)v.v[i], z[1][m]);
            }
        }
    }
    float zg = 0.0f, zu = 0.0f;              // of token `lane`
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const float a = join64(z[0][m]), b = join64(z[1][m]);
        if (lane == m) {
            zg = a;
            zu = b;
        }
    }
    if (lane >= M) return;
    if (g.a.bias) {
        zg += g.a.bias[u];
        zu += g.a.bias[g.K + u];
    }
    ((T*)g.a.y)[(int64_t)lane * g.K + u] = (T)(gate(zg, g.act) * zu);
}

// dz's power of two taken out of a product.
template <typename T, typename S>
__device__ __forceinline__ void take_down(f32x16 (&acc)[S::AB][S::BB], const float* ups) {
    if constexpr (std::is_same_v<T, _Float16>) {
        const float down = ups[1];
#pragma unroll
        for (int i = 0; i < S::AB; ++i)
#pragma unroll
            for (int j = 0; j < S::BB; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] *= down;
    }
}

// A tile's results to out[q][p], P of p: 64 columns of a wave at a time.
template <typename S, typename O>
__device__ __forceinline__ void put_tile(const f32x16 (&acc)[S::AB][S::BB], char* lds, O* out, int p0, int P, int64_t q0,
                                         int64_t Q, bool vec) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    const int wa = wave % S::WA, wb = wave / S::WA;
    const Rows64<O> rows{lds + wave * Rows64<O>::kBytes};
#pragma unroll
    for (int j = 0; j < S::BB; ++j) {
        const int64_t q = q0 + (wb * S::BB + j) * 32;
        const int left = (int)(Q - q < 32 ? Q - q : 32);
        if (left <= 0) continue;
        // with more waves than one a block's columns are not next to the next one's
        constexpr int each = S::WA == 1 && S::AB > 1 ? 2 : 1;
#pragma unroll
        for (int i = 0; i < S::AB; i += each) {
            const int p = p0 + 32 * (i * S::WA + wa);
            wave_sync();
#pragma unroll
            for (int e = 0; e < each; ++e)
#pragma unroll
                for (int b = 0; b < 4; ++b)
                    rows.put4(32 * e + 8 * b + 4 * h, acc[i + e][j][4 * b], acc[i + e][j][4 * b + 1],
                              acc[i + e][j][4 * b + 2], acc[i + e][j][4 * b + 3]);
            wave_sync();
            rows.template move<true>(out + q * P + p, P, left, P - p < 32 * each ? P - p : 32 * each, vec);
        }
    }
}

// dx of a tile's tokens and channels: dz [M][2 K] by w [2 K][C], over a part of the units.
template <typename T, typename S, bool kDirect>
__global__ __launch_bounds__(256, 2) void k_gated_dx(GatedK g) {
    using A = Side<T, S::kA, true, kDirect>;
    using B = Side<T, S::kB, false, kDirect>;
    __shared__ alignas(16) char lds[lds_of<S, A, B>(kDirect, Rows64<float>::kBytes)];
    const int item = item_of(g.items);
    if (item < 0) return;
    const int at = (uint32_t)item / (uint32_t)g.tiles, mt = (uint32_t)at / (uint32_t)g.splits;
    const int c0 = (item - at * g.tiles) * S::kA, F = 2 * g.K, split = at - mt * g.splits;
    const int64_t m0 = (int64_t)mt * S::kB;
    int64_t lo, hi;
    part_of(F, kBk, split, g.splits, lo, hi);
    f32x16 acc[S::AB][S::BB];
    A a;
    B b;
    a.init({(const T*)g.a.w + c0, F, g.C - c0, g.C, kBk, 0}, g.vec);
    b.init({(const T*)g.dz + m0 * F, g.M - m0 < S::kB ? g.M - m0 : S::kB, F, F, S::kB, 0}, g.vec);
    product<S>(acc, a, b, lds, lo, hi, kDirect);
    take_down<T, S>(acc, g.ups);
    if (g.splits > 1) put_tile<S>(acc, lds, g.part + (int64_t)split * g.M * g.C, c0, g.C, m0, g.M, (g.C & 3) == 0);
    else put_tile<S>(acc, lds, (T*)g.a.dx, c0, g.C, m0, g.M, g.vec);
}

// dw of a tile's units and channels, over a part of the tokens: dz^T by x.
template <typename T, typename S, bool kDirect>
__global__ __launch_bounds__(256, 2) void k_gated_dw(GatedK g) {
    using A = Side<T, S::kA, true, kDirect>;
    using B = Side<T, S::kB, true, kDirect>;
    __shared__ alignas(16) char lds[lds_of<S, A, B>(kDirect, Rows64<float>::kBytes)];
    const int item = item_of(g.items);
    if (item < 0) return;
    const int F = 2 * g.K;
    const int ft = (F + S::kB - 1) / S::kB, at = (uint32_t)item / (uint32_t)g.tiles, split = (uint32_t)at / (uint32_t)ft;
    const int c0 = (item - at * g.tiles) * S::kA, f0 = (at - split * ft) * S::kB;
    int64_t lo, hi;
    part_of(g.M, kBk, split, g.splits, lo, hi);
    f32x16 acc[S::AB][S::BB];
    A a;
    B b;
    a.init({(const T*)g.a.x + c0, g.M, g.C - c0, g.C, kBk, 0}, g.vec);
    b.init({(const T*)g.dz + f0, g.M, F - f0, F, kBk, 0}, g.vec);
    product<S>(acc, a, b, lds, lo, hi, kDirect);
    take_down<T, S>(acc, g.ups);
    if (g.splits > 1) put_tile<S>(acc, lds, g.part + (int64_t)split * F * g.C, c0, g.C, f0, F, (g.C & 3) == 0);
    else put_tile<S>(acc, lds, (T*)g.a.dw, c0, g.C, f0, F, g.vec);
}

// What a backward call's products left in parts, in one launch (three took 5 us each): dbias, a
// column's rows by 16 threads, then dx, then dw.
struct GatedEnd {
    const float *rows, *px, *pw;             // [tiles][F]; [x_splits][nx]; [w_splits][nw]
    float* dbias;
    void *dx, *dw;
    int64_t tiles, nx, nw;
    int F, x_splits, w_splits;
    unsigned db_blocks, dx_blocks;           // workgroups of the first two; 0: none to do
};
template <typename T>
__global__ __launch_bounds__(256) void k_gated_end(GatedEnd g) {
    __shared__ float s[16][17];
    if (blockIdx.x < g.db_blocks) {
        const int f = blockIdx.x * 16 + (threadIdx.x & 15), i0 = threadIdx.x >> 4;
        float sum = 0.0f;
        if (f < g.F)
#pragma unroll 8
            for (int64_t i = i0; i < g.tiles; i += 16) sum += g.rows[i * g.F + f];
        s[i0][threadIdx.x & 15] = sum;
        __syncthreads();
        if (threadIdx.x < 16 && f < g.F) {
            float all = 0.0f;
#pragma unroll
            for (int i = 0; i < 16; ++i) all += s[i][threadIdx.x];
            g.dbias[f] = all;
        }
        return;
    }
    const unsigned at = blockIdx.x - g.db_blocks;
    const bool x = at < g.dx_blocks;
    const int64_t i = (int64_t)(x ? at : at - g.dx_blocks) * 256 + threadIdx.x, n = x ? g.nx : g.nw;
    if (i >= n) return;
    const float* part = x ? g.px : g.pw;
    const int splits = x ? g.x_splits : g.w_splits;
    float sum = 0.0f;
#pragma unroll 8
    for (int k = 0; k < splits; ++k) sum += part[k * n + i];
    ((T*)(x ? g.dx : g.dw))[i] = (T)sum;
}

template <typename F>
hipError_t with_io(Io io, F f) {
    return io == Io::F32 ? f(float()) : io == Io::F16 ? f((_Float16)0) : f((__bf16)0.0f);
}

GatedK args_of(const GatedArgs& a, const GatedShape& s) {
    GatedK g{};
    g.a = a;
    g.M = s.M;
    g.C = s.C;
    g.K = s.K;
    g.act = s.act;
    const int z = io_size(s.io);
    g.vec = s.C * (int64_t)z % 16 == 0 && s.K * (int64_t)z % 16 == 0;
    for (const void* p : {a.dy, a.x, a.w, (const void*)a.y, (const void*)a.dx, (const void*)a.dw})
        g.vec = g.vec && aligned16(p);
    return g;
}


// A product's tile shape and the parts of its sum.
enum { kWide, kSquare, kNarrow, kSmall };
struct Cut {
    int shape, splits;
};
int64_t tiles_by(int shape, int64_t p, int64_t q) {
    return shape == kWide     ? tiles_of(p, Wide::kA) * tiles_of(q, Wide::kB)
           : shape == kSquare ? tiles_of(p, Square::kA) * tiles_of(q, Square::kB)
           : shape == kNarrow ? tiles_of(p, Narrow::kA) * tiles_of(q, Narrow::kB)
                              : tiles_of(p, Small::kA) * tiles_of(q, Small::kB);
}
// The cut of a product of p by q results of n terms, in `most` parts at most, that takes the
// least time by an estimate: the fullest CU's tiles at the rate that the shape reaches (of 16
// bits some 3.6 GFLOP a ms and CU with the wide one; 0.6 of a shape's where a CU has one
// workgroup), and the parts, 4 bytes a result, written and read again.  Measured against it, bf16:
// 6272 tokens of 512 channels by 2048 units, forward, wide 43.6 us, square 39.4, narrow 48.0 (four
// tiles a CU of 32768 results, seven of 16384); by 1024 units, backward, the last product wide in
// 16 parts 106 us, square in 8 98.6, narrow in 4 91.4.  fp32 operands of the wide shape pass a
// wave's registers.
Cut cut_of(int64_t p, int64_t q, int64_t n, int64_t most, Io io, bool pairs) {
    constexpr double kResults[] = {128 * 256, 128 * 128, 64 * 128, 64 * 64};
    constexpr double kRate16[] = {1.0, 0.9, 0.75, 0.5}, kRate32[] = {0.0, 0.2, 0.17, 0.12};
    const int64_t steps = tiles_of(n, kBk);
    most = most < 1 ? 1 : most > 64 ? 64 : most;
    Cut best{io == Io::F32 ? kSquare : kWide, 1};
    double least = 1e300;
    for (int shape = best.shape; shape <= (pairs ? kNarrow : kSmall); ++shape) {
        const int64_t tiles = tiles_by(shape, p, q);
        for (int k = 0; k <= 4; ++k) {                   // so many a CU
            const int64_t want = k * 256 / tiles, s = want < 1 ? 1 : want > most ? most : want;
            const int64_t full = tiles_of(tiles * s, 256);
            const double rate = 3.6e6 * (io == Io::F32 ? kRate32 : kRate16)[shape] * (full == 1 ? 0.6 : 1.0);
            const double us = full * kResults[shape] * tiles_of(steps, (int)s) * (2 * kBk) / rate +
                              (s > 1 ? 3.0 + s * (double)p * q * 8 / 5e6 : 0.0);
            if (us < least) {
                least = us;
                best = {shape, (int)s};
            }
        }
    }
    return best;
}

// f(type, shape, straight to LDS); kPairs: a unit's gate and value are to be in one wave
template <bool kPairs, typename F>
hipError_t with_all(const GatedK& g, Io io, int shape, F f) {
    // offsets of a tile's rows, and from a unit's gate to its value, below 2^31
    const bool direct = g.vec && g.C <= 1 << 20 && g.K <= 1 << 19 && (int64_t)g.K * g.C < 1 << 27;
    return with_io(io, [&](auto t) {
        auto shaped = [&](auto d) {
            if constexpr (sizeof(t) == 2)
                if (shape == kWide) return f(t, Wide(), d);
            if (shape == kSquare) return f(t, Square(), d);
            if constexpr (!kPairs)
                if (shape == kSmall) return f(t, Small(), d);
            return f(t, Narrow(), d);
        };
        return direct ? shaped(std::true_type()) : shaped(std::false_type());
    });
}

}  // namespace

int gated_results(int shape) {
    return shape == kWide     ? Wide::kA * Wide::kB
           : shape == kSquare ? Square::kA * Square::kB
           : shape == kNarrow ? Narrow::kA * Narrow::kB
                              : Small::kA * Small::kB;
}
bool gated_few(const GatedShape& s) { return s.M <= kFewTokens; }

GatedPlan gated_plan(const GatedShape& s, bool backward) {
    GatedPlan p{};
    const int64_t F = 2 * (int64_t)s.K;
    // a launch has fewer than 2^32 threads, 256 a workgroup; grids are rounded up to eight
    auto fits = [](int64_t items) { return items <= ((int64_t)1 << 24) - 8; };
    p.fits = s.M <= INT32_MAX && s.K <= INT32_MAX / 2 && (int64_t)s.K * s.C < (int64_t)1 << 37;
    if (!p.fits) return p;
    p.first = cut_of(F, s.M, s.C, 1, s.io, true).shape;
    p.fits = !backward && gated_few(s) ? fits(tiles_of(s.K, 4)) : fits(tiles_by(p.first, F, s.M));
    if (!p.fits || !backward) return p;
    // parts of 256 units or tokens at least
    const Cut x = cut_of(s.C, s.M, F, F / 256, s.io, false), w = cut_of(s.C, F, s.M, s.M / 256, s.io, false);
    p.dx = x.shape; p.dx_splits = x.splits;
    p.dw = w.shape; p.dw_splits = w.splits;
    // the last launch: dbias's columns, and sums of at most 512 tiles of 128 by 256 for each product
    p.fits = fits(tiles_by(p.dx, s.C, s.M) * p.dx_splits) && fits(tiles_by(p.dw, s.C, F) * p.dw_splits) &&
             fits(tiles_of(F, 16) + 2 * 512 * (128 * 256 / 256));
    if (!p.fits) return p;
    p.dz = round_up((size_t)s.M * F * io_size(s.io), 16);
    p.dbias = round_up((size_t)tiles_of(s.M, Narrow::kB) * F * 4, 16);
    p.px = p.dx_splits > 1 ? round_up((size_t)p.dx_splits * s.M * s.C * 4, 16) : 0;
    p.pw = p.dw_splits > 1 ? round_up((size_t)p.dw_splits * F * s.C * 4, 16) : 0;
    p.tops = s.io == Io::F16 ? round_up((size_t)tiles_by(p.first, F, s.M) * 4, 16) + 16 : 0;
    p.need = p.dz + p.dbias + p.px + p.pw + p.tops;
    return p;
}

hipError_t launch_gated(const GatedArgs& a, const GatedShape& s, const GatedPlan& p, hipStream_t st) {
    GatedK g = args_of(a, s);
    if (gated_few(s))
        return with_io(s.io, [&](auto t) {
            typedef decltype(t) T;
            const unsigned blocks = (unsigned)tiles_of(s.K, 4);
            if (s.M == 1) k_gated_few<T, 1><<<blocks, 256, 0, st>>>(g);
            else if (s.M == 2) k_gated_few<T, 2><<<blocks, 256, 0, st>>>(g);
            else if (s.M <= 4) k_gated_few<T, 4><<<blocks, 256, 0, st>>>(g);
            else k_gated_few<T, 8><<<blocks, 256, 0, st>>>(g);
            return hipGetLastError();
        });
    return with_all<true>(g, s.io, p.first, [&](auto t, auto sh, auto direct) {
        typedef decltype(sh) S;
        g.tiles = (int)tiles_of(s.K, S::kA / 2);
        g.items = (int)(tiles_of(s.M, S::kB) * g.tiles);
        k_gated<decltype(t), S, false, direct.value><<<grid_of(g.items), 256, 0, st>>>(g);
        return hipGetLastError();
    });
}

hipError_t launch_gated_backward(const GatedArgs& a, const GatedShape& s, const GatedPlan& p, void* ws, hipStream_t st) {
    GatedK g = args_of(a, s);
    const int64_t F = 2 * (int64_t)s.K;
    g.dz = ws;
    g.dbias = (float*)((char*)ws + p.dz);
    char* parts = (char*)ws + p.dz + p.dbias;
    g.ups = (float*)(parts + p.px + p.pw);
    g.tops = g.ups + 4;
    GatedEnd end{};
    end.F = (int)F;
    hipError_t e = with_all<true>(g, s.io, p.first, [&](auto t, auto sh, auto direct) {
        typedef decltype(sh) S;
        g.tiles = (int)tiles_of(s.K, S::kA / 2);
        end.tiles = tiles_of(s.M, S::kB);
        g.items = (int)(end.tiles * g.tiles);
        k_gated<decltype(t), S, true, direct.value><<<grid_of(g.items), 256, 0, st>>>(g);
        if constexpr (std::is_same_v<decltype(t), _Float16>) {
            const hipError_t first = hipGetLastError();
            if (first != hipSuccess) return first;
            k_gated_again<S, direct.value><<<g.items < 512 ? g.items : 512, 256, 0, st>>>(g);
        }
        return hipGetLastError();
    });
    if (e != hipSuccess) return e;
    if (a.dbias) {
        end.rows = g.dbias;
        end.dbias = a.dbias;
        end.db_blocks = (unsigned)tiles_of(F, 16);
    }
    if (a.dx) {
        g.part = (float*)parts;
        g.splits = p.dx_splits;
        if (g.splits > 1) {
            end.px = g.part;
            end.dx = a.dx;
            end.nx = s.M * s.C;
            end.x_splits = g.splits;
            end.dx_blocks = (unsigned)tiles_of(end.nx, 256);
        }
        e = with_all<false>(g, s.io, p.dx, [&](auto t, auto sh, auto direct) {
            typedef decltype(sh) S;
            g.tiles = (int)tiles_of(s.C, S::kA);
            g.items = (int)(tiles_of(s.M, S::kB) * g.tiles * g.splits);
            k_gated_dx<decltype(t), S, direct.value><<<grid_of(g.items), 256, 0, st>>>(g);
            return hipGetLastError();
        });
        if (e != hipSuccess) return e;
    }
    unsigned dw_blocks = 0;
    if (a.dw) {
        g.part = (float*)(parts + p.px);
        g.splits = p.dw_splits;
        if (g.splits > 1) {
            end.pw = g.part;
            end.dw = a.dw;
            end.nw = F * s.C;
            end.w_splits = g.splits;
            dw_blocks = (unsigned)tiles_of(end.nw, 256);
        }
        e = with_all<false>(g, s.io, p.dw, [&](auto t, auto sh, auto direct) {
            typedef decltype(sh) S;
            g.tiles = (int)tiles_of(s.C, S::kA);
            g.items = (int)(g.tiles * tiles_of(F, S::kB) * g.splits);
            k_gated_dw<decltype(t), S, direct.value><<<grid_of(g.items), 256, 0, st>>>(g);
            return hipGetLastError();
        });
        if (e != hipSuccess) return e;
    }
    const unsigned blocks = end.db_blocks + end.dx_blocks + dw_blocks;
    if (!blocks) return hipSuccess;
    return with_io(s.io, [&](auto t) {
        k_gated_end<decltype(t)><<<blocks, 256, 0, st>>>(end);
        return hipGetLastError();
    });
}

}  // namespace wino
