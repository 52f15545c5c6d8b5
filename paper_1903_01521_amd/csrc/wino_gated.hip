// The gated layer of channel-last tensors, y = act(zg) * zu with zg = x w0^T + b0 and
// zu = x w1^T + b1, and its backward pass
//   dzg = dy zu act'(zg), dzu = dy act(zg), dx = dzg w0 + dzu w1, dw = dz^T x, db = sum dz.
//
// Matrix products on 32x32 matrix-core tiles, their operands staged through LDS.  A
// workgroup of four waves has 128 x 128 results: the left operand's index runs down a
// lane's registers and is the output's contiguous one, the right operand's runs over the
// lanes.  Forward, a workgroup's 128 left rows are 64 units' gates and their values, so
// that both of a unit meet in one lane and neither leaves it.  Backward is three products:
// zg and zu once more, ending in dz (kept in the tensors' type, as any gradient between two
// layers), then dx from dz and w, and dw from dz and x, the sum over tokens in parts.
#include "wino_attn_device.h"
#include "wino_checks.h"
#include "wino_gated.h"
#include "wino_norm_device.h"

namespace wino {

namespace {

constexpr int kTile = 128, kUnits = 64;

struct GatedK {
    GatedArgs a;
    int64_t M;
    int C, K;
    Act act;
    bool vec;
    void* dz;                                // [M][2 K]
    float *dbias, *part;                     // [token tiles][2 K]; [splits][2 K][C]
    int64_t items, tiles;                    // tiles: of the faster axis
    int splits;
};

// One operand of a product: a tile of 128 indices by BK terms of the sum.  T_: its memory
// is [sum][index], else [index][sum].
template <typename T, bool T_>
struct Side {
    static constexpr int kBk = sizeof(T) == 4 ? 32 : 64;
    static constexpr int kRows = T_ ? kBk : kTile;
    static constexpr int kD16 = T_ ? kTile / 16 : kBk / 16;
    using Tl = Tile<T, kD16, kRows>;
    static constexpr int kBytes = Tl::kBytes;
    // terms 16 c .. of indices 32 blk ..
    __device__ static __forceinline__ Frag<T> read(const char* t, int blk, int c, int lane) {
        if constexpr (T_) return Tl::turned8(t, 16 * c, blk, lane);
        else return Tl::read(t, 32 * blk + (lane & 31), c, lane >> 5);
    }
};

// acc[i][j] = products of left block a0 + i * da and right block b0 + j, over the terms
// lo .. hi.  left(r, k), right(r, k): the memory row r of a tile at term k, or null; the
// values that a row holds from there on are limit_left(k), limit_right(k).
template <typename T, bool AT, bool BT, typename L, typename R, typename LL, typename LR>
__device__ __forceinline__ void product(f32x16 (&acc)[2][2], char* sa, char* sb, int64_t lo, int64_t hi, int a0, int da,
                                        int b0, bool vec, L left, R right, LL limit_left, LR limit_right) {
    using A = Side<T, AT>;
    using B = Side<T, BT>;
    constexpr int BK = A::kBk;
    const int lane = threadIdx.x & 63;
    Moving<T, A::kD16, A::kRows, 256> ma;
    Moving<T, B::kD16, B::kRows, 256> mb;
    auto load = [&](int64_t k) {
        ma.load([&](int r) { return left(r, k); }, limit_left(k), vec);
        mb.load([&](int r) { return right(r, k); }, limit_right(k), vec);
    };
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = f32x16{};
    if (lo < hi) load(lo);
    for (int64_t k = lo; k < hi; k += BK) {
        __syncthreads();
        ma.store(sa);
        mb.store(sb);
        __syncthreads();
        if (k + BK < hi) load(k + BK);
#pragma unroll
        for (int c = 0; c < BK / 16; ++c) {
            Frag<T> a[2], b[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                a[i] = A::read(sa, a0 + i * da, c, lane);
                b[i] = B::read(sb, b0 + i, c, lane);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[i][j] = mma(a[i], b[j], acc[i][j]);
        }
    }
}

// Workgroups that share a tile's tokens follow each other on one XCD, whose L2 then holds
// them: workgroup ids go round the eight XCDs.  Item of `all`, or -1.
__device__ __forceinline__ int64_t item_of(int64_t all) {
    const int64_t each = (all + 7) / 8, i = (int64_t)(blockIdx.x & 7) * each + (blockIdx.x >> 3);
    return (blockIdx.x >> 3) < each && i < all ? i : -1;
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

// Four neighbouring values at p + d, those from D on zero.
template <typename T>
__device__ __forceinline__ void load4(const T* p, int d, int D, bool vec, float (&v)[4]) {
    if (vec) {
        const Raw<T, 4> r = d < D ? *(const Raw<T, 4>*)(p + d) : Raw<T, 4>{};
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = (float)r.v[i];
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = d + i < D ? (float)p[d + i] : 0.0f;
}

// y of 128 tokens by 64 units, or dz of them and the tile's sums of it.
template <typename T, bool BACK>
__global__ __launch_bounds__(256) void k_gated(GatedK g) {
    using S = Side<T, false>;
    __shared__ alignas(16) char sa[S::kBytes];
    __shared__ alignas(16) char sb[S::kBytes];
    const int64_t item = item_of(g.items);
    if (item < 0) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5;
    const int64_t mt = item / g.tiles, m0 = mt * kTile;
    const int u0 = (int)(item % g.tiles) * kUnits;
    const T *x = (const T*)g.a.x, *w = (const T*)g.a.w;
    f32x16 acc[2][2];                                    // gates and values by two blocks of 32 tokens
    product<T, false, false>(
        acc, sa, sb, 0, g.C, wave & 1, 2, wave >> 1 << 1, g.vec,
        [&](int r, int64_t k) {
            const int u = u0 + (r & (kUnits - 1));
            return u < g.K ? w + ((int64_t)(r / kUnits) * g.K + u) * g.C + k : nullptr;
        },
        [&](int r, int64_t k) { return m0 + r < g.M ? x + (m0 + r) * g.C + k : nullptr; },
        [&](int64_t k) { return g.C - (int)k; }, [&](int64_t k) { return g.C - (int)k; });
    const int ub = u0 + 32 * (wave & 1) + 4 * h;
    float db[2][16];
    if constexpr (BACK) {
#pragma unroll
        for (int i = 0; i < 16; ++i) db[0][i] = db[1][i] = 0.0f;
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int64_t m = m0 + ((wave >> 1) * 2 + j) * 32 + (lane & 31);
        if (m >= g.M) continue;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int u = ub + 8 * b;
            float bg[4] = {0, 0, 0, 0}, bu[4] = {0, 0, 0, 0}, og[4], ou[4], dy[4];
            if (g.a.bias) {
                load4(g.a.bias, u, g.K, false, bg);
                load4(g.a.bias + g.K, u, g.K, false, bu);
            }
            if constexpr (BACK) load4((const T*)g.a.dy + m * g.K, u, g.K, g.vec, dy);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float zg = acc[0][j][4 * b + i] + bg[i], zu = acc[1][j][4 * b + i] + bu[i];
                if constexpr (BACK) {
                    float v, d;
                    gate_slope(zg, g.act, v, d);
                    og[i] = dy[i] * zu * d;
                    ou[i] = dy[i] * v;
                    db[0][4 * b + i] += og[i];
                    db[1][4 * b + i] += ou[i];
                } else {
                    og[i] = gate(zg, g.act) * zu;
                }
            }
            if constexpr (BACK) {
                T* dz = (T*)g.dz + m * 2 * g.K;
                store4(dz, u, g.K, g.vec, og[0], og[1], og[2], og[3]);
                store4(dz + g.K, u, g.K, g.vec, ou[0], ou[1], ou[2], ou[3]);
            } else {
                store4((T*)g.a.y + m * g.K, u, g.K, g.vec, og[0], og[1], og[2], og[3]);
            }
        }
    }
    if constexpr (BACK) {
        if (!g.a.dbias) return;
        // over the 32 lanes of a half, then over the two waves that have these units
        __shared__ float rows[4][2][2][16];
#pragma unroll
        for (int w2 = 0; w2 < 2; ++w2)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                float v = db[w2][i];
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) v += __shfl_xor(v, d, 64);
                if ((lane & 31) == 0) rows[wave][w2][h][i] = v;
            }
        __syncthreads();
        if (threadIdx.x < 2 * kUnits) {
            // value w2, unit 32 wu + 8 b + 4 h + i
            const int w2 = threadIdx.x >> 6, u = threadIdx.x & 63, wu = u >> 5, hh = (u >> 2) & 1;
            const int i = ((u & 31) >> 3) * 4 + (u & 3);
            if (u0 + u < g.K)
                g.dbias[mt * 2 * g.K + (int64_t)w2 * g.K + u0 + u] = rows[wu][w2][hh][i] + rows[wu + 2][w2][hh][i];
        }
    }
}

// Results 32 (wa blocks) of P down, lanes 32 (wb blocks) of Q across, to out[q][p].
template <typename T, typename O>
__device__ __forceinline__ void put_tile(const f32x16 (&acc)[2][2], O* out, int p0, int P, int64_t q0, int64_t Q, bool vec) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int64_t q = q0 + ((wave >> 1) * 2 + j) * 32 + (lane & 31);
        if (q >= Q) continue;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int b = 0; b < 4; ++b)
                store4(out + q * P, p0 + ((wave & 1) * 2 + i) * 32 + 8 * b + 4 * h, P, vec, acc[i][j][4 * b],
                       acc[i][j][4 * b + 1], acc[i][j][4 * b + 2], acc[i][j][4 * b + 3]);
    }
}

// dx of 128 tokens by 128 channels: dz [M][2 K] by w [2 K][C].
template <typename T>
__global__ __launch_bounds__(256) void k_gated_dx(GatedK g) {
    __shared__ alignas(16) char sa[Side<T, true>::kBytes];
    __shared__ alignas(16) char sb[Side<T, false>::kBytes];
    const int64_t item = item_of(g.items);
    if (item < 0) return;
    const int wave = threadIdx.x >> 6;
    const int64_t m0 = item / g.tiles * kTile;
    const int c0 = (int)(item % g.tiles) * kTile, F = 2 * g.K;
    const T *dz = (const T*)g.dz, *w = (const T*)g.a.w;
    f32x16 acc[2][2];
    product<T, true, false>(
        acc, sa, sb, 0, F, (wave & 1) * 2, 1, (wave >> 1) * 2, g.vec,
        [&](int r, int64_t k) { return k + r < F ? w + (k + r) * g.C + c0 : nullptr; },
        [&](int r, int64_t k) { return m0 + r < g.M ? dz + (m0 + r) * F + k : nullptr; },
        [&](int64_t) { return g.C - c0; }, [&](int64_t k) { return F - (int)k; });
    put_tile<T>(acc, (T*)g.a.dx, c0, g.C, m0, g.M, g.vec);
}

// dw of 128 units by 128 channels, over a part of the tokens: dz^T by x.
template <typename T>
__global__ __launch_bounds__(256) void k_gated_dw(GatedK g) {
    using S = Side<T, true>;
    __shared__ alignas(16) char sa[S::kBytes];
    __shared__ alignas(16) char sb[S::kBytes];
    const int64_t item = item_of(g.items);
    if (item < 0) return;
    const int wave = threadIdx.x >> 6, F = 2 * g.K;
    const int64_t ft = (F + kTile - 1) / kTile;
    const int c0 = (int)(item % g.tiles) * kTile, f0 = (int)(item / g.tiles % ft) * kTile;
    const int split = (int)(item / g.tiles / ft);
    const T *dz = (const T*)g.dz, *x = (const T*)g.a.x;
    int64_t lo, hi;
    part_of(g.M, S::kBk, split, g.splits, lo, hi);
    f32x16 acc[2][2];
    product<T, true, true>(
        acc, sa, sb, lo, hi, (wave & 1) * 2, 1, (wave >> 1) * 2, g.vec,
        [&](int r, int64_t k) { return k + r < hi ? x + (k + r) * g.C + c0 : nullptr; },
        [&](int r, int64_t k) { return k + r < hi ? dz + (k + r) * F + f0 : nullptr; },
        [&](int64_t) { return g.C - c0; }, [&](int64_t) { return F - f0; });
    if (g.splits > 1)
        put_tile<T>(acc, g.part + (int64_t)split * F * g.C, c0, g.C, f0, F, (g.C & 3) == 0);
    else
        put_tile<T>(acc, (T*)g.a.dw, c0, g.C, f0, F, g.vec);
}

template <typename T>
__global__ __launch_bounds__(256) void k_gated_dw_sum(GatedK g) {
    const int64_t all = (int64_t)2 * g.K * g.C, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= all) return;
    float sum = 0.0f;
    for (int k = 0; k < g.splits; ++k) sum += g.part[k * all + i];
    ((T*)g.a.dw)[i] = (T)sum;
}

// dbias: 16 columns a workgroup, 16 threads a column.
__global__ __launch_bounds__(256) void k_gated_db(GatedK g) {
    const int F = 2 * g.K, f = blockIdx.x * 16 + (threadIdx.x & 15), i0 = threadIdx.x >> 4;
    const int64_t rows = (g.M + kTile - 1) / kTile;
    float sum = 0.0f;
    if (f < F)
        for (int64_t i = i0; i < rows; i += 16) sum += g.dbias[i * F + f];
    __shared__ float s[16][17];
    s[i0][threadIdx.x & 15] = sum;
    __syncthreads();
    if (threadIdx.x < 16 && f < F) {
        float all = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) all += s[i][threadIdx.x];
        g.a.dbias[f] = all;
    }
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

inline int64_t tiles_of(int64_t n, int each) { return (n + each - 1) / each; }

}  // namespace

GatedPlan gated_plan(const GatedShape& s, bool backward) {
    GatedPlan p{};
    const int64_t mt = tiles_of(s.M, kTile), ut = tiles_of(s.K, kUnits), ct = tiles_of(s.C, kTile);
    const int64_t ft = tiles_of(2 * (int64_t)s.K, kTile), most = (int64_t)1 << 30;
    // 512 workgroups fill the card; a part has 256 tokens at least
    const int64_t want = (512 + ct * ft - 1) / (ct * ft), few = s.M / 256;
    p.splits = (int)(want < few ? want : few);
    if (p.splits < 1) p.splits = 1;
    if (p.splits > 64) p.splits = 64;
    p.fits = s.M <= INT32_MAX && s.K <= INT32_MAX / 2 && mt * ut <= most && mt * ct <= most && ct * ft * p.splits <= most &&
             (int64_t)s.K * s.C <= INT32_MAX * (int64_t)64;
    if (!p.fits || !backward) return p;
    p.dz = round_up((size_t)s.M * 2 * s.K * io_size(s.io), 16);
    p.dbias = round_up((size_t)mt * 2 * s.K * 4, 16);
    p.part = p.splits > 1 ? round_up((size_t)p.splits * 2 * s.K * s.C * 4, 16) : 0;
    p.need = p.dz + p.dbias + p.part;
    return p;
}

hipError_t launch_gated(const GatedArgs& a, const GatedShape& s, const GatedPlan& p, hipStream_t st) {
    GatedK g = args_of(a, s);
    g.tiles = tiles_of(s.K, kUnits);
    g.items = tiles_of(s.M, kTile) * g.tiles;
    return with_io(s.io, [&](auto t) {
        k_gated<decltype(t), false><<<grid_of(g.items), 256, 0, st>>>(g);
        return hipGetLastError();
    });
}

hipError_t launch_gated_backward(const GatedArgs& a, const GatedShape& s, const GatedPlan& p, void* ws, hipStream_t st) {
    GatedK g = args_of(a, s);
    g.dz = ws;
    g.dbias = (float*)((char*)ws + p.dz);
    g.part = (float*)((char*)ws + p.dz + p.dbias);
    return with_io(s.io, [&](auto t) {
        typedef decltype(t) T;
        g.tiles = tiles_of(s.K, kUnits);
        g.items = tiles_of(s.M, kTile) * g.tiles;
        k_gated<T, true><<<grid_of(g.items), 256, 0, st>>>(g);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        if (a.dbias) {
            k_gated_db<<<(unsigned)tiles_of(2 * (int64_t)s.K, 16), 256, 0, st>>>(g);
            if ((e = hipGetLastError()) != hipSuccess) return e;
        }
        g.tiles = tiles_of(s.C, kTile);
        if (a.dx) {
            g.items = tiles_of(s.M, kTile) * g.tiles;
            k_gated_dx<T><<<grid_of(g.items), 256, 0, st>>>(g);
            if ((e = hipGetLastError()) != hipSuccess) return e;
        }
        if (a.dw) {
            g.splits = p.splits;
            g.items = g.tiles * tiles_of(2 * (int64_t)s.K, kTile) * g.splits;
            k_gated_dw<T><<<grid_of(g.items), 256, 0, st>>>(g);
            if ((e = hipGetLastError()) != hipSuccess) return e;
            if (g.splits > 1)
                k_gated_dw_sum<T><<<(unsigned)tiles_of((int64_t)2 * s.K * s.C, 256), 256, 0, st>>>(g);
        }
        return hipGetLastError();
    });
}

}  // namespace wino
