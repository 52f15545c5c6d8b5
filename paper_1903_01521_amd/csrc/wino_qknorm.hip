// Norm of each head of queries and keys with the position rotation.
//
// A head's vector x of D channels: r = 1 / sqrt(mean x^2 + eps), n = x r, z = n gamma,
// and pairs (a, b) of the first R channels turned to (a c - b s, b c + a s) by the row
// of the table at the token's position.  Backward: dz = dy turned back, dgamma = sum dz n,
// and with dn = dz gamma, dx = r (dn - n mean(dn n)).
//
// Both are bound by memory: each value is read once and written once (64 images of 3136 tokens,
// 8 heads of 64, bf16: 96 us, 4.3 TB/s; backward, fp32, 382 MB: 77 us, 5.0).  A lane has `VP`
// whole pairs of a vector, two loads of VP values (its parts of the two halves, or
// neighbours), so that a rotation stays inside it, and keeps the cosines, sines and
// gammas of its pairs for the heads of a token that it does in turn.  A vector's sum of
// squares is one over 2 to 64 lanes.
#include "wino_checks.h"
#include "wino_fastdiv.h"
#include "wino_norm_device.h"
#include "wino_qknorm.h"

namespace wino {

namespace {

constexpr int kHeads = 4;                    // heads of a token that a team does in turn
constexpr int kBackBlocks = 2048;            // workgroups of a backward launch, each a row of dgamma's parts

struct QkK {
    QkShape s;
    QkSide t[2];
    int blocks0;                             // workgroups of the first tensor
    int64_t items[2];
    int chunks[2];                           // of a token's heads
    FastDiv by_chunk[2], by_len[2];
    int lanes;                               // of a team that have pairs
    float* part;                             // [workgroups][D]
};

template <int TEAM>
__device__ __forceinline__ float team_sum(float x) {
#pragma unroll
    for (int d = 1; d < TEAM; d <<= 1) x += __shfl_xor(x, d, 64);
    return x;
}

template <int TEAM>
__device__ __forceinline__ float team_max(float x) {
#pragma unroll
    for (int d = 1; d < TEAM; d <<= 1) x = fmaxf(x, __shfl_xor(x, d, 64));
    return x;
}

// 1 / sqrt(mean x^2 + eps) from the sum of squares.  Where that is out of range (past 2^100, or so small
// that squares may have lost bits; fp16's are in it), of a vector of the wave, x is taken times a power
// of two, `up`, which the result belongs to, and `again` sums anew: n = x r is as before, and r of the
// vector as it was is r up.
template <typename T, int TEAM, int N, typename F>
__device__ __forceinline__ float unit(float (&x)[N], float sq, int D, float eps, float& up, const F& again) {
    up = 1.0f;
    float mean = sq / (float)D + eps;
    if constexpr (sizeof(T) == 4 || std::is_same_v<T, __bf16>) {
        const bool out = !(mean >= 0x1p-80f && mean <= 0x1p100f);
        if (__any(out)) {
            float top = 0.0f;
#pragma unroll
            for (int j = 0; j < N; ++j) top = fmaxf(top, fabsf(x[j]));
            top = fmaxf(team_max<TEAM>(top), sqrtf(eps));
            if (out && top > 0.0f && top < INFINITY) {
                const int e = (int)(__float_as_uint(top) >> 23) - 127;
                up = __uint_as_float((uint32_t)(min(max(-e, -126), 126) + 127) << 23);
            }
#pragma unroll
            for (int j = 0; j < N; ++j) x[j] *= up;
            mean = again() / (float)D + eps * up * up;
        }
    }
    return 1.0f / sqrtf(mean);
}

// VP values at p + d as floats; those from D on are zero.
template <typename T, int VP>
__device__ __forceinline__ void get(const T* p, int d, int D, float* v) {
    if constexpr (VP == 1) {
        v[0] = d < D ? (float)p[d] : 0.0f;
    } else {
        T r[VP];
        __builtin_memcpy(r, p + d, sizeof(r));           // one load, on any address
#pragma unroll
        for (int i = 0; i < VP; ++i) v[i] = (float)r[i];
    }
}
template <typename T, int VP>
__device__ __forceinline__ void set(T* p, int d, int D, const float* v) {
    if constexpr (VP == 1) {
        if (d < D) p[d] = (T)v[0];
    } else {
        T r[VP];
#pragma unroll
        for (int i = 0; i < VP; ++i) r[i] = (T)v[i];
        __builtin_memcpy(p + d, r, sizeof(r));
    }
}

// What a lane has of every vector: values at d0 and d1, VP each; pair i is (i, VP + i),
// or (2 i, 2 i + 1).
template <int VP, bool PAIRS>
struct Mine {
    int d0, d1;
    bool on, turned;                         // its pairs turn: all of them, or none
    float g[2 * VP], c[VP], s[VP];
    __device__ __forceinline__ void place(const QkShape& k, int lane, int lanes, const float* gamma) {
        on = lane < lanes;
        const int p = lane * VP;
        turned = p < k.R / 2;
        if (!PAIRS && turned) {
            d0 = p;
            d1 = k.R / 2 + p;
        } else {
            d0 = 2 * p;
            d1 = 2 * p + VP;
        }
#pragma unroll
        for (int i = 0; i < VP; ++i) {
            g[i] = !gamma || !on ? 1.0f : d0 + i < k.D ? gamma[d0 + i] : 0.0f;
            g[VP + i] = !gamma || !on ? 1.0f : d1 + i < k.D ? gamma[d1 + i] : 0.0f;
            c[i] = 1.0f;
            s[i] = 0.0f;
        }
    }
    // Cosines and sines at position `at`; a position outside the table turns to NaN.
    __device__ __forceinline__ void turn(const QkShape& k, int lane, int64_t at) {
        const int p = lane * VP;
        if (!on || !turned) return;
        const bool in = at >= 0 && at < k.T;
        const float* row = k.rot + (in ? at : 0) * k.R + 2 * p;
#pragma unroll
        for (int i = 0; i < VP; ++i) {
            c[i] = in ? row[2 * i] : NAN;
            s[i] = in ? row[2 * i + 1] : NAN;
        }
    }
    // (za, zb) turned by pair i's angle, or back (s negative); channels from R on stay apart, as 0 times
    // what is not finite is NaN
    __device__ __forceinline__ void turn_pair(float za, float zb, float c, float s, float& a, float& b) const {
        a = turned ? za * c - zb * s : za;
        b = turned ? zb * c + za * s : zb;
    }
    __device__ __forceinline__ static int first(int i) { return PAIRS ? 2 * i : i; }
    __device__ __forceinline__ static int second(int i) { return PAIRS ? 2 * i + 1 : VP + i; }
    template <typename T>
    __device__ __forceinline__ void load(const T* p, int D, float (&v)[2 * VP]) const {
#pragma unroll
        for (int i = 0; i < 2 * VP; ++i) v[i] = 0.0f;
        if (!on) return;
        get<T, VP>(p, d0, D, v);
        get<T, VP>(p, d1, D, v + VP);
    }
    template <typename T>
    __device__ __forceinline__ void store(T* p, int D, const float (&v)[2 * VP]) const {
        if (!on) return;
        set<T, VP>(p, d0, D, v);
        set<T, VP>(p, d1, D, v + VP);
    }
};

// Item of tensor w: token (n, t) and a run of its heads.
struct QkItem {
    int64_t tok, at;
    int h0, h1;
};
__device__ __forceinline__ QkItem qk_item(const QkK& g, int w, int64_t item) {
    const QkSide& t = g.t[w];
    const uint32_t tok = fdiv((uint32_t)item, g.by_chunk[w]);
    const int h0 = ((int)item - (int)tok * g.chunks[w]) * kHeads;
    const int64_t at = t.pos ? t.pos[tok] : (int64_t)(tok - fdiv(tok, g.by_len[w]) * (uint32_t)t.L);
    return {tok, at, h0, min(h0 + kHeads, t.heads)};
}

template <typename T, int VP, int TEAM, bool PAIRS>
__global__ __launch_bounds__(256) void k_qk_norm(QkK g) {
    const int w = blockIdx.x < g.blocks0 ? 0 : 1;
    const QkSide& t = g.t[w];
    const int lane = threadIdx.x & (TEAM - 1);
    const int64_t item = (int64_t)(blockIdx.x - (w ? g.blocks0 : 0)) * (256 / TEAM) + threadIdx.x / TEAM;
    if (item >= g.items[w]) return;                  // whole teams
    const QkItem me = qk_item(g, w, item);
    const int D = g.s.D;
    Mine<VP, PAIRS> m;
    m.place(g.s, lane, g.lanes, t.gamma);
    float v[kHeads][2 * VP];
#pragma unroll
    for (int i = 0; i < kHeads; ++i)
        if (me.h0 + i < me.h1) m.load((const T*)t.x + me.tok * t.ld + (int64_t)(me.h0 + i) * D, D, v[i]);
    m.turn(g.s, lane, me.at);
#pragma unroll
    for (int i = 0; i < kHeads; ++i) {
        if (me.h0 + i >= me.h1) break;
        auto squares = [&] {
            float sq = 0.0f;
#pragma unroll
            for (int j = 0; j < 2 * VP; ++j) sq = __builtin_fmaf(v[i][j], v[i][j], sq);
            return team_sum<TEAM>(sq);
        };
        float up;
        const float r = unit<T, TEAM>(v[i], squares(), D, g.s.eps, up, squares);
#pragma unroll
        for (int j = 0; j < VP; ++j) {
            const int a = m.first(j), b = m.second(j);
            const float za = v[i][a] * r * m.g[a], zb = v[i][b] * r * m.g[b];
            m.turn_pair(za, zb, m.c[j], m.s[j], v[i][a], v[i][b]);
        }
        m.store((T*)t.y + (me.tok * t.heads + me.h0 + i) * D, D, v[i]);
    }
}

// A team walks items of one tensor and keeps its channels' sums of dgamma, which the
// workgroup's teams join in a fixed order.
template <typename T, int VP, int TEAM, bool PAIRS>
__global__ __launch_bounds__(256) void k_qk_norm_back(QkK g) {
    const int w = blockIdx.x < g.blocks0 ? 0 : 1;
    const QkSide& t = g.t[w];
    const int lane = threadIdx.x & (TEAM - 1), D = g.s.D;
    const int block = blockIdx.x - (w ? g.blocks0 : 0), blocks = w ? gridDim.x - g.blocks0 : g.blocks0;
    Mine<VP, PAIRS> m;
    m.place(g.s, lane, g.lanes, t.gamma);
    float sum[2 * VP];
#pragma unroll
    for (int j = 0; j < 2 * VP; ++j) sum[j] = 0.0f;
    for (int64_t item = (int64_t)block * (256 / TEAM) + threadIdx.x / TEAM; item < g.items[w];
         item += (int64_t)blocks * (256 / TEAM)) {
        const QkItem me = qk_item(g, w, item);
        m.turn(g.s, lane, me.at);
        for (int head = me.h0; head < me.h1; ++head) {
            float x[2 * VP], dz[2 * VP];
            m.load((const T*)t.x + me.tok * t.ld + (int64_t)head * D, D, x);
            m.load((const T*)t.dy + (me.tok * t.heads + head) * D, D, dz);
#pragma unroll
            for (int j = 0; j < VP; ++j) {
                const int a = m.first(j), b = m.second(j);
                m.turn_pair(dz[a], dz[b], m.c[j], -m.s[j], dz[a], dz[b]);
            }
            float dot, up;
            auto sums = [&] {
                float sq = 0.0f;
                dot = 0.0f;
#pragma unroll
                for (int j = 0; j < 2 * VP; ++j) {
                    sq = __builtin_fmaf(x[j], x[j], sq);
                    dot = __builtin_fmaf(dz[j] * m.g[j], x[j], dot);
                }
                return team_sum<TEAM>(sq);
            };
            const float r = unit<T, TEAM>(x, sums(), D, g.s.eps, up, sums);
            const float mean = team_sum<TEAM>(dot) * r / (float)D, rx = r * up;
#pragma unroll
            for (int j = 0; j < 2 * VP; ++j) {
                const float n = x[j] * r;
                sum[j] = __builtin_fmaf(dz[j], n, sum[j]);
                x[j] = rx * (dz[j] * m.g[j] - n * mean);
            }
            m.store((T*)t.dx + me.tok * t.ld + (int64_t)head * D, D, x);
        }
    }
    if (!t.dgamma) return;                           // of the whole workgroup
    // teams of a wave, then the four waves
    __shared__ float rows[4][128];
    const int wave = threadIdx.x >> 6;
#pragma unroll
    for (int j = 0; j < 2 * VP; ++j) {
        float x = sum[j];
#pragma unroll
        for (int d = TEAM; d < 64; d <<= 1) x += __shfl_xor(x, d, 64);
        const int at = j < VP ? m.d0 + j : m.d1 + j - VP;
        if (m.on && (threadIdx.x & 63) < TEAM && at < D) rows[wave][at] = x;
    }
    __syncthreads();
    if (threadIdx.x < (unsigned)D) {
        const int d = threadIdx.x;
        g.part[(int64_t)blockIdx.x * D + d] = (rows[0][d] + rows[1][d]) + (rows[2][d] + rows[3][d]);
    }
}

// dgamma of tensor blockIdx.y, channels 4 blockIdx.x ..: 64 threads a channel.
__global__ __launch_bounds__(256) void k_qk_norm_gamma(QkK g, int blocks1) {
    const int w = blockIdx.y, d = blockIdx.x * 4 + (threadIdx.x & 3), i0 = threadIdx.x >> 2;
    if (!g.t[w].dgamma) return;
    const int count = w ? blocks1 : g.blocks0;
    const float* p = g.part + (int64_t)(w ? g.blocks0 : 0) * g.s.D;
    float sum = 0.0f;
    if (d < g.s.D)
#pragma unroll 8
        for (int i = i0; i < count; i += 64) sum += p[(int64_t)i * g.s.D + d];
    __shared__ float s[64][4];
    s[i0][threadIdx.x & 3] = sum;
    __syncthreads();
    if (threadIdx.x < 4 && d < g.s.D) {
        float all = 0.0f;
#pragma unroll 16
        for (int i = 0; i < 64; ++i) all += s[i][threadIdx.x];
        g.t[w].dgamma[d] = all;
    }
}

int team_of(int lanes) {
    int t = 2;
    while (t < lanes) t *= 2;
    return t;
}

QkK args_of(const QkShape& s, const QkSide (&t)[2], const QkPlan& p) {
    QkK g{};
    g.s = s;
    g.lanes = ((s.D + 1) / 2 + p.vp - 1) / p.vp;
    g.blocks0 = p.blocks[0];
    for (int w = 0; w < 2; ++w) {
        g.t[w] = t[w];
        g.items[w] = p.items[w];
        g.chunks[w] = t[w].heads ? (t[w].heads + kHeads - 1) / kHeads : 1;
        g.by_chunk[w] = make_fastdiv((uint32_t)g.chunks[w]);
        g.by_len[w] = make_fastdiv((uint32_t)(t[w].L ? t[w].L : 1));
    }
    return g;
}

// f(value of the type, pairs a lane, team, pairs) for the plan
template <typename T, int VP, typename F>
void with_team(int team, bool pairs, F f) {
    auto go = [&](auto tm) {
        if (pairs) f(T(), std::integral_constant<int, VP>(), tm, std::true_type());
        else f(T(), std::integral_constant<int, VP>(), tm, std::false_type());
    };
    // the widest team that VP pairs a lane of 64 pairs need
    constexpr int most = 64 / VP;
    if (team == 2) go(std::integral_constant<int, 2>());
    else if (team == 4) go(std::integral_constant<int, 4>());
    else if (team == 8) go(std::integral_constant<int, 8>());
    else if (team == 16) { if constexpr (most >= 16) go(std::integral_constant<int, 16>()); }
    else if (team == 32) { if constexpr (most >= 32) go(std::integral_constant<int, 32>()); }
    else { if constexpr (most >= 64) go(std::integral_constant<int, 64>()); }
}
template <typename F>
void with_plan(const QkShape& s, const QkPlan& p, F f) {
    auto type = [&](auto t) {
        typedef decltype(t) T;
        if constexpr (sizeof(T) == 2)
            if (p.vp == 8) return with_team<T, 8>(p.team, s.pairs, f);
        if (p.vp == 4) return with_team<T, 4>(p.team, s.pairs, f);
        if (p.vp == 2) return with_team<T, 2>(p.team, s.pairs, f);
        with_team<T, 1>(p.team, s.pairs, f);
    };
    if (s.io == Io::F32) type(float());
    else if (s.io == Io::F16) type((_Float16)0);
    else type((__bf16)0.0f);
}

}  // namespace

// Loads of VP values where D, R and R/2 are multiples of VP, so that pairs that do not turn
// together (channels from R on) come in whole lanes.
QkPlan qk_plan(const QkShape& s, const QkSide (&t)[2], bool backward) {
    QkPlan p{};
    auto whole = [&](int vp) { return s.D % (2 * vp) == 0 && (s.pairs ? s.R % (2 * vp) == 0 : s.R / 2 % vp == 0); };
    p.vp = s.io != Io::F32 && whole(8) ? 8 : whole(4) ? 4 : whole(2) ? 2 : 1;
    p.team = team_of(((s.D + 1) / 2 + p.vp - 1) / p.vp);
    p.fits = true;
    for (int w = 0; w < 2; ++w) {
        p.items[w] = (int64_t)s.N * t[w].L * ((t[w].heads + kHeads - 1) / kHeads);
        if (p.items[w] > INT32_MAX) p.fits = false;
        const int64_t blocks = (p.items[w] + 256 / p.team - 1) / (256 / p.team);
        p.blocks[w] = (int)(backward && blocks > kBackBlocks / 2 ? kBackBlocks / 2 : blocks);
    }
    // a launch has fewer than 2^32 threads
    if ((int64_t)p.blocks[0] + p.blocks[1] >= (int64_t)1 << 24) p.fits = false;
    if (!backward) return p;
    // whatever R is: teams of the most lanes have the most workgroups
    const int per = 256 / team_of((s.D + 1) / 2);
    size_t rows = 0;
    for (int w = 0; w < 2; ++w) rows += (size_t)(p.items[w] / per + 1 < kBackBlocks / 2 ? p.items[w] / per + 1 : kBackBlocks / 2);
    p.need = round_up(rows * s.D * 4, 16);
    return p;
}

hipError_t launch_qk_norm(const QkShape& s, const QkSide (&t)[2], const QkPlan& p, hipStream_t st) {
    const QkK g = args_of(s, t, p);
    with_plan(s, p, [&](auto v, auto vp, auto team, auto pairs) {
        k_qk_norm<decltype(v), vp.value, team.value, pairs.value><<<p.blocks[0] + p.blocks[1], 256, 0, st>>>(g);
    });
    return hipGetLastError();
}

hipError_t launch_qk_norm_backward(const QkShape& s, const QkSide (&t)[2], const QkPlan& p, void* ws, hipStream_t st) {
    QkK g = args_of(s, t, p);
    g.part = (float*)ws;
    with_plan(s, p, [&](auto v, auto vp, auto team, auto pairs) {
        k_qk_norm_back<decltype(v), vp.value, team.value, pairs.value><<<p.blocks[0] + p.blocks[1], 256, 0, st>>>(g);
    });
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || (!t[0].dgamma && !t[1].dgamma)) return e;
    k_qk_norm_gamma<<<dim3((s.D + 3) / 4, 2), 256, 0, st>>>(g, p.blocks[1]);
    return hipGetLastError();
}

}  // namespace wino
