// Group norm with an activation, its backward pass and the 8-bit activation
// checkpoint, on channel-last tensors [N][P][C].
//
//   mean, rstd = 1 / sqrt(var + eps) over the P pixels of a group's D channels
//   n = (x - mean) rstd,  z = n gamma + beta,  y = act(z)
// and backwards, with dz = dy act'(z), m1 and m2 the group's means of gamma dz
// and gamma dz n:
//   dbeta = sum dz,  dgamma = sum dz n,  dx = rstd (gamma dz - m1 - n m2).
//
// All of it is bound by memory: about 20 operations a value.  So a workgroup
// loads its part of the tensor once and keeps it in registers.  Where a whole
// image of one group (or a few neighbouring ones) fits, the statistics are taken
// and the result is formed from there: one read, one write, one launch, and the
// variance about the mean itself.  Else three launches: every workgroup reduces
// its pixels, one joins these parts, and a second pass over the tensor forms the
// result.  All sums are in 32 bits and in a fixed order.
#include <math.h>

#include <type_traits>

#include "wino_norm_device.h"

namespace wino {

namespace {

constexpr int kMaxBlocks = 1 << 20;           // workgroups of a launch; they loop over the rest
constexpr int kXcds = 8;

// The part of the tensor that a workgroup works on, and its threads' share.
struct Cut {
    int C, G, D, cb, cv, rows, ncb, chunks;
    int64_t P, px, items;                     // px pixels a chunk; items = N * chunks * ncb
};

struct Item {
    int64_t n, p0, px;
    int chunk, c0;
};

// Item of a virtual block.  Blocks go to the 8 XCDs in turn; each XCD gets
// neighbouring items, channels fastest, so that workgroups that share the cache
// lines of a pixel share an L2.
__device__ __forceinline__ bool item_of(int64_t vb, const Cut& k, Item* it) {
    const int64_t per = (k.items + kXcds - 1) / kXcds, i = (vb % kXcds) * per + vb / kXcds;
    if (vb / kXcds >= per || i >= k.items) return false;
    const int64_t r = i / k.ncb;
    it->c0 = (int)(i - r * k.ncb) * k.cb;
    it->n = r / k.chunks;
    it->chunk = (int)(r - it->n * k.chunks);
    it->p0 = it->chunk * k.px;
    it->px = k.P - it->p0 < k.px ? k.P - it->p0 : k.px;
    return true;
}

// A thread's column of channels and first pixel; count: its pixels of the chunk,
// `rows` apart.
struct Share {
    int col, row, c, count;
};

__device__ __forceinline__ Share share_of(const Cut& k, const Item& it, int vec) {
    Share s;
    s.col = (int)threadIdx.x % k.cv;
    s.row = (int)threadIdx.x / k.cv;
    s.c = it.c0 + s.col * vec;
    const bool active = s.row < k.rows && s.c < k.C && s.row < it.px;
    s.count = active ? (int)((it.px - s.row + k.rows - 1) / k.rows) : 0;
    return s;
}

struct Add {
    static constexpr float identity = 0.0f;
    __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};
// NaN stays: a channel that holds one has no range.
struct Low {
    static constexpr float identity = INFINITY;
    __device__ __forceinline__ float operator()(float a, float b) const { return a != a || a < b ? a : b; }
};
struct High {
    static constexpr float identity = -INFINITY;
    __device__ __forceinline__ float operator()(float a, float b) const { return a != a || a > b ? a : b; }
};

// out[cb] = the threads' values of each channel joined: `sub` partial rows, then
// those; about 2 sqrt(rows) LDS reads a thread.
template <int VEC, typename Op>
__device__ void col_reduce(const float (&v)[VEC], const Cut& k, int sub, float* red, float* tmp, float* out, Op op) {
    const int t = threadIdx.x, nt = blockDim.x;
    if (t < k.rows * k.cv) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) red[t * VEC + j] = v[j];
    }
    __syncthreads();
    for (int i = t; i < sub * k.cb; i += nt) {
        const int c = i % k.cb;
        float a = Op::identity;
        for (int r = i / k.cb; r < k.rows; r += sub) a = op(a, red[r * k.cb + c]);
        tmp[i] = a;
    }
    __syncthreads();
    for (int c = t; c < k.cb; c += nt) {
        float a = tmp[c];
        for (int r = 1; r < sub; ++r) a = op(a, tmp[r * k.cb + c]);
        out[c] = a;
    }
    __syncthreads();
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int m = 32; m; m >>= 1) v += __shfl_xor(v, m);
    return v;
}

// gsum[g] = sum of csum over the group's channels, a wave a group.
template <typename F>
__device__ __forceinline__ void group_reduce(int groups, int D, float* gsum, F value) {
    const int lane = threadIdx.x & 63;
    for (int g = threadIdx.x >> 6; g < groups; g += blockDim.x >> 6) {
        float a = 0.0f;
        for (int d = lane; d < D; d += 64) a += value(g * D + d);
        a = wave_sum(a);
        if (lane == 0) gsum[g] = a;
    }
    __syncthreads();
}

template <typename F>
__device__ __forceinline__ void with_act(Act act, F&& f) {
    if (act == Act::Silu) f(std::integral_constant<Act, Act::Silu>());
    else if (act == Act::Relu) f(std::integral_constant<Act, Act::Relu>());
    else f(std::integral_constant<Act, Act::None>());
}

// ------------------------------------------------------------------ forward

struct FwdArgs {
    const void* x;
    const float *gamma, *beta;
    void* y;
    float* stats;
    int8_t* codes;
    float* rows;
    float* part;                              // [N][chunks][C][4] of mean, squares about it, low, high
    float eps;
    Act act;
    int sub;
};

// One image of whole groups (ONE), or the parts of the statistics.
template <typename T, int VEC, int NV, bool ONE>
__global__ __launch_bounds__(1024) void k_norm(FwdArgs a, Cut k) {
    extern __shared__ float lds[];
    float* red = lds;
    float* tmp = red + k.rows * k.cb;
    float* ca = tmp + a.sub * k.cb;
    float *cl = ca + k.cb, *ch = cl + k.cb, *gm = ch + k.cb, *gr = gm + k.cb;
    Item it;
    for (int64_t vb = blockIdx.x; vb / kXcds < (k.items + kXcds - 1) / kXcds; vb += gridDim.x) {
        if (!item_of(vb, k, &it)) continue;
        const Share s = share_of(k, it, VEC);
        const size_t at = ((size_t)it.n * k.P + it.p0 + s.row) * k.C + s.c, step = (size_t)k.rows * k.C;
        Raw<T, VEC> raw[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (i < s.count) raw[i] = *(const Raw<T, VEC>*)((const T*)a.x + at + i * step);
        const bool norm = !ONE || a.y || a.stats;
        float mean[VEC], v[VEC];
        if (norm) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) v[j] = 0.0f;
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (i < s.count)
#pragma unroll
                    for (int j = 0; j < VEC; ++j) v[j] += (float)raw[i].v[j];
            col_reduce(v, k, a.sub, red, tmp, ca, Add());
            if constexpr (ONE) {
                const float inv = 1.0f / ((float)k.P * (float)k.D);
                group_reduce(k.cb / k.D, k.D, gm, [&](int c) { return ca[c] * inv; });
            }
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const int c = s.col * VEC + j;
                mean[j] = ONE ? gm[c / k.D] : ca[c] / (float)it.px;
                v[j] = 0.0f;
            }
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (i < s.count)
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        const float d = (float)raw[i].v[j] - mean[j];
                        v[j] += d * d;
                    }
            col_reduce(v, k, a.sub, red, tmp, ca, Add());
            if constexpr (ONE) {
                const float inv = 1.0f / ((float)k.P * (float)k.D), eps = a.eps;
                group_reduce(k.cb / k.D, k.D, gr, [&](int c) { return ca[c] * inv; });
                for (int g = threadIdx.x; g < k.cb / k.D; g += blockDim.x) {
                    gr[g] = 1.0f / sqrtf(gr[g] + eps);
                    if (a.stats) {
                        float* st = a.stats + ((size_t)it.n * k.G + it.c0 / k.D + g) * 2;
                        st[0] = gm[g];
                        st[1] = gr[g];
                    }
                }
                __syncthreads();
            }
        }
        if (a.codes) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) v[j] = Low::identity;
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (i < s.count)
#pragma unroll
                    for (int j = 0; j < VEC; ++j) v[j] = Low()((float)raw[i].v[j], v[j]);
            col_reduce(v, k, a.sub, red, tmp, cl, Low());
#pragma unroll
            for (int j = 0; j < VEC; ++j) v[j] = High::identity;
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (i < s.count)
#pragma unroll
                    for (int j = 0; j < VEC; ++j) v[j] = High()((float)raw[i].v[j], v[j]);
            col_reduce(v, k, a.sub, red, tmp, ch, High());
        }
        if constexpr (!ONE) {
            // the mean of the channel's pixels of this chunk is in the threads of row 0
            if (s.row == 0 && s.c < k.C) {
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const int c = s.col * VEC + j;
                    float* p = a.part + (((size_t)it.n * k.chunks + it.chunk) * k.C + it.c0 + c) * 4;
                    p[0] = mean[j];
                    p[1] = ca[c];
                    p[2] = a.codes ? cl[c] : 0.0f;
                    p[3] = a.codes ? ch[c] : 0.0f;
                }
            }
        } else {
            if (a.codes) {
                Row r[VEC];
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const int c = s.col * VEC + j;
                    r[j] = row_of(cl[c], ch[c]);
                    if (s.row == 0) {
                        float* p = a.rows + ((size_t)it.n * k.C + s.c + j) * 2;
                        p[0] = r[j].centre;
                        p[1] = r[j].step;
                    }
                }
#pragma unroll
                for (int i = 0; i < NV; ++i)
                    if (i < s.count) {
                        Raw<int8_t, VEC> q;
#pragma unroll
                        for (int j = 0; j < VEC; ++j) q.v[j] = code_of((float)raw[i].v[j], r[j]);
                        *(Raw<int8_t, VEC>*)(a.codes + at + i * step) = q;
                    }
            }
            if (a.y) {
                Affine f[VEC];
                if (s.count)
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        const int c = s.col * VEC + j;
                        f[j] = Affine{mean[j], gr[c / k.D], a.gamma ? a.gamma[s.c + j] : 1.0f,
                                      a.beta ? a.beta[s.c + j] : 0.0f};
                    }
                with_act(a.act, [&](auto act) {
#pragma unroll
                    for (int i = 0; i < NV; ++i)
                        if (i < s.count) {
                            Raw<T, VEC> o;
#pragma unroll
                            for (int j = 0; j < VEC; ++j)
                                o.v[j] = (T)act_of<act.value>(f[j].z(f[j].norm((float)raw[i].v[j])));
                            *(Raw<T, VEC>*)((T*)a.y + at + i * step) = o;
                        }
                });
            }
        }
        __syncthreads();                      // the next item writes the LDS arrays
    }
}

// Joins the parts of one image and group: mean and variance about it, and each
// channel's range.  A workgroup an (image, group).
__global__ __launch_bounds__(256) void k_norm_join(const float* __restrict__ part, float* __restrict__ stats,
                                                   float* __restrict__ rows, float* __restrict__ inverse, Cut k,
                                                   int64_t groups, float eps) {
    __shared__ float acc[4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int64_t ng = blockIdx.x; ng < groups; ng += gridDim.x) {
        const int64_t n = ng / k.G;
        const int g = (int)(ng - n * k.G);
        const float* p = part + ((size_t)n * k.chunks * k.C + (size_t)g * k.D) * 4;
        const int64_t all = (int64_t)k.chunks * k.D;
        const float inv = 1.0f / ((float)k.P * (float)k.D);
        auto total = [&](auto value) {
            float a = 0.0f;
            for (int64_t i = threadIdx.x; i < all; i += 256) {
                const int64_t ch = i / k.D, d = i - ch * k.D;
                const int64_t px = k.P - ch * k.px < k.px ? k.P - ch * k.px : k.px;
                a += value(p + ((size_t)ch * k.C + d) * 4, (float)px);
            }
            a = wave_sum(a);
            __syncthreads();
            if (lane == 0) acc[wave] = a;
            __syncthreads();
            return acc[0] + acc[1] + acc[2] + acc[3];
        };
        if (stats) {
            const float mean = total([&](const float* q, float px) { return q[0] * px; }) * inv;
            const float var = total([&](const float* q, float px) {
                const float d = q[0] - mean;
                return q[1] + px * d * d;
            }) * inv;
            if (threadIdx.x == 0) {
                stats[((size_t)n * k.G + g) * 2] = mean;
                stats[((size_t)n * k.G + g) * 2 + 1] = 1.0f / sqrtf(var + eps);
            }
        }
        if (rows)
            for (int d = threadIdx.x; d < k.D; d += 256) {
                float lo = Low::identity, hi = High::identity;
                for (int ch = 0; ch < k.chunks; ++ch) {
                    const float* q = p + ((size_t)ch * k.C + d) * 4;
                    lo = Low()(q[2], lo);
                    hi = High()(q[3], hi);
                }
                const Row r = row_of(lo, hi);
                float* o = rows + ((size_t)n * k.C + (size_t)g * k.D + d) * 2;
                o[0] = r.centre;
                o[1] = r.step;
                inverse[(size_t)n * k.C + (size_t)g * k.D + d] = r.inverse;
            }
    }
}

struct ApplyArgs {
    const void* x;
    const int8_t* codes;                      // in place of x, with rows
    const float *rows, *stats, *gamma, *beta;
    void* y;
    int8_t* out;                              // codes to write, from x, with rows and
    const float* inverse;                     // 1 / step [N][C]
    Act act;
};

// The second pass: y (and the codes) from x or codes and the statistics.
template <typename T, int VEC, bool X8>
__global__ __launch_bounds__(256) void k_norm_apply(ApplyArgs a, Cut k) {
    constexpr int U = VEC == 1 ? 8 : 4;       // loads in flight
    typedef typename std::conditional<X8, int8_t, T>::type S;
    Item it;
    for (int64_t vb = blockIdx.x; vb / kXcds < (k.items + kXcds - 1) / kXcds; vb += gridDim.x) {
        if (!item_of(vb, k, &it)) continue;
        const Share s = share_of(k, it, VEC);
        if (!s.count) continue;
        const size_t at = ((size_t)it.n * k.P + it.p0 + s.row) * k.C + s.c, step = (size_t)k.rows * k.C;
        const S* src = (X8 ? (const S*)a.codes : (const S*)a.x) + at;
        Affine f[VEC];
        Row r[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            const int c = s.c + j;
            if (a.stats) {
                const float* st = a.stats + ((size_t)it.n * k.G + c / k.D) * 2;
                f[j] = Affine{st[0], st[1], a.gamma ? a.gamma[c] : 1.0f, a.beta ? a.beta[c] : 0.0f};
            }
            if (X8 || a.out) {
                const float* p = a.rows + ((size_t)it.n * k.C + c) * 2;
                r[j].centre = p[0];
                r[j].step = p[1];
                r[j].inverse = a.out ? a.inverse[(size_t)it.n * k.C + c] : 0.0f;
            }
        }
        with_act(a.act, [&](auto act) {
            for (int i0 = 0; i0 < s.count; i0 += U) {
                Raw<S, VEC> raw[U];
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (i0 + u < s.count) raw[u] = *(const Raw<S, VEC>*)(src + (i0 + u) * step);
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (i0 + u < s.count) {
                        Raw<T, VEC> o;
#pragma unroll
                        for (int j = 0; j < VEC; ++j) {
                            float v;
                            if constexpr (X8) v = value_of(raw[u].v[j], r[j].centre, r[j].step);
                            else v = (float)raw[u].v[j];
                            o.v[j] = (T)(a.stats ? act_of<act.value>(f[j].z(f[j].norm(v))) : v);
                        }
                        if (a.y) *(Raw<T, VEC>*)((T*)a.y + at + (i0 + u) * step) = o;
                    }
                if constexpr (!X8) {
                    if (a.out) {
#pragma unroll
                        for (int u = 0; u < U; ++u)
                            if (i0 + u < s.count) {
                                Raw<int8_t, VEC> q;
#pragma unroll
                                for (int j = 0; j < VEC; ++j) q.v[j] = code_of((float)raw[u].v[j], r[j]);
                                *(Raw<int8_t, VEC>*)(a.out + at + (i0 + u) * step) = q;
                            }
                    }
                }
            }
        });
    }
}

// ------------------------------------------------------------------ backward

struct BwdArgs {
    const void *dy, *x;
    const int8_t* codes;
    const float *rows, *stats, *gamma, *beta;
    void* dx;
    float* part;                              // [N][chunks][C][2] of sum dz, sum dz n
    float* means;                             // [N][G][2] of m1, m2 (not ONE)
    Act act;
    int sub;
};

// One thread's channel constants.
template <int VEC, bool X8>
__device__ __forceinline__ void bwd_rows(const BwdArgs& a, const Cut& k, int64_t n, int c0, Affine (&f)[VEC],
                                         float (&centre)[VEC], float (&step)[VEC]) {
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
        const int c = c0 + j;
        const float* st = a.stats + ((size_t)n * k.G + c / k.D) * 2;
        f[j] = Affine{st[0], st[1], a.gamma ? a.gamma[c] : 1.0f, a.beta ? a.beta[c] : 0.0f};
        if constexpr (X8) {
            centre[j] = a.rows[((size_t)n * k.C + c) * 2];
            step[j] = a.rows[((size_t)n * k.C + c) * 2 + 1];
        }
    }
}

template <bool X8, typename S, int VEC>
__device__ __forceinline__ float x_of(const Raw<S, VEC>& raw, int j, const float (&centre)[VEC],
                                      const float (&step)[VEC]) {
    if constexpr (X8) return value_of(raw.v[j], centre[j], step[j]);
    else return (float)raw.v[j];
}

template <typename T, int VEC, int NV, bool X8, bool ONE>
__global__ __launch_bounds__(1024) void k_norm_back(BwdArgs a, Cut k) {
    extern __shared__ float lds[];
    typedef typename std::conditional<X8, int8_t, T>::type S;
    float* red = lds;
    float* tmp = red + k.rows * k.cb;
    float* cz = tmp + a.sub * k.cb;
    float *cn = cz + k.cb, *g1 = cn + k.cb, *g2 = g1 + k.cb;
    Item it;
    for (int64_t vb = blockIdx.x; vb / kXcds < (k.items + kXcds - 1) / kXcds; vb += gridDim.x) {
        if (!item_of(vb, k, &it)) continue;
        const Share s = share_of(k, it, VEC);
        const size_t at = ((size_t)it.n * k.P + it.p0 + s.row) * k.C + s.c, step = (size_t)k.rows * k.C;
        const S* src = (X8 ? (const S*)a.codes : (const S*)a.x) + at;
        Raw<T, VEC> dy[NV];
        Raw<S, VEC> x[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (i < s.count) {
                dy[i] = *(const Raw<T, VEC>*)((const T*)a.dy + at + i * step);
                x[i] = *(const Raw<S, VEC>*)(src + i * step);
            }
        Affine f[VEC];
        float centre[VEC], stp[VEC], sz[VEC], sn[VEC];
        if (s.count) bwd_rows<VEC, X8>(a, k, it.n, s.c, f, centre, stp);
#pragma unroll
        for (int j = 0; j < VEC; ++j) sz[j] = sn[j] = 0.0f;
        with_act(a.act, [&](auto act) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (i < s.count)
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        const float n = f[j].norm(x_of<X8, S, VEC>(x[i], j, centre, stp));
                        const float dz = dact<act.value>(f[j].z(n), (float)dy[i].v[j]);
                        sz[j] += dz;
                        sn[j] += dz * n;
                    }
        });
        col_reduce(sz, k, a.sub, red, tmp, cz, Add());
        col_reduce(sn, k, a.sub, red, tmp, cn, Add());
        for (int c = threadIdx.x; c < k.cb && it.c0 + c < k.C; c += blockDim.x) {
            float* p = a.part + (((size_t)it.n * k.chunks + it.chunk) * k.C + it.c0 + c) * 2;
            p[0] = cz[c];
            p[1] = cn[c];
        }
        if constexpr (ONE) {
            const float inv = 1.0f / ((float)k.P * (float)k.D);
            auto weight = [&](int c) { return a.gamma ? a.gamma[it.c0 + c] * inv : inv; };
            group_reduce(k.cb / k.D, k.D, g1, [&](int c) { return cz[c] * weight(c); });
            group_reduce(k.cb / k.D, k.D, g2, [&](int c) { return cn[c] * weight(c); });
            float m1[VEC], m2[VEC];
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const int g = (s.col * VEC + j) / k.D;
                m1[j] = g1[g];
                m2[j] = g2[g];
            }
            with_act(a.act, [&](auto act) {
#pragma unroll
                for (int i = 0; i < NV; ++i)
                    if (i < s.count) {
                        Raw<T, VEC> o;
#pragma unroll
                        for (int j = 0; j < VEC; ++j) {
                            const float n = f[j].norm(x_of<X8, S, VEC>(x[i], j, centre, stp));
                            const float dz = dact<act.value>(f[j].z(n), (float)dy[i].v[j]);
                            o.v[j] = (T)(f[j].rstd * (dz * f[j].gamma - m1[j] - n * m2[j]));
                        }
                        *(Raw<T, VEC>*)((T*)a.dx + at + i * step) = o;
                    }
            });
        }
        __syncthreads();
    }
}

// means[n][g] = the group's m1, m2 from its channels' parts.  A workgroup an
// (image, group).
__global__ __launch_bounds__(256) void k_norm_back_join(const float* __restrict__ part, const float* __restrict__ gamma,
                                                        float* __restrict__ means, Cut k, int64_t groups) {
    __shared__ float acc[8];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int64_t ng = blockIdx.x; ng < groups; ng += gridDim.x) {
        const int64_t n = ng / k.G;
        const int g = (int)(ng - n * k.G);
        const float* p = part + ((size_t)n * k.chunks * k.C + (size_t)g * k.D) * 2;
        const float inv = 1.0f / ((float)k.P * (float)k.D);
        float m1 = 0.0f, m2 = 0.0f;
        for (int64_t i = threadIdx.x; i < (int64_t)k.chunks * k.D; i += 256) {
            const int64_t ch = i / k.D, d = i - ch * k.D;
            const float w = gamma ? gamma[(size_t)g * k.D + d] * inv : inv;
            const float* q = p + ((size_t)ch * k.C + d) * 2;
            m1 += q[0] * w;
            m2 += q[1] * w;
        }
        m1 = wave_sum(m1);
        m2 = wave_sum(m2);
        if (lane == 0) {
            acc[wave * 2] = m1;
            acc[wave * 2 + 1] = m2;
        }
        __syncthreads();
        if (threadIdx.x < 2)
            means[((size_t)n * k.G + g) * 2 + threadIdx.x] =
                acc[threadIdx.x] + acc[threadIdx.x + 2] + acc[threadIdx.x + 4] + acc[threadIdx.x + 6];
        __syncthreads();
    }
}

template <typename T, int VEC, bool X8>
__global__ __launch_bounds__(256) void k_norm_back_apply(BwdArgs a, Cut k) {
    constexpr int U = VEC == 1 ? 8 : 4;
    typedef typename std::conditional<X8, int8_t, T>::type S;
    Item it;
    for (int64_t vb = blockIdx.x; vb / kXcds < (k.items + kXcds - 1) / kXcds; vb += gridDim.x) {
        if (!item_of(vb, k, &it)) continue;
        const Share s = share_of(k, it, VEC);
        if (!s.count) continue;
        const size_t at = ((size_t)it.n * k.P + it.p0 + s.row) * k.C + s.c, step = (size_t)k.rows * k.C;
        const S* src = (X8 ? (const S*)a.codes : (const S*)a.x) + at;
        Affine f[VEC];
        float centre[VEC], stp[VEC], m1[VEC], m2[VEC];
        bwd_rows<VEC, X8>(a, k, it.n, s.c, f, centre, stp);
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            const float* m = a.means + ((size_t)it.n * k.G + (s.c + j) / k.D) * 2;
            m1[j] = m[0];
            m2[j] = m[1];
        }
        with_act(a.act, [&](auto act) {
            for (int i0 = 0; i0 < s.count; i0 += U) {
                Raw<T, VEC> dy[U];
                Raw<S, VEC> x[U];
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (i0 + u < s.count) {
                        dy[u] = *(const Raw<T, VEC>*)((const T*)a.dy + at + (i0 + u) * step);
                        x[u] = *(const Raw<S, VEC>*)(src + (i0 + u) * step);
                    }
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (i0 + u < s.count) {
                        Raw<T, VEC> o;
#pragma unroll
                        for (int j = 0; j < VEC; ++j) {
                            const float n = f[j].norm(x_of<X8, S, VEC>(x[u], j, centre, stp));
                            const float dz = dact<act.value>(f[j].z(n), (float)dy[u].v[j]);
                            o.v[j] = (T)(f[j].rstd * (dz * f[j].gamma - m1[j] - n * m2[j]));
                        }
                        *(Raw<T, VEC>*)((T*)a.dx + at + (i0 + u) * step) = o;
                    }
            }
        });
    }
}

// dgamma, dbeta: the parts of every image and chunk, 32 channels a workgroup.
__global__ __launch_bounds__(256) void k_norm_params(const float* __restrict__ part, float* __restrict__ dgamma,
                                                     float* __restrict__ dbeta, int64_t lists, int C) {
    __shared__ float acc[2][8][32];
    const int c = blockIdx.x * 32 + (threadIdx.x & 31), row = threadIdx.x >> 5;
    float z = 0.0f, n = 0.0f;
    if (c < C)
        for (int64_t i = row; i < lists; i += 8) {
            const float* p = part + ((size_t)i * C + c) * 2;
            z += p[0];
            n += p[1];
        }
    acc[0][row][threadIdx.x & 31] = z;
    acc[1][row][threadIdx.x & 31] = n;
    __syncthreads();
    if (row == 0 && c < C) {
        for (int r = 1; r < 8; ++r) {
            z += acc[0][r][threadIdx.x];
            n += acc[1][r][threadIdx.x];
        }
        if (dbeta) dbeta[c] = z;
        if (dgamma) dgamma[c] = n;
    }
}

// ------------------------------------------------------------------ host

int64_t gcd(int64_t a, int64_t b) { return b ? gcd(b, a % b) : a; }
int sub_rows(int threads, int rows, int cb) {
    int s = 1;
    while (s * s < rows && (s + 1) * cb <= threads) ++s;
    return s;
}

Cut cut_of(const NormShape& s, const NormPlan& p) {
    Cut k;
    k.C = s.C; k.G = s.G; k.D = s.D;
    k.cb = p.cb; k.cv = p.cv; k.rows = p.rows;
    k.ncb = (s.C + p.cb - 1) / p.cb;
    k.chunks = p.chunks;
    k.P = s.P;
    k.px = p.px;
    k.items = (int64_t)s.N * p.chunks * k.ncb;
    return k;
}

unsigned blocks_of(int64_t items) {
    const int64_t b = (items + kXcds - 1) / kXcds * kXcds;
    return (unsigned)(b < kMaxBlocks ? b : kMaxBlocks);
}

// The cut of the element-wise pass: 256 threads, 16 pixels a thread.
NormPlan apply_plan(const NormShape& s, bool aligned) {
    NormPlan p = {};
    const int full = 16 / io_size(s.io);
    p.vec = aligned && s.C % full == 0 ? full : 1;
    p.threads = 256;
    const int cols = (s.C + p.vec - 1) / p.vec;
    p.cv = cols < 256 ? cols : 256;
    p.cb = p.cv * p.vec;
    p.rows = 256 / p.cv;
    p.px = (int64_t)p.rows * 16;
    p.chunks = (int)((s.P + p.px - 1) / p.px);
    return p;
}

// f(T, VEC) for the element type and vector width.
template <typename F>
void with_type(Io io, int vec, F&& f) {
    if (io == Io::F32) {
        if (vec == 1) f(float(), std::integral_constant<int, 1>());
        else f(float(), std::integral_constant<int, 4>());
    } else if (io == Io::F16) {
        if (vec == 1) f(_Float16(), std::integral_constant<int, 1>());
        else f(_Float16(), std::integral_constant<int, 8>());
    } else {
        if (vec == 1) f(__bf16(), std::integral_constant<int, 1>());
        else f(__bf16(), std::integral_constant<int, 8>());
    }
}

}  // namespace

NormPlan norm_plan(const NormShape& s, bool backward, bool aligned) {
    NormPlan p = {};
    const int full = 16 / io_size(s.io);
    p.vec = aligned && s.C % full == 0 ? full : 1;
    const int most = (p.vec == 1 ? 64 : 16) / (backward ? 2 : 1);
    // one pass: whole groups whose image fits the registers
    const int64_t unit = (int64_t)s.D / gcd(s.D, p.vec) * p.vec;
    for (int64_t k = 1; !p.one && unit * k <= 1024 && unit * k <= s.C; ++k) {
        if (s.C % (unit * k)) continue;
        const int64_t cb = unit * k;
        if (cb * io_size(s.io) < 32 && cb < s.C && cb < 1024 && s.P * cb / p.vec < 256 * most) continue;
        for (int threads = 256; threads <= 1024 && !p.one; threads *= 2) {
            const int cv = (int)(cb / p.vec);
            if (cv > threads) continue;
            const int rows = threads / cv;
            for (int nv = most / 4; nv <= most && !p.one; nv *= 4) {
                if (s.P > (int64_t)rows * nv) continue;
                p.one = true;
                p.nv = nv;
                p.threads = threads;
                p.cb = (int)cb;
                p.cv = cv;
                p.rows = rows;
                p.chunks = 1;
                p.px = s.P;
            }
        }
    }
    if (!p.one) {
        p.threads = 256;
        p.nv = most;
        const int cols = (s.C + p.vec - 1) / p.vec;
        p.cv = cols < 128 ? cols : 128;
        p.cb = p.cv * p.vec;
        p.rows = p.threads / p.cv;
        p.px = (int64_t)p.rows * p.nv;
        p.chunks = (int)((s.P + p.px - 1) / p.px);
    }
    const int sub = sub_rows(p.threads, p.rows, p.cb);
    p.lds = ((size_t)p.rows * p.cb + (size_t)sub * p.cb + 5 * (size_t)p.cb) * sizeof(float);
    const size_t lists = (size_t)s.N * p.chunks * s.C, groups = (size_t)s.N * s.G * 2 * sizeof(float);
    if (backward) p.need = lists * 2 * sizeof(float) + (p.one ? 0 : groups);
    else p.need = p.one ? 0 : (lists * 4 + (size_t)s.N * s.C) * sizeof(float) + groups;
    return p;
}

hipError_t launch_norm_apply(const NormApply& a, const NormShape& s, bool aligned, hipStream_t st) {
    const NormPlan p = apply_plan(s, aligned);
    const Cut k = cut_of(s, p);
    const ApplyArgs g{a.x, a.codes, a.rows, a.stats, a.gamma, a.beta, a.y, nullptr, nullptr, s.act};
    with_type(s.io, p.vec, [&](auto t, auto vec) {
        typedef decltype(t) T;
        if (a.codes) k_norm_apply<T, vec.value, true><<<blocks_of(k.items), 256, 0, st>>>(g, k);
        else k_norm_apply<T, vec.value, false><<<blocks_of(k.items), 256, 0, st>>>(g, k);
    });
    return hipGetLastError();
}

hipError_t launch_norm(const NormFwd& a, const NormShape& s, const NormPlan& p, void* ws, hipStream_t st) {
    const Cut k = cut_of(s, p);
    float* part = (float*)ws;
    float* inverse = part + (size_t)s.N * p.chunks * s.C * 4;
    float* own = inverse + (size_t)s.N * s.C;                  // the statistics, where the caller wants none
    const FwdArgs g{a.x, a.gamma, a.beta, a.y, a.stats, a.codes, a.rows, part, a.eps, s.act,
                    sub_rows(p.threads, p.rows, p.cb)};
    with_type(s.io, p.vec, [&](auto t, auto vec) {
        typedef decltype(t) T;
        constexpr int V = vec.value, most = V == 1 ? 64 : 16;
        const unsigned b = blocks_of(k.items);
        if (!p.one) k_norm<T, V, most, false><<<b, p.threads, p.lds, st>>>(g, k);
        else if (p.nv == most) k_norm<T, V, most, true><<<b, p.threads, p.lds, st>>>(g, k);
        else k_norm<T, V, most / 4, true><<<b, p.threads, p.lds, st>>>(g, k);
    });
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.one) return e;
    const bool norm = a.y || a.stats;
    float* stats = a.stats ? a.stats : own;
    k_norm_join<<<blocks_of((int64_t)s.N * s.G), 256, 0, st>>>(part, norm ? stats : nullptr,
                                                              a.codes ? a.rows : nullptr, inverse, k, (int64_t)s.N * s.G,
                                                              a.eps);
    e = hipGetLastError();
    if (e != hipSuccess || (!a.y && !a.codes)) return e;
    const NormPlan q = apply_plan(s, p.vec > 1);
    const Cut kq = cut_of(s, q);
    const ApplyArgs h{a.x, nullptr, a.rows, a.y ? stats : nullptr, a.gamma, a.beta, a.y, a.codes, inverse,
                      s.act};
    with_type(s.io, q.vec, [&](auto t, auto vec) {
        typedef decltype(t) T;
        k_norm_apply<T, vec.value, false><<<blocks_of(kq.items), 256, 0, st>>>(h, kq);
    });
    return hipGetLastError();
}

hipError_t launch_norm_backward(const NormBwd& a, const NormShape& s, const NormPlan& p, void* ws, hipStream_t st) {
    const Cut k = cut_of(s, p);
    float* part = (float*)ws;
    float* means = part + (size_t)s.N * p.chunks * s.C * 2;
    const BwdArgs g{a.dy, a.x, a.codes, a.rows, a.stats, a.gamma, a.beta, a.dx, part, means, s.act,
                    sub_rows(p.threads, p.rows, p.cb)};
    const bool x8 = a.codes != nullptr;
    with_type(s.io, p.vec, [&](auto t, auto vec) {
        typedef decltype(t) T;
        constexpr int V = vec.value, most = V == 1 ? 64 : 16;
        const unsigned b = blocks_of(k.items);
        auto go = [&](auto c8) {
            constexpr bool X8 = c8.value;
            if (!p.one) k_norm_back<T, V, most / 2, X8, false><<<b, p.threads, p.lds, st>>>(g, k);
            else if (p.nv == most / 2) k_norm_back<T, V, most / 2, X8, true><<<b, p.threads, p.lds, st>>>(g, k);
            else k_norm_back<T, V, most / 8, X8, true><<<b, p.threads, p.lds, st>>>(g, k);
        };
        if (x8) go(std::true_type());
        else go(std::false_type());
    });
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (!p.one) {
        k_norm_back_join<<<blocks_of((int64_t)s.N * s.G), 256, 0, st>>>(part, a.gamma, means, k, (int64_t)s.N * s.G);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
        const NormPlan q = apply_plan(s, p.vec > 1);
        const Cut kq = cut_of(s, q);
        with_type(s.io, q.vec, [&](auto t, auto vec) {
            typedef decltype(t) T;
            if (x8) k_norm_back_apply<T, vec.value, true><<<blocks_of(kq.items), 256, 0, st>>>(g, kq);
            else k_norm_back_apply<T, vec.value, false><<<blocks_of(kq.items), 256, 0, st>>>(g, kq);
        });
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (a.dgamma || a.dbeta)
        k_norm_params<<<(s.C + 31) / 32, 256, 0, st>>>(part, a.dgamma, a.dbeta, (int64_t)s.N * p.chunks, s.C);
    return hipGetLastError();
}

}  // namespace wino
