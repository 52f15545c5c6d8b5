// Group norm with an activation, its backward pass and the 8-bit activation
// checkpoint, on channel-last tensors [N][P][C].
//
//   mean, rstd = 1 / sqrt(var + eps) over the P pixels of a group's D channels
//   n = (x - mean) rstd,  z = n gamma + beta,  y = act(z)
// and backwards, with dz = dy act'(z), m1 and m2 the group's means of gamma dz
// and gamma dz n:
//   dbeta = sum dz,  dgamma = sum dz n,  dx = rstd (gamma dz - m1 - n m2).
//
// All of it is bound by memory, about 20 operations a value, if it reads the
// tensor once.  So where a whole image of one group (or a few neighbouring ones)
// fits a workgroup's registers, it is loaded once and the statistics are taken and
// the result formed from there: one read, one write, one launch, and the variance
// about the mean itself.  Else three launches: every workgroup reduces its pixels,
// one joins these parts, and a second pass over the tensor forms the result.  Sums are in
// a fixed order: a thread's in 32 bits, of kFlush terms and then of kFlush of these, so
// that with the joins (64 bits where they are long) no sum is more than 256 roundings off,
// whatever the tensor's size (4096 terms in turn: 6e-5 of the sum; the second level costs
// 1% of the large tensors' time at most, 3% one channel a lane).
#include <math.h>

#include <type_traits>

#include "wino_norm_device.h"

namespace wino {

namespace {

constexpr unsigned kMaxBlocks = 1 << 20;      // workgroups of a launch; they loop over the rest
constexpr unsigned kXcds = 8;
constexpr int kMaxThreads = 512;              // of the one-pass kernels
constexpr int kFlush = 64;                    // terms of a thread's sum before they join its total

// The part of the tensor that a workgroup works on, and its threads' share.  A
// thread has one column of `vec` channels and the pixels of its row, `rows`
// apart.  wrows > 0: a wave holds wrows whole rows of cv lanes (the lanes left
// over idle) and joins them by lane shuffles; else the columns run on from wave
// to wave.  `parts` values of each channel are left to join through LDS.
struct Cut {
    int C, G, D, cb, cv, rows, wrows, parts;
    uint32_t ncb, chunks, items, per;         // items = N * chunks * ncb, per XCD
    int64_t P, px;                            // px pixels a chunk
    FastDiv dcv, dD, dncb, dchunks;
    float inv;                                // 1 / (P D)
};

struct Item {
    int64_t n, p0, px;
    int chunk, c0;
};

// Item of a virtual block.  Blocks go to the 8 XCDs in turn; each XCD gets
// neighbouring items, channels fastest, so that workgroups that share the cache
// lines of a pixel share an L2.
__device__ __forceinline__ bool item_of(uint32_t vb, const Cut& k, Item* it) {
    const uint32_t i = vb % kXcds * k.per + vb / kXcds;
    if (i >= k.items) return false;
    const uint32_t r = fdiv(i, k.dncb), n = fdiv(r, k.dchunks);
    it->c0 = (int)(i - r * k.ncb) * k.cb;
    it->n = n;
    it->chunk = (int)(r - n * k.chunks);
    it->p0 = it->chunk * k.px;
    it->px = k.P - it->p0 < k.px ? k.P - it->p0 : k.px;
    return true;
}

// A thread's column of channels, first pixel and number of pixels.
struct Share {
    int col, row, c, count;
};

__device__ __forceinline__ Share share_of(const Cut& k, const Item& it, int vec) {
    Share s;
    const int t = threadIdx.x, i = k.wrows ? t & 63 : t, row = (int)fdiv(i, k.dcv);
    const bool idle = k.wrows && row >= k.wrows;
    s.col = idle ? 0 : i - row * k.cv;
    s.row = idle ? k.rows : k.wrows ? (t >> 6) * k.wrows + row : row;
    s.c = it.c0 + s.col * vec;
    const bool active = s.row < k.rows && s.c < k.C && s.row < it.px;
    s.count = active ? (int)((uint32_t)(it.px - s.row + k.rows - 1) / (uint32_t)k.rows) : 0;
    return s;
}

struct Add {
    __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};
// These keep NaN: a channel that holds one has no range.
struct Low {
    static constexpr float identity = INFINITY;
    __device__ __forceinline__ float operator()(float a, float b) const { return __builtin_elementwise_minimum(a, b); }
};
struct High {
    static constexpr float identity = -INFINITY;
    __device__ __forceinline__ float operator()(float a, float b) const { return __builtin_elementwise_maximum(a, b); }
};

// v joined with the lanes `ROR` further on, in turn, of each row of 16 (DPP row_ror).
template <int ROR, typename Op>
__device__ __forceinline__ float join_ror(float v, Op op) {
    const int i = __float_as_int(v);
    return op(v, __int_as_float(__builtin_amdgcn_update_dpp(i, i, 0x120 | ROR, 0xf, 0xf, false)));
}

// v joined over the lanes whose numbers differ by multiples of `apart`, a power of two:
// rotations within the rows of 16, then the rows' swaps.  No LDS, 8 cycles a step where
// a shuffle through LDS takes about 120.
template <typename Op>
__device__ __forceinline__ float join_lanes(float v, int apart, Op op) {
    if (apart <= 8) v = join_ror<8>(v, op);
    if (apart <= 4) v = join_ror<4>(v, op);
    if (apart <= 2) v = join_ror<2>(v, op);
    if (apart <= 1) v = join_ror<1>(v, op);
    if (apart <= 16) {
        const auto q = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = op(__uint_as_float(q[0]), __uint_as_float(q[1]));
    }
    const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return op(__uint_as_float(q[0]), __uint_as_float(q[1]));
}

__device__ __forceinline__ float wave_sum(float v) { return join_lanes(v, 1, Add()); }

// red[parts][cb] = the threads' values of each channel, joined over a wave's rows.
template <int VEC, typename Op>
__device__ __forceinline__ void join_rows(float (&v)[VEC], const Cut& k, float* red, Op op) {
    const int t = threadIdx.x, lane = t & 63;
    if (k.wrows) {
        if (k.wrows * k.cv == 64) {           // both powers of two
#pragma unroll
            for (int j = 0; j < VEC; ++j) v[j] = join_lanes(v[j], k.cv, op);
        } else {
            const int row = (int)fdiv(lane, k.dcv);
            for (int n = k.wrows; n > 1;) {
                const int h = (n + 1) / 2;
                const bool take = row + h < n;
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const float o = __shfl(v[j], (lane + h * k.cv) & 63);
                    if (take) v[j] = op(v[j], o);
                }
                n = h;
            }
        }
        if (lane < k.cv) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) red[(t >> 6) * k.cb + lane * VEC + j] = v[j];
        }
    } else if (t < k.rows * k.cv) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) red[t * VEC + j] = v[j];
    }
}

// red joined over the parts, for channel c.
template <typename Op>
__device__ __forceinline__ float join_parts(const Cut& k, const float* red, int c, Op op) {
    float a = red[c];
#pragma unroll 4
    for (int r = 1; r < k.parts; ++r) a = op(a, red[r * k.cb + c]);
    return a;
}

// out[g] = sum of weight(c) red[part][c] over the parts and the group's channels,
// `lanes` neighbouring lanes a group.
template <typename F>
__device__ __forceinline__ void join_groups(const Cut& k, const float* red, float* out, F weight) {
    const int n = k.parts * k.D, groups = (int)fdiv(k.cb, k.dD);
    const int bits = n >= 64 ? 6 : 32 - __builtin_clz(n | 1) - ((n & (n - 1)) == 0), lanes = 1 << bits;
    const int per = blockDim.x >> bits, sub = threadIdx.x & (lanes - 1);
    for (int g0 = 0; g0 < groups; g0 += per) {
        const int g = g0 + (threadIdx.x >> bits);
        float a = 0.0f;
        if (g < groups)
            for (int i = sub; i < n; i += lanes) {
                const int part = (int)fdiv(i, k.dD), c = g * k.D + i - part * k.D;
                a += weight(c) * red[part * k.cb + c];
            }
        if (lanes == 64) a = wave_sum(a);
        else
            for (int m = lanes >> 1; m; m >>= 1) a += __shfl_xor(a, m);
        if (g < groups && sub == 0) out[g] = a;
    }
}

template <typename T, int VEC, int NV>
__device__ __forceinline__ void pin(Held<T, VEC> (&h)[NV]) {
#pragma unroll
    for (int i = 0; i < NV; ++i) h[i].pin();
}

// A thread's sums since the last time to its totals.
template <int VEC>
__device__ __forceinline__ void flush(float (&sum)[VEC], float (&total)[VEC]) {
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
        total[j] += sum[j];
        sum[j] = 0.0f;
    }
}

// p moved on, so that the compiler does not keep the addresses of an earlier pass
// over the same pixels in registers.
template <typename T>
__device__ __forceinline__ void advance(T*& p, size_t step) {
    p += step;
    asm volatile("" : "+v"(p));
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
    bool relu;
};

// One image of whole groups: loads, three joins at most and stores in turn, so bound by
// latency where it is used (N = 8, 128 channels at 28x28: 8.6 us, of which an empty
// launch is 6.1; with the checkpoint 12).
template <typename T, int VEC, int NV, bool SILU>
__global__ __launch_bounds__(kMaxThreads) void k_norm(FwdArgs a, Cut k) {
    extern __shared__ float lds[];
    const int words = k.parts * k.cb;
    float *red = lds, *rl = red + words, *rh = rl + words, *cl = rh + words;
    float *ch = cl + k.cb, *gm = ch + k.cb, *gr = gm + k.cb;
    Item it;
    for (uint32_t vb = blockIdx.x; vb < k.per * kXcds; vb += gridDim.x) {
        if (!item_of(vb, k, &it)) continue;
        const Share s = share_of(k, it, VEC);
        const size_t at = ((size_t)it.n * k.P + s.row) * k.C + s.c, step = (size_t)k.rows * k.C;
        Held<T, VEC> raw[NV];
        const T* x = (const T*)a.x + at;
#pragma unroll
        for (int i = 0; i < NV; ++i, advance(x, step))
            if (i < s.count) raw[i].load(x);
        const bool norm = a.y || a.stats;
        float mean[VEC], v[VEC];              // mean: first the group's first value, which the sums are about
        if (norm) {
            const T* group = (const T*)a.x + (size_t)it.n * k.P * k.C + it.c0;
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                mean[j] = (float)group[fdiv(s.col * VEC + j, k.dD) * k.D];
                v[j] = 0.0f;
            }
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (i < s.count)
#pragma unroll
                    for (int j = 0; j < VEC; ++j) v[j] += raw[i].value(j) - mean[j];
            join_rows(v, k, red, Add());
        }
        if (a.codes) {
            pin(raw);
            float hi[VEC];
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                v[j] = Low::identity;
                hi[j] = High::identity;
            }
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (i < s.count)
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        v[j] = Low()(raw[i].value(j), v[j]);
                        hi[j] = High()(raw[i].value(j), hi[j]);
                    }
            join_rows(v, k, rl, Low());
            join_rows(hi, k, rh, High());
        }
        __syncthreads();
        if (a.codes)
            for (int c = threadIdx.x; c < k.cb; c += blockDim.x) {
                const Row r = row_of(join_parts(k, rl, c, Low()), join_parts(k, rh, c, High()));
                cl[c] = r.centre;
                ch[c] = r.inverse;
                float* p = a.rows + ((size_t)it.n * k.C + it.c0 + c) * 2;
                p[0] = r.centre;
                p[1] = r.step;
            }
        if (norm) join_groups(k, red, gm, [&](int) { return k.inv; });
        __syncthreads();
        if (norm) {
            pin(raw);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                mean[j] += gm[fdiv(s.col * VEC + j, k.dD)];
                v[j] = 0.0f;
            }
            if (a.stats && s.row == 0)
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const int g = (int)fdiv(s.col * VEC + j, k.dD);
                    if (s.col * VEC + j == g * k.D) a.stats[((size_t)it.n * k.G + fdiv(it.c0, k.dD) + g) * 2] = mean[j];
                }
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (i < s.count)
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        const float d = raw[i].value(j) - mean[j];
                        v[j] = fmaf(d, d, v[j]);
                    }
            join_rows(v, k, red, Add());
            __syncthreads();
            join_groups(k, red, gr, [&](int) { return k.inv; });
            __syncthreads();
            if (a.stats)
                for (int g = threadIdx.x; g < (int)fdiv(k.cb, k.dD); g += blockDim.x)
                    a.stats[((size_t)it.n * k.G + fdiv(it.c0, k.dD) + g) * 2 + 1] = rstd_of(gr[g], a.eps);
        }
        if (a.codes) {
            pin(raw);
            float centre[VEC], inverse[VEC];
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                centre[j] = cl[s.col * VEC + j];
                inverse[j] = ch[s.col * VEC + j];
            }
            int8_t* codes = a.codes + at;
#pragma unroll
            for (int i = 0; i < NV; ++i, advance(codes, step))
                if (i < s.count) {
                    uint32_t q[VEC];
#pragma unroll
                    for (int j = 0; j < VEC; ++j) q[j] = code_bits(raw[i].value(j), centre[j], inverse[j]);
                    store_codes(codes, q);
                }
        }
        if (a.y) {
            pin(raw);
            Norm<SILU, false> f[VEC];
            if (s.count)
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const float st[2] = {mean[j], rstd_of(gr[fdiv(s.col * VEC + j, k.dD)], a.eps)};
                    f[j].set(st, a.gamma ? a.gamma[s.c + j] : 1.0f, a.beta ? a.beta[s.c + j] : 0.0f, nullptr);
                }
            T* y = (T*)a.y + at;
#pragma unroll
            for (int i = 0; i < NV; ++i, advance(y, step))
                if (i < s.count) {
                    Raw<T, VEC> o;
#pragma unroll
                    for (int j = 0; j < VEC; ++j) o.v[j] = (T)act_of<SILU>(f[j].z(f[j].n(raw[i].value(j))), a.relu);
                    put(y, o);
                }
        }
        __syncthreads();                      // the next item writes the LDS arrays
    }
}

// The parts of the statistics of a chunk of an image.  A thread's sums are about its
// mean so far, at first its first value, and join its mean and squares kFlush values at a
// time: a mean far from zero costs nothing, and a first value far from the others no more
// than in one such part (all of 4096 values about it: 12% of the variance).  Threads are
// joined as means, about the chunk's first value, and squares about the chunk's mean.
// Bound by memory: 411 MB (N = 32, 64 channels at 224x224, fp32) in 72 us, 5.7 TB/s.
template <typename T, int VEC, bool CODES>
__global__ __launch_bounds__(256) void k_norm_part(FwdArgs a, Cut k) {
    constexpr int U = VEC == 1 ? 16 : 8;      // loads in flight
    extern __shared__ float lds[];
    const int words = k.parts * k.cb;
    float *red = lds, *rl = red + words, *rh = rl + words, *cm = rh + words, *cr = cm + k.cb;
    Item it;
    for (uint32_t vb = blockIdx.x; vb < k.per * kXcds; vb += gridDim.x) {
        if (!item_of(vb, k, &it)) continue;
        const Share s = share_of(k, it, VEC);
        const size_t step = (size_t)k.rows * k.C;
        const T* x = (const T*)a.x + ((size_t)it.n * k.P + it.p0 + s.row) * k.C + s.c;
        float first[VEC], off[VEC], m2[VEC], s1[VEC], s2[VEC], lo[VEC], hi[VEC];
        Held<T, VEC> raw[U], ref;
        if (s.count) {
            raw[0].load(x);
            ref.load(x - (size_t)s.row * k.C);
        }
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            first[j] = s.count ? raw[0].value(j) : 0.0f;
            off[j] = m2[j] = s1[j] = s2[j] = 0.0f;
            lo[j] = Low::identity;
            hi[j] = High::identity;
        }
        auto take = [&](const Held<T, VEC>& r) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float v = r.value(j), d = v - first[j] - off[j];
                s1[j] += d;
                s2[j] = fmaf(d, d, s2[j]);
                if constexpr (CODES) {
                    lo[j] = Low()(v, lo[j]);
                    hi[j] = High()(v, hi[j]);
                }
            }
        };
        static_assert(kFlush % U == 0, "whole batches of loads");
        for (int i = 0; i < s.count;) {
            const int before = i, end = i + kFlush < s.count ? i + kFlush : s.count;
            for (; i + U <= end; i += U) {
#pragma unroll
                for (int u = 0; u < U; ++u, x += step) raw[u].load(x);
#pragma unroll
                for (int u = 0; u < U; ++u) take(raw[u]);
            }
            for (; i < end; ++i, x += step) {
                raw[0].load(x);
                take(raw[0]);
            }
            // the mean moves by the part's share of its distance d
            const float now = (float)(end - before), share = now / (float)end;
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float d = s1[j] / now;
                off[j] = fmaf(d, share, off[j]);
                m2[j] += s2[j] - s1[j] * d + d * d * ((float)before * share);
                s1[j] = s2[j] = 0.0f;
            }
        }
        const float n = (float)s.count;
        float mean[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            mean[j] = first[j] + off[j];
            s2[j] = m2[j];
            const float r = s.count ? ref.value(j) : 0.0f;
            s1[j] = n * (mean[j] - r);
            if (s.row == 0) cr[s.col * VEC + j] = r;
        }
        join_rows(s1, k, red, Add());
        if (CODES) {
            join_rows(lo, k, rl, Low());
            join_rows(hi, k, rh, High());
        }
        __syncthreads();
        for (int c = threadIdx.x; c < k.cb; c += blockDim.x) cm[c] = cr[c] + join_parts(k, red, c, Add()) / (float)it.px;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            const float d = mean[j] - cm[s.col * VEC + j];
            s2[j] = s.count ? fmaf(n * d, d, s2[j]) : 0.0f;
        }
        join_rows(s2, k, red, Add());
        __syncthreads();
        for (int c = threadIdx.x; c < k.cb && it.c0 + c < k.C; c += blockDim.x) {
            Raw<float, 4> o;
            o.v[0] = cm[c];
            o.v[1] = join_parts(k, red, c, Add());
            o.v[2] = CODES ? join_parts(k, rl, c, Low()) : 0.0f;
            o.v[3] = CODES ? join_parts(k, rh, c, High()) : 0.0f;
            *(Raw<float, 4>*)(a.part + (((size_t)it.n * k.chunks + it.chunk) * k.C + it.c0 + c) * 4) = o;
        }
        __syncthreads();
    }
}

// Joins the parts of one image and group: mean and variance about it, and each
// channel's row.  A workgroup an (image, group).
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
        auto total = [&](auto value) {
            double sum = 0.0;
            for (int64_t i = threadIdx.x; i < all; i += 256) {
                const int64_t ch = i / k.D, d = i - ch * k.D;
                const int64_t px = k.P - ch * k.px < k.px ? k.P - ch * k.px : k.px;
                sum += value(p + ((size_t)ch * k.C + d) * 4, (float)px);
            }
            const float a = wave_sum((float)sum);
            __syncthreads();
            if (lane == 0) acc[wave] = a;
            __syncthreads();
            return acc[0] + acc[1] + acc[2] + acc[3];
        };
        if (stats) {
            const float ref = p[0], mean = ref + total([&](const float* q, float px) { return (q[0] - ref) * px; }) * k.inv;
            const float var = total([&](const float* q, float px) {
                const float d = q[0] - mean;
                return q[1] + px * d * d;
            }) * k.inv;
            if (threadIdx.x == 0) {
                stats[((size_t)n * k.G + g) * 2] = mean;
                stats[((size_t)n * k.G + g) * 2 + 1] = rstd_of(var, eps);
            }
        }
        if (rows)
            for (int d = wave; d < k.D; d += 4) {
                float lo = Low::identity, hi = High::identity;
                for (int ch = lane; ch < (int)k.chunks; ch += 64) {
                    const float* q = p + ((size_t)ch * k.C + d) * 4;
                    lo = Low()(q[2], lo);
                    hi = High()(q[3], hi);
                }
#pragma unroll
                for (int m = 32; m; m >>= 1) {
                    lo = Low()(lo, __shfl_xor(lo, m));
                    hi = High()(hi, __shfl_xor(hi, m));
                }
                if (lane == 0) {
                    const Row r = row_of(lo, hi);
                    const size_t c = (size_t)n * k.C + (size_t)g * k.D + d;
                    rows[c * 2] = r.centre;
                    rows[c * 2 + 1] = r.step;
                    inverse[c] = r.inverse;
                }
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
    bool relu;
};

// The second pass: y (and the codes) from x or codes and the statistics.  Bound by
// memory: 822 MB of the same tensor in 121 us, 6.8 TB/s.
template <typename T, int VEC, bool X8, bool SILU>
__global__ __launch_bounds__(256) void k_norm_apply(ApplyArgs a, Cut k) {
    constexpr int U = VEC == 1 ? 8 : 4;       // loads in flight
    typedef typename std::conditional<X8, int8_t, T>::type S;
    Item it;
    for (uint32_t vb = blockIdx.x; vb < k.per * kXcds; vb += gridDim.x) {
        if (!item_of(vb, k, &it)) continue;
        const Share s = share_of(k, it, VEC);
        if (!s.count) continue;
        size_t at = ((size_t)it.n * k.P + it.p0 + s.row) * k.C + s.c;
        const size_t step = (size_t)k.rows * k.C;
        const S* src = X8 ? (const S*)a.codes : (const S*)a.x;
        Norm<SILU, X8> f[VEC];
        float centre[VEC], inverse[VEC], stp[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            const int c = s.c + j;
            const float* row = a.rows + ((size_t)it.n * k.C + c) * 2;
            if (a.stats)
                f[j].set(a.stats + ((size_t)it.n * k.G + fdiv(c, k.dD)) * 2, a.gamma ? a.gamma[c] : 1.0f,
                         a.beta ? a.beta[c] : 0.0f, row);
            centre[j] = X8 || a.out ? row[0] : 0.0f;
            stp[j] = X8 ? row[1] : 1.0f;
            inverse[j] = a.out ? a.inverse[(size_t)it.n * k.C + c] : 0.0f;
        }
        auto give = [&](const Held<S, VEC>& r, size_t at) {
            if (a.y) {
                Raw<T, VEC> o;
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const float v = r.value(j);
                    o.v[j] = (T)(a.stats ? act_of<SILU>(f[j].z(f[j].n(v)), a.relu)
                                 : X8    ? value_of(v, centre[j], stp[j])
                                         : v);
                }
                put((T*)a.y + at, o);
            }
            if (!X8 && a.out) {
                uint32_t q[VEC];
#pragma unroll
                for (int j = 0; j < VEC; ++j) q[j] = code_bits(r.value(j), centre[j], inverse[j]);
                store_codes(a.out + at, q);
            }
        };
        Held<S, VEC> raw[U];
        int i = 0;
        for (; i + U <= s.count; i += U, at += U * step) {
#pragma unroll
            for (int u = 0; u < U; ++u) raw[u].get(src + at + u * step);
#pragma unroll
            for (int u = 0; u < U; ++u) give(raw[u], at + u * step);
        }
        for (; i < s.count; ++i, at += step) {
            raw[0].get(src + at);
            give(raw[0], at);
        }
    }
}

// ------------------------------------------------------------------ backward

struct BwdArgs {
    const void *dy, *x;
    const int8_t* codes;
    const float *rows, *stats, *gamma, *beta;
    void* dx;
    float* part;                              // [N][chunks][C][2] of sum dz, sum dz n
    float* means;                             // [N][G][2] of m1, m2 (not of k_norm_back)
    bool relu;
};

template <int VEC, bool SILU, bool X8>
__device__ __forceinline__ void set_norm(Norm<SILU, X8> (&f)[VEC], const BwdArgs& a, const Cut& k, int64_t n, int c0) {
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
        const int c = c0 + j;
        f[j].set(a.stats + ((size_t)n * k.G + fdiv(c, k.dD)) * 2, a.gamma ? a.gamma[c] : 1.0f,
                 a.beta ? a.beta[c] : 0.0f, X8 ? a.rows + ((size_t)n * k.C + c) * 2 : nullptr);
    }
}

// dx = dz scale + n slope + shift
struct Grad {
    float scale, slope, shift;
    __device__ __forceinline__ void set(float rstd, float gamma, float m1, float m2) {
        scale = rstd * gamma;
        slope = -rstd * m2;
        shift = -rstd * m1;
    }
    __device__ __forceinline__ float operator()(float dz, float n) const { return fmaf(dz, scale, fmaf(n, slope, shift)); }
};

// One image of whole groups: dy and x are loaded once, and dz takes dy's registers
// (the activation's gradient is not computed twice).  N = 8, 128 channels at 28x28:
// 9 us, N = 32, 512 at 14x14 from the checkpoint 11.
template <typename T, int VEC, int NV, bool X8, bool SILU>
__global__ __launch_bounds__(kMaxThreads) void k_norm_back(BwdArgs a, Cut k) {
    extern __shared__ float lds[];
    typedef typename std::conditional<X8, int8_t, T>::type S;
    const int words = k.parts * k.cb;
    float *rz = lds, *rn = rz + words, *g1 = rn + words, *g2 = g1 + k.cb;
    Item it;
    for (uint32_t vb = blockIdx.x; vb < k.per * kXcds; vb += gridDim.x) {
        if (!item_of(vb, k, &it)) continue;
        const Share s = share_of(k, it, VEC);
        const size_t at = ((size_t)it.n * k.P + s.row) * k.C + s.c, step = (size_t)k.rows * k.C;
        const S* src = (X8 ? (const S*)a.codes : (const S*)a.x) + at;
        const T* grad = (const T*)a.dy + at;
        Held<float, VEC> dz[NV];              // dy as loaded, in the first words, then dz
        Held<S, VEC> x[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i, advance(src, step), advance(grad, step))
            if (i < s.count) {
                x[i].load(src);
                Held<T, VEC> dy;
                dy.load(grad);
#pragma unroll
                for (int w = 0; w < Held<T, VEC>::kWords; ++w) dz[i].w[w] = dy.w[w];
            }
        Norm<SILU, X8> f[VEC];
        float sz[VEC], sn[VEC];
        if (s.count) set_norm<VEC, SILU, X8>(f, a, k, it.n, s.c);
#pragma unroll
        for (int j = 0; j < VEC; ++j) sz[j] = sn[j] = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (i < s.count) {
                Held<T, VEC> dy;
#pragma unroll
                for (int w = 0; w < Held<T, VEC>::kWords; ++w) dy.w[w] = dz[i].w[w];
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const float n = f[j].n(x[i].value(j)), d = act_grad<SILU>(f[j].z(n), dy.value(j), a.relu);
                    dz[i].w[j] = __float_as_uint(d);
                    sz[j] += d;
                    sn[j] = fmaf(d, n, sn[j]);
                }
                dz[i].pin();
                x[i].pin();
            }
        join_rows(sz, k, rz, Add());
        join_rows(sn, k, rn, Add());
        __syncthreads();
        for (int c = threadIdx.x; c < k.cb; c += blockDim.x) {
            Raw<float, 2> o;
            o.v[0] = join_parts(k, rz, c, Add());
            o.v[1] = join_parts(k, rn, c, Add());
            *(Raw<float, 2>*)(a.part + ((size_t)it.n * k.C + it.c0 + c) * 2) = o;
        }
        auto weight = [&](int c) { return a.gamma ? a.gamma[it.c0 + c] * k.inv : k.inv; };
        join_groups(k, rz, g1, weight);
        join_groups(k, rn, g2, weight);
        __syncthreads();
        pin(x);
        Grad h[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            const int g = (int)fdiv(s.col * VEC + j, k.dD);
            h[j].set(f[j].rstd, f[j].gamma, g1[g], g2[g]);
        }
        T* dx = (T*)a.dx + at;
#pragma unroll
        for (int i = 0; i < NV; ++i, advance(dx, step))
            if (i < s.count) {
                Raw<T, VEC> o;
#pragma unroll
                for (int j = 0; j < VEC; ++j) o.v[j] = (T)h[j](dz[i].value(j), f[j].n(x[i].value(j)));
                put(dx, o);
            }
        __syncthreads();
    }
}

// The parts of the sums of a chunk of an image.  Bound by memory and, in 16 bits, by
// SiLU's exponential and reciprocal too: 514 MB (N = 32, 64 channels at 224x224, fp32
// dy and codes) in 93 us, 5.5 TB/s; 206 MB (N = 64, 256 at 56x56, bf16) in 41, 5.0.
template <typename T, int VEC, bool X8, bool SILU>
__global__ __launch_bounds__(256) void k_norm_back_part(BwdArgs a, Cut k) {
    constexpr int U = VEC == 1 ? 8 : 4;
    extern __shared__ float lds[];
    typedef typename std::conditional<X8, int8_t, T>::type S;
    float *rz = lds, *rn = rz + k.parts * k.cb;
    Item it;
    for (uint32_t vb = blockIdx.x; vb < k.per * kXcds; vb += gridDim.x) {
        if (!item_of(vb, k, &it)) continue;
        const Share s = share_of(k, it, VEC);
        size_t at = ((size_t)it.n * k.P + it.p0 + s.row) * k.C + s.c;
        const size_t step = (size_t)k.rows * k.C;
        const S* src = X8 ? (const S*)a.codes : (const S*)a.x;
        Norm<SILU, X8> f[VEC];
        float sz[VEC], sn[VEC];
        if (s.count) set_norm<VEC, SILU, X8>(f, a, k, it.n, s.c);
#pragma unroll
        for (int j = 0; j < VEC; ++j) sz[j] = sn[j] = 0.0f;
        auto take = [&](const Held<S, VEC>& x, const Held<T, VEC>& dy) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float n = f[j].n(x.value(j));
                const float dz = act_grad<SILU>(f[j].z(n), dy.value(j), a.relu);
                sz[j] += dz;
                sn[j] = fmaf(dz, n, sn[j]);
            }
        };
        Held<S, VEC> x[U];
        Held<T, VEC> dy[U];
        float tz[VEC], tn[VEC];               // totals
#pragma unroll
        for (int j = 0; j < VEC; ++j) tz[j] = tn[j] = 0.0f;
        static_assert(kFlush % U == 0, "whole batches of loads");
        for (int i = 0; i < s.count;) {
            const int end = i + kFlush < s.count ? i + kFlush : s.count;
            for (; i + U <= end; i += U, at += U * step) {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    x[u].load(src + at + u * step);
                    dy[u].load((const T*)a.dy + at + u * step);
                }
#pragma unroll
                for (int u = 0; u < U; ++u) take(x[u], dy[u]);
            }
            for (; i < end; ++i, at += step) {
                x[0].load(src + at);
                dy[0].load((const T*)a.dy + at);
                take(x[0], dy[0]);
            }
            flush(sz, tz);
            flush(sn, tn);
        }
        join_rows(tz, k, rz, Add());
        join_rows(tn, k, rn, Add());
        __syncthreads();
        for (int c = threadIdx.x; c < k.cb && it.c0 + c < k.C; c += blockDim.x) {
            Raw<float, 2> o;
            o.v[0] = join_parts(k, rz, c, Add());
            o.v[1] = join_parts(k, rn, c, Add());
            *(Raw<float, 2>*)(a.part + (((size_t)it.n * k.chunks + it.chunk) * k.C + it.c0 + c) * 2) = o;
        }
        __syncthreads();
    }
}

// Joins the chunks' parts of one image and group: sums[n][c] of dz and dz n, and
// means[n][g] = m1, m2.  A workgroup an (image, group).
__global__ __launch_bounds__(256) void k_norm_back_join(const float* __restrict__ part, const float* __restrict__ gamma,
                                                        float* __restrict__ sums, float* __restrict__ means, Cut k,
                                                        int64_t groups) {
    __shared__ float acc[8], red[2][256];
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    // columns of channels, and threads along the chunks
    int wide = 1;
    while (wide < 256 && wide < k.D) wide *= 2;
    const int col = t & (wide - 1), row = t / wide, rows = 256 / wide;
    for (int64_t ng = blockIdx.x; ng < groups; ng += gridDim.x) {
        const int64_t n = ng / k.G;
        const int g = (int)(ng - n * k.G);
        const float* p = part + ((size_t)n * k.chunks * k.C + (size_t)g * k.D) * 2;
        double s1 = 0.0, s2 = 0.0;
        for (int d0 = 0; d0 < k.D; d0 += wide) {
            const int d = d0 + col;
            double z = 0.0, v = 0.0;
            if (d < k.D)
                for (int ch = row; ch < (int)k.chunks; ch += rows) {
                    const float* q = p + ((size_t)ch * k.C + d) * 2;
                    z += q[0];
                    v += q[1];
                }
            __syncthreads();
            red[0][t] = (float)z;
            red[1][t] = (float)v;
            __syncthreads();
            if (t < wide && d < k.D) {
                for (int r = 1; r < rows; ++r) {
                    z += red[0][r * wide + t];
                    v += red[1][r * wide + t];
                }
                float* o = sums + ((size_t)n * k.C + (size_t)g * k.D + d) * 2;
                o[0] = (float)z;
                o[1] = (float)v;
                const float w = gamma ? gamma[(size_t)g * k.D + d] * k.inv : k.inv;
                s1 += z * w;
                s2 += v * w;
            }
        }
        const float m1 = wave_sum((float)s1), m2 = wave_sum((float)s2);
        if (lane == 0) {
            acc[wave * 2] = m1;
            acc[wave * 2 + 1] = m2;
        }
        __syncthreads();
        if (t < 2) means[((size_t)n * k.G + g) * 2 + t] = acc[t] + acc[t + 2] + acc[t + 4] + acc[t + 6];
        __syncthreads();
    }
}

// The second pass: dx.  925 MB of the first of these tensors in 148 us, 6.3 TB/s.
template <typename T, int VEC, bool X8, bool SILU>
__global__ __launch_bounds__(256) void k_norm_back_apply(BwdArgs a, Cut k) {
    constexpr int U = VEC == 1 ? 8 : 4;
    typedef typename std::conditional<X8, int8_t, T>::type S;
    Item it;
    for (uint32_t vb = blockIdx.x; vb < k.per * kXcds; vb += gridDim.x) {
        if (!item_of(vb, k, &it)) continue;
        const Share s = share_of(k, it, VEC);
        if (!s.count) continue;
        size_t at = ((size_t)it.n * k.P + it.p0 + s.row) * k.C + s.c;
        const size_t step = (size_t)k.rows * k.C;
        const S* src = X8 ? (const S*)a.codes : (const S*)a.x;
        Norm<SILU, X8> f[VEC];
        Grad h[VEC];
        set_norm<VEC, SILU, X8>(f, a, k, it.n, s.c);
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            const float* m = a.means + ((size_t)it.n * k.G + fdiv(s.c + j, k.dD)) * 2;
            h[j].set(f[j].rstd, f[j].gamma, m[0], m[1]);
        }
        auto give = [&](const Held<S, VEC>& x, const Held<T, VEC>& dy, size_t at) {
            Raw<T, VEC> o;
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float n = f[j].n(x.value(j));
                o.v[j] = (T)h[j](act_grad<SILU>(f[j].z(n), dy.value(j), a.relu), n);
            }
            put((T*)a.dx + at, o);
        };
        Held<S, VEC> x[U];
        Held<T, VEC> dy[U];
        int i = 0;
        for (; i + U <= s.count; i += U, at += U * step) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                x[u].get(src + at + u * step);
                dy[u].get((const T*)a.dy + at + u * step);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) give(x[u], dy[u], at + u * step);
        }
        for (; i < s.count; ++i, at += step) {
            x[0].get(src + at);
            dy[0].get((const T*)a.dy + at);
            give(x[0], dy[0], at);
        }
    }
}

// dgamma, dbeta: every image's sums, 32 channels a workgroup at a time.
__global__ __launch_bounds__(256) void k_norm_params(const float* __restrict__ sums, float* __restrict__ dgamma,
                                                     float* __restrict__ dbeta, int N, int C) {
    __shared__ double acc[2][8][32];
    const int lane = threadIdx.x & 31, row = threadIdx.x >> 5;
    for (int c0 = blockIdx.x * 32; c0 < C; c0 += gridDim.x * 32) {
        const int c = c0 + lane;
        double z = 0.0, n = 0.0;
        if (c < C) {
            int i = row;
            for (; i + 24 < N; i += 32) {     // four loads in flight
                Raw<float, 2> p[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) p[u] = *(const Raw<float, 2>*)(sums + ((size_t)(i + u * 8) * C + c) * 2);
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    z += p[u].v[0];
                    n += p[u].v[1];
                }
            }
            for (; i < N; i += 8) {
                const Raw<float, 2> p = *(const Raw<float, 2>*)(sums + ((size_t)i * C + c) * 2);
                z += p.v[0];
                n += p.v[1];
            }
        }
        acc[0][row][lane] = z;
        acc[1][row][lane] = n;
        __syncthreads();
        if (row == 0 && c < C) {
            for (int r = 1; r < 8; ++r) {
                z += acc[0][r][lane];
                n += acc[1][r][lane];
            }
            if (dbeta) dbeta[c] = (float)z;
            if (dgamma) dgamma[c] = (float)n;
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------ host

int vector_of(const NormShape& s, bool aligned) { return aligned && s.C % 4 == 0 ? 4 : 1; }
int64_t gcd(int64_t a, int64_t b) { return b ? gcd(b, a % b) : a; }

int64_t items_of(const NormShape& s, const NormPlan& p) {
    return (int64_t)s.N * p.chunks * ((s.C + p.cb - 1) / p.cb);
}

Cut cut_of(const NormShape& s, const NormPlan& p) {
    Cut k;
    k.C = s.C; k.G = s.G; k.D = s.D;
    k.cb = p.cb; k.cv = p.cv; k.rows = p.rows; k.wrows = p.wrows; k.parts = p.parts;
    k.ncb = (uint32_t)((s.C + p.cb - 1) / p.cb);
    k.chunks = (uint32_t)p.chunks;
    k.items = (uint32_t)items_of(s, p);
    k.per = (k.items + kXcds - 1) / kXcds;
    k.P = s.P;
    k.px = p.px;
    k.dcv = make_fastdiv(p.cv);
    k.dD = make_fastdiv(s.D);
    k.dncb = make_fastdiv(k.ncb);
    k.dchunks = make_fastdiv(k.chunks);
    k.inv = 1.0f / ((float)s.P * (float)s.D);
    return k;
}

unsigned blocks_of(int64_t items) {
    const int64_t b = (items + kXcds - 1) / kXcds * kXcds;
    return (unsigned)(b < kMaxBlocks ? b : kMaxBlocks);
}

// The rows of a workgroup's threads: whole rows by wave where they leave few
// lanes idle.
void set_rows(NormPlan* p, int threads, int cv) {
    p->threads = threads;
    p->cv = cv;
    p->cb = cv * p->vec;
    p->wrows = cv <= 32 && 64 / cv * cv >= 56 ? 64 / cv : 0;
    p->rows = p->wrows ? threads / 64 * p->wrows : threads / cv;
    p->parts = p->wrows ? threads / 64 : p->rows;
}

// Chunks of least to most rows of the workgroup's threads, for about 1024
// workgroups in all (norm N = 1, 64 channels at 112x112: 13 us with 4 rows, 17 with
// 16; N = 16, 256 at 56x56: 34 with 12 to 16, 40 with 4).
void set_chunks(NormPlan* p, const NormShape& s, int64_t least, int64_t most) {
    const int64_t steps = (s.P + p->rows - 1) / p->rows, ncb = (s.C + p->cb - 1) / p->cb;
    int64_t per = steps * s.N * ncb / 1024;
    per = per < least ? least : per > most ? most : per;
    p->px = per * p->rows;
    p->chunks = (int)((s.P + p->px - 1) / p->px);
}

// The cut of the element-wise pass.
NormPlan apply_plan(const NormShape& s, bool aligned) {
    NormPlan p = {};
    p.vec = vector_of(s, aligned);
    const int cols = (s.C + p.vec - 1) / p.vec;
    set_rows(&p, 256, cols < 256 ? cols : 256);
    set_chunks(&p, s, 4, 16);
    return p;
}

// f(T, VEC, SILU) for the element type, vector width and activation.
template <typename F>
void with_type(const NormShape& s, int vec, F&& f) {
    auto act = [&](auto t, auto v) {
        if (s.act == Act::Silu) f(t, v, std::true_type());
        else f(t, v, std::false_type());
    };
    auto go = [&](auto t) {
        if (vec == 1) act(t, std::integral_constant<int, 1>());
        else act(t, std::integral_constant<int, 4>());
    };
    if (s.io == Io::F32) go(float());
    else if (s.io == Io::F16) go(_Float16());
    else go(__bf16());
}

// Vectors that a thread may hold, of x or of dy and x: up to 32 and up to 72
// registers, so that a CU has two workgroups at least.
template <int VEC>
constexpr int held(bool backward, bool many) {
    return VEC == 1 ? (many ? 64 : 16) / (backward ? 2 : 1) : backward ? (many ? 9 : 4) : (many ? 16 : 8);
}
int held_of(int vec, bool backward, bool many) { return vec == 1 ? held<1>(backward, many) : held<4>(backward, many); }

}  // namespace

NormPlan norm_plan(const NormShape& s, bool backward, bool aligned) {
    NormPlan p = {};
    p.vec = vector_of(s, aligned);
    // One pass, where whole groups' image fits a workgroup's registers, 64 bytes of a
    // pixel at least: with 32 the caches move half lines (N = 64, 256 channels at
    // 56x56: 237 us, in three launches 106), which pays only as long as the workgroups
    // are few (N = 1: 12 and 16, N = 4: 18 and 20).  N = 32, 512 channels at 14x14: 9 us
    // in one pass, 19 in three launches.
    const int64_t unit = (int64_t)s.D / gcd(s.D, p.vec) * p.vec;
    for (int64_t cb = unit; !p.one && cb <= 512 && cb <= s.C; cb += unit) {
        const bool wide = cb * io_size(s.io) >= 64 || cb == s.C;
        if (s.C % cb || cb / p.vec > kMaxThreads || (!wide && s.N * (s.C / cb) > 128)) continue;
        for (int threads = 256; threads <= kMaxThreads && !p.one; threads *= 2)
            for (int many = 0; many < 2 && !p.one && cb / p.vec <= threads; ++many) {
                set_rows(&p, threads, (int)(cb / p.vec));
                p.nv = held_of(p.vec, backward, many);
                p.one = s.P <= (int64_t)p.rows * p.nv;
            }
    }
    if (p.one) {
        p.chunks = 1;
        p.px = s.P;
    } else {
        const int cols = (s.C + p.vec - 1) / p.vec;
        set_rows(&p, 256, cols < 128 ? cols : 128);
        set_chunks(&p, s, 4, kFlush * kFlush);
    }
    p.lds = ((backward ? 2 : 3) * (size_t)p.parts + 4) * p.cb * sizeof(float);
    const size_t lists = (size_t)s.N * p.chunks * s.C, all = (size_t)s.N * s.C, groups = (size_t)s.N * s.G * 2;
    p.need = (backward ? all * 2 + (p.one ? 0 : lists * 2 + groups) : p.one ? 0 : lists * 4 + all + groups) * sizeof(float);
    p.fits = items_of(s, p) < (int64_t)1 << 30 && items_of(s, apply_plan(s, aligned)) < (int64_t)1 << 30;
    return p;
}

hipError_t launch_norm_apply(const NormApply& a, const NormShape& s, bool aligned, hipStream_t st) {
    const NormPlan p = apply_plan(s, aligned);
    const Cut k = cut_of(s, p);
    const ApplyArgs g{a.x, a.codes, a.rows, a.stats, a.gamma, a.beta, a.y, nullptr, nullptr, s.act == Act::Relu};
    with_type(s, p.vec, [&](auto t, auto vec, auto silu) {
        typedef decltype(t) T;
        if (a.codes) k_norm_apply<T, vec.value, true, silu.value><<<blocks_of(k.items), 256, 0, st>>>(g, k);
        else k_norm_apply<T, vec.value, false, silu.value><<<blocks_of(k.items), 256, 0, st>>>(g, k);
    });
    return hipGetLastError();
}

hipError_t launch_norm(const NormFwd& a, const NormShape& s, const NormPlan& p, void* ws, hipStream_t st) {
    const Cut k = cut_of(s, p);
    const bool relu = s.act == Act::Relu;
    if (p.one) {
        const FwdArgs g{a.x, a.gamma, a.beta, a.y, a.stats, a.codes, a.rows, nullptr, a.eps, relu};
        with_type(s, p.vec, [&](auto t, auto vec, auto silu) {
            typedef decltype(t) T;
            constexpr int V = vec.value;
            constexpr bool SILU = silu.value;
            const unsigned b = blocks_of(k.items);
            if (p.nv == held<V>(false, true)) k_norm<T, V, held<V>(false, true), SILU><<<b, p.threads, p.lds, st>>>(g, k);
            else k_norm<T, V, held<V>(false, false), SILU><<<b, p.threads, p.lds, st>>>(g, k);
        });
        return hipGetLastError();
    }
    const Cut kq = cut_of(s, apply_plan(s, p.vec > 1));
    const int64_t groups = (int64_t)s.N * s.G;
    float* part = (float*)ws;
    float* inverse = part + (size_t)s.N * p.chunks * s.C * 4;
    float* own = inverse + (size_t)s.N * s.C;                  // the statistics, where the caller wants none
    float* stats = a.stats ? a.stats : a.y ? own : nullptr;
    const FwdArgs g{a.x, a.gamma, a.beta, a.y, stats, a.codes, a.rows, part, a.eps, relu};
    const ApplyArgs h{a.x, nullptr, a.rows, a.y ? stats : nullptr, a.gamma, a.beta, a.y, a.codes, inverse, relu};
    hipError_t e = hipSuccess;
    with_type(s, p.vec, [&](auto t, auto vec, auto silu) {
        typedef decltype(t) T;
        if (a.codes) k_norm_part<T, vec.value, true><<<blocks_of(k.items), p.threads, p.lds, st>>>(g, k);
        else k_norm_part<T, vec.value, false><<<blocks_of(k.items), p.threads, p.lds, st>>>(g, k);
        e = hipGetLastError();
        if (e != hipSuccess) return;
        k_norm_join<<<blocks_of(groups), 256, 0, st>>>(part, stats, a.codes ? a.rows : nullptr, inverse, k, groups, a.eps);
        e = hipGetLastError();
        if (e != hipSuccess || (!a.y && !a.codes)) return;
        k_norm_apply<T, vec.value, false, silu.value><<<blocks_of(kq.items), 256, 0, st>>>(h, kq);
        e = hipGetLastError();
    });
    return e;
}

hipError_t launch_norm_backward(const NormBwd& a, const NormShape& s, const NormPlan& p, void* ws, hipStream_t st) {
    const bool x8 = a.codes != nullptr, relu = s.act == Act::Relu;
    const Cut k = cut_of(s, p);
    float* sums = (float*)ws;                                  // [N][C][2]
    float* part = p.one ? sums : sums + (size_t)s.N * s.C * 2;
    float* means = p.one ? nullptr : part + (size_t)s.N * p.chunks * s.C * 2;
    const BwdArgs g{a.dy, a.x, a.codes, a.rows, a.stats, a.gamma, a.beta, a.dx, part, means, relu};
    hipError_t e = hipSuccess;
    with_type(s, p.vec, [&](auto t, auto vec, auto silu) {
        typedef decltype(t) T;
        constexpr int V = vec.value;
        constexpr bool SILU = silu.value;
        const unsigned b = blocks_of(k.items);
        auto go = [&](auto codes) {
            constexpr bool X8 = codes.value;
            if (p.one) {
                constexpr int few = held<V>(true, false), most = held<V>(true, true);
                if (p.nv == most) k_norm_back<T, V, most, X8, SILU><<<b, p.threads, p.lds, st>>>(g, k);
                else k_norm_back<T, V, few, X8, SILU><<<b, p.threads, p.lds, st>>>(g, k);
                e = hipGetLastError();
                return;
            }
            const Cut kq = cut_of(s, apply_plan(s, V > 1));
            const int64_t groups = (int64_t)s.N * s.G;
            k_norm_back_part<T, V, X8, SILU><<<b, p.threads, p.lds, st>>>(g, k);
            e = hipGetLastError();
            if (e != hipSuccess) return;
            k_norm_back_join<<<blocks_of(groups), 256, 0, st>>>(part, a.gamma, sums, means, k, groups);
            e = hipGetLastError();
            if (e != hipSuccess) return;
            k_norm_back_apply<T, V, X8, SILU><<<blocks_of(kq.items), 256, 0, st>>>(g, kq);
            e = hipGetLastError();
        };
        if (x8) go(std::true_type());
        else go(std::false_type());
    });
    if (e != hipSuccess || (!a.dgamma && !a.dbeta)) return e;
    k_norm_params<<<blocks_of((s.C + 31) / 32), 256, 0, st>>>(sums, a.dgamma, a.dbeta, s.N, s.C);
    return hipGetLastError();
}

}  // namespace wino
