// Weight gradient of the 3x3 stride-1 layer on channel-last tensors:
//   dg[k][c][r][s] = sum over n, i, j of a[n][i + r - pad][j + s - pad][c] dy[n][i][j][k]
// with a the layer's input, read as zero outside the image: x, a checkpoint's
// values, or act(norm(either)) formed on load.
//
// Nine products over the pixels, on the 16-bit matrix cores.  Their operands have
// the summed index innermost, eight values of it a lane, while channel-last tensors
// have it outermost, and the nine taps need it shifted.  Both are met by summing over
// pixels of eight different images at once (of eight bands of rows, where the batch is
// no multiple of eight): a lane's eight values are one pixel of eight images, so every
// tap reads whole 16-byte words, only from another row or column, and the transpose
// happens in the registers that the eight loads fill.
//
// fp32 operands are held in two fp16 terms, 22 significand bits, and three of the four
// products are summed in fp32: a product is off by less than 2^-20 (2^-22 from each
// operand and from the term left out), and results of many products as near the exact
// ones as fp32 sums are (two bf16 terms, 16 bits, gave 4.5e-6 of the norm at N = 8,
// 128 -> 128, 28x28, where these give 2e-7; 1.2e-6 at N = 64, 256 -> 256, 56x56, from the
// fp32 sums of 200704 products, torch's 4.2e-6).  For fp16's range every channel of the input and every filter of dy is
// scaled by a power of two of its own, which takes the largest finite value that it
// holds to 2^14, found by a launch before: values below 2^-17 of that lose bits, in all
// less than 2^-39 of it.  dg has one channel and one filter an element, so what the others
// hold costs it nothing.  bf16 values have one term then (exact from 2^-31 of their
// filter's largest), and tensors that are both bf16 or both fp16 are multiplied as they are.
#include <math.h>

#include <type_traits>

#include "wino_device.h"
#include "wino_norm_device.h"
#include "wino_wgrad.h"

namespace wino {

namespace {

constexpr int kMost = 256;                    // blocks that look for a tensor's largest magnitudes
constexpr int kMostThreads = 1024;
constexpr int kSeg = 8;                       // images or bands that a lane sums over
constexpr uint32_t kOutside = 1u << 31;        // an offset past every image

// How the pixels are walked: segments of `hb` output rows (2^lb to an image), eight
// segments an octet, strips of columns, and in a strip row by row.
struct Walk {
    int lb, hb, strips;
    int64_t rows;                             // octets * strips * hb
    int form, slices, ctiles, ktiles;
    FastDiv dstrips, dhb;
};

struct Args {
    WgradArgs a;
    WgradShape s;
    Walk w;
    float* part;                              // [slices][9][C][K]
    uint8_t* most;                            // exponents: nx rows of the input's channels, nd of dy's filters
    int nx, nd;                               // none: not scaled
};

// 16-byte words of eight values' terms: hi, and with two terms what is left.
template <typename H, int TERMS>
__device__ __forceinline__ void split8(const float (&v)[kSeg], uint4 (&o)[TERMS]) {
    typedef H h2 __attribute__((ext_vector_type(2)));
    typedef float f2 __attribute__((ext_vector_type(2)));
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f2 x = {v[2 * i], v[2 * i + 1]};
        const h2 h = __builtin_convertvector(x, h2);
        hi[i] = __builtin_bit_cast(uint32_t, h);
        if constexpr (TERMS == 2) {
            const f2 back = __builtin_convertvector(h, f2), left = {x[0] - back[0], x[1] - back[1]};
            lo[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(left, h2));
        }
    }
    o[0] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
    if constexpr (TERMS == 2) o[1] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
}

// The power of two for a channel or filter whose largest magnitude has this biased
// exponent, which goes to 2^14, and two values' larger one: infinities and NaN do not count.
__device__ __forceinline__ int exponent_of(uint32_t biased) {
    const int e = 14 + 127 - (int)biased;
    return e > 126 ? 126 : e;
}
__device__ __forceinline__ float power(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }
__device__ __forceinline__ uint32_t larger(uint32_t m, float v) {
    const uint32_t b = __float_as_uint(v) & 0x7fffffffu;
    return b < 0x7f800000u && b > m ? b : m;
}
__host__ __device__ __forceinline__ int most_row(int channels) { return (channels + 3) / 4 * 4; }

// Four channels from c on of a row's bytes, the largest of `rows` rows, `per` apart.
struct Most4 {
    uint32_t m[4];
    __device__ __forceinline__ void load(const uint8_t* most, int rows, int channels, int c, int row, int per) {
        const int stride = most_row(channels);
        m[0] = m[1] = m[2] = m[3] = 0;
        if (c >= channels) return;
        for (int r = row; r < rows; r += 4 * per) {
            uint32_t w[4];                    // four loads in flight, of the last row again past it
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int at = r + u * per < rows ? r + u * per : rows - 1;
                w[u] = *(const uint32_t*)(most + (size_t)at * stride + c);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t e = w[u] >> (8 * j) & 0xff;
                    m[j] = e > m[j] ? e : m[j];
                }
        }
    }
    __device__ __forceinline__ void join(uint32_t* exps) const {
#pragma unroll
        for (int j = 0; j < 4; ++j) atomicMax(exps + j, m[j]);
    }
};

// One step of the walk: local row t of a strip of an octet; below the first row of
// the range only the input's row is fetched.
struct Step {
    int oct, strip, t, end;                   // rows up to `end`
    bool active;
};

// WC waves of 16 channels, by KW waves of 64 filters or KS waves of 4 columns each.
// T: the tensors' type; TA, TB: terms of the input and of dy.
template <typename T, bool X8, bool NORM, int WC, int KW, int KS>
struct Wgrad {
    static constexpr bool kAsIs = sizeof(T) == 2 && !X8 && !NORM;     // both tensors in 16 bits, unscaled
    static constexpr int TA = kAsIs ? 1 : 2, TB = sizeof(T) == 2 ? 1 : 2;
    typedef typename std::conditional<kAsIs && std::is_same<T, __bf16>::value, __bf16, _Float16>::type H;
    static constexpr int kPrec = std::is_same<H, _Float16>::value ? 1 : 2;
    static constexpr int kWaves = WC * KW * KS, kThreads = kWaves * 64;
    static constexpr int CT = 16 * WC, KT = 64 * KW, kCols = 4 * KS, kACols = kCols + 2;
    static constexpr int kAItems = kACols * CT / 64, kItems = kAItems + kCols * KT / 64;
    static constexpr int kPer = (kItems + kWaves - 1) / kWaves;       // items a wave loads
    typedef typename std::conditional<X8, int8_t, T>::type S;

    struct Lds {
        uint4 a[4][TA][kACols][CT];           // ring of input rows
        uint4 d[2][TB][kCols][KT];
        float2 f[2][kSeg][CT];                // constants by image and channel, of this octet and the next
    };

    const Args& g;
    Lds& l;
    const int wave, lane, c0, k0;
    const uint32_t in_image, in_row, dy_image, dy_row;        // bytes
    int64_t row, row1;                        // rows still to be entered
    Step next;                                // the step fetched last or next
    int first;                                // its strip's first active row
    const uint32_t *in_exps, *dy_exps;        // of the tile's channels' and filters' largest values, in LDS
    float in_scale, dy_scale;                 // of the lane's channel, lane % CT of the tile, and
    float gamma, beta;                        // filter; its channel's parameters
    // One step's loads: values as they are, and the byte of the first segment's image
    // that a lane loads.
    struct Raws {
        uint32_t v[kPer][kSeg], from[kPer];
    };
    f32x4 acc[9][4];

    __device__ __forceinline__ Wgrad(const Args& args, Lds& lds, int c, int k, int64_t r0, int64_t r1, const uint32_t* xe, const uint32_t* de)
        : g(args), l(lds), wave(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)), lane(threadIdx.x & 63), c0(c), k0(k),
          in_image((uint32_t)(args.s.H * args.s.W * args.s.C) * (uint32_t)sizeof(S)),
          in_row((uint32_t)(args.s.W * args.s.C) * (uint32_t)sizeof(S)),
          dy_image((uint32_t)(args.s.Ho * args.s.Wo * args.s.K) * (uint32_t)sizeof(T)),
          dy_row((uint32_t)(args.s.Wo * args.s.K) * (uint32_t)sizeof(T)), row(r0), row1(r1), in_exps(xe), dy_exps(de) {
        static_assert(64 % CT == 0 && KT % 64 == 0, "a lane's channel and filter are the same in all its items");
        static_assert(KT == 64 || (KT == 128 && kAItems % 2 == 0 && kWaves % 2 == 0), "and its wave's half of them");
        in_scale = kAsIs ? 1.0f : power(exponent_of(in_exps[lane % CT]));
        dy_scale = kAsIs ? 1.0f : power(exponent_of(dy_exps[(wave * 64 + lane) % KT]));
        if constexpr (NORM && !X8) {
            const int own = c0 + lane % CT;
            gamma = g.a.gamma && own < g.s.C ? g.a.gamma[own] : 1.0f;
            beta = g.a.beta && own < g.s.C ? g.a.beta[own] : 0.0f;
        }
    }

    // The steps of rows [row, row1): of each strip's share two rows more.
    __device__ __forceinline__ bool enter() {
        if (row >= row1) return false;
        const int unit = (int)fdiv((uint32_t)row, g.w.dhb), t = (int)(row - (int64_t)unit * g.w.hb);
        next.oct = (int)fdiv(unit, g.w.dstrips);
        next.strip = unit - next.oct * g.w.strips;
        next.end = row1 - row < g.w.hb - t ? t + (int)(row1 - row) : g.w.hb;
        next.t = t - 2;
        next.active = false;
        row += next.end - t;
        first = t;
        return true;
    }
    __device__ __forceinline__ bool advance() {
        if (next.t + 1 < next.end) {
            ++next.t;
            next.active = next.t >= first;
            return true;
        }
        return enter();
    }

    // The constants of an octet: mean and rstd of x; of a checkpoint, whose centre the
    // mean is subtracted from, those of z = code scale + shift.
    __device__ __forceinline__ void fill_norm(int oct) {
        if constexpr (NORM) {
            for (int i = threadIdx.x; i < kSeg * CT; i += kThreads) {
                const int e = i / CT, c = c0 + i % CT, seg = oct * kSeg + e;
                float2 f = make_float2(0.0f, 0.0f);
                if (c < g.s.C) {
                    const int n = seg >> g.w.lb;
                    const float* st = g.a.stats + ((size_t)n * g.s.G + c / g.s.D) * 2;
                    if constexpr (X8) {
                        const float* r = g.a.rows + ((size_t)n * g.s.C + c) * 2;
                        const float scale = st[1] * (g.a.gamma ? g.a.gamma[c] : 1.0f);
                        f.x = scale * r[1];
                        f.y = fmaf(r[0] - st[0], scale, g.a.beta ? g.a.beta[c] : 0.0f);
                    } else {
                        f = make_float2(st[0], st[1]);
                    }
                }
                l.f[oct & 1][e][i % CT] = f;
            }
        } else if constexpr (X8) {
            for (int i = threadIdx.x; i < kSeg * CT; i += kThreads) {
                const int e = i / CT, c = c0 + i % CT, seg = oct * kSeg + e;
                const float* r = g.a.rows + ((size_t)(seg >> g.w.lb) * g.s.C + c) * 2;
                l.f[oct & 1][e][i % CT] = c < g.s.C ? make_float2(r[1] * in_scale, r[0] * in_scale) : make_float2(0.0f, 0.0f);
            }
        }
    }

    // Byte of its own image that a lane loads for segment e: of its e mod 2^lb th band.
    __device__ __forceinline__ uint32_t byte_of(uint32_t from, int e, uint32_t row_bytes) const {
        const uint32_t band = (uint32_t)g.w.hb * row_bytes;
        const uint32_t b1 = g.w.lb >= 1 ? band : 0, b2 = g.w.lb >= 2 ? 2 * band : 0, b4 = g.w.lb >= 3 ? 4 * band : 0;
        return from + (e & 1 ? b1 : 0) + (e & 2 ? b2 : 0) + (e & 4 ? b4 : 0);
    }

    // Eight loads of one item: an image is a buffer of its own, so that rows above and
    // below it and lanes beside it (kOutside, and a band's offset) read as zero: images
    // are below 2^31 bytes, and so are the rows that are asked for outside them.  The
    // image's address goes on from segment to segment, which takes few scalar registers.
    template <typename V>
    __device__ __forceinline__ void load8(uint32_t (&r)[kSeg], const void* base, uint32_t image, uint32_t row_bytes,
                                          uint32_t at) const {
        // in scalar registers, as the compiler does not see by itself
        const int first_image = __builtin_amdgcn_readfirstlane(next.oct) * kSeg >> g.w.lb;
        const char* p = (const char*)base + (size_t)first_image * image;
        const uint32_t i1 = g.w.lb == 0 ? image : 0, i2 = g.w.lb <= 1 ? image : 0, i4 = g.w.lb <= 2 ? image : 0;
#pragma unroll
        for (int e = 0; e < kSeg; ++e) {
            if (e) {
                p += e & 1 ? i1 : e & 2 ? i2 : i4;
                asm volatile("" : "+s"(p));
            }
            const auto b = __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, (int)image, kRsrcWord3);
            const int o = (int)byte_of(at, e, row_bytes);
            if constexpr (sizeof(V) == 4) r[e] = __builtin_amdgcn_raw_buffer_load_b32(b, o, 0, 0);
            else if constexpr (sizeof(V) == 2) r[e] = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(b, o, 0, 0);
            else r[e] = (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(b, o, 0, 0);
        }
    }

    // Loads of step `next`: the input's row t + 2 of the strip's columns and one more on
    // each side, dy's row t.  A lane takes one column and channel, of the eight segments.
    // One code path for both where their elements are as wide: the compiler joins two
    // and then waits for the loads at once.
    __device__ __forceinline__ void fetch(Raws& raw) const {
#pragma unroll
        for (int p = 0; p < kPer; ++p) {
            const int item = wave + p * kWaves;
            const bool input = item < kAItems;
            if (item >= kItems || (!input && !next.active)) continue;
            const int at = (input ? item : item - kAItems) * 64 + lane;
            const int wide = input ? g.s.W : g.s.Wo, chs = input ? g.s.C : g.s.K;
            const int col = next.strip * kCols + (input ? at / CT - g.s.pad : at / KT);
            const int ch = input ? c0 + at % CT : k0 + at % KT;
            const int y = input ? next.t + 2 - g.s.pad : next.t;
            const bool inside = col >= 0 && col < wide && ch < chs;
            const uint32_t value = (uint32_t)((y * wide + col) * chs + ch);
            if constexpr (!X8) {
                const uint32_t from = inside ? value * (uint32_t)sizeof(T) : kOutside;
                raw.from[p] = from;
                load8<T>(raw.v[p], input ? g.a.x : g.a.dy, input ? in_image : dy_image, input ? in_row : dy_row, from);
            } else if (input) {
                raw.from[p] = inside ? value : kOutside;
                load8<S>(raw.v[p], g.a.codes, in_image, in_row, raw.from[p]);
            } else {
                load8<T>(raw.v[p], g.a.dy, dy_image, dy_row, inside ? value * (uint32_t)sizeof(T) : kOutside);
            }
        }
    }

    template <typename V>
    static __device__ __forceinline__ float value(uint32_t w) {
        Held<V, 1> h;
        h.w[0] = w;
        return h.value(0);
    }

    // The activation's argument: of x as the norm's own passes form it (folded constants
    // lose the bits of a mean far from zero, and take 600 us where this takes 610 at
    // N = 64, 256 -> 256, 56x56); of a code it is there already.
    template <bool SILU>
    __device__ __forceinline__ float argument(float v, float2 f) const {
        if constexpr (X8) return v;
        Norm<SILU, false> norm;
        norm.mean = f.x;
        norm.rstd = f.y;
        norm.gamma = gamma;
        norm.beta = beta;
        return norm.z(norm.n(v));
    }

    // The fetched values to LDS, in terms: `slot` of the ring, buffer slot & 1 of dy.
    __device__ __forceinline__ void store(int slot, const Step& s, const Raws& raw) {
#pragma unroll
        for (int p = 0; p < kPer; ++p) {
            const int item = wave + p * kWaves;
            const bool input = item < kAItems;
            if (item >= kItems || (!input && !s.active)) continue;
            float v[kSeg];
            if constexpr (kAsIs) {                    // the operands are the tensors' own 16 bits
                const int at = (input ? item : item - kAItems) * 64 + lane;
                uint32_t w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = raw.v[p][2 * i] | raw.v[p][2 * i + 1] << 16;
                const uint4 o = make_uint4(w[0], w[1], w[2], w[3]);
                if (input) l.a[slot & 3][0][at / CT][at % CT] = o;
                else l.d[slot & 1][0][at / KT][at % KT] = o;
            } else if (input) {
                const int at = item * 64 + lane, c = at % CT;
                if constexpr (!X8 && !NORM) {
#pragma unroll
                    for (int e = 0; e < kSeg; ++e) v[e] = value<S>(raw.v[p][e]) * in_scale;
                } else {
                    float2 f[kSeg];                   // read together
#pragma unroll
                    for (int e = 0; e < kSeg; ++e) f[e] = l.f[s.oct & 1][e][c];
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int e = 0; e < kSeg; ++e) {
                        const float stored = value<S>(raw.v[p][e]);
                        v[e] = X8 ? fmaf(stored, f[e].x, f[e].y) : stored;
                    }
                    if constexpr (NORM) {
                        if (g.s.act == Act::Silu) {
#pragma unroll
                            for (int e = 0; e < kSeg; ++e) v[e] = in_scale * act_of<true>(argument<true>(v[e], f[e]), false);
                        } else {
                            const bool relu = g.s.act == Act::Relu;
#pragma unroll
                            for (int e = 0; e < kSeg; ++e) v[e] = in_scale * act_of<false>(argument<false>(v[e], f[e]), relu);
                        }
                    }
#pragma unroll
                    for (int e = 0; e < kSeg; ++e) v[e] = byte_of(raw.from[p], e, in_row) < in_image ? v[e] : 0.0f;
                }
                uint4 o[TA];
                split8<H, TA>(v, o);
#pragma unroll
                for (int t = 0; t < TA; ++t) l.a[slot & 3][t][at / CT][c] = o[t];
            } else {
                const int at = (item - kAItems) * 64 + lane;
#pragma unroll
                for (int e = 0; e < kSeg; ++e) v[e] = value<T>(raw.v[p][e]) * dy_scale;
                uint4 o[TB];
                split8<H, TB>(v, o);
#pragma unroll
                for (int t = 0; t < TB; ++t) l.d[slot & 1][t][at / KT][at % KT] = o[t];
            }
        }
    }

    // The nine taps of step `slot`: input rows of the last three steps.
    __device__ __forceinline__ void multiply(int slot) {
        const int wc = wave % WC, wk = wave / WC, ks = KS > 1 ? wk : 0, kw = KS > 1 ? 0 : wk;
        const int col = ks * 4 + (lane >> 4), c = wc * 16 + (lane & 15);
        uint4 b[4][TB];
#pragma unroll
        for (int f = 0; f < 4; ++f)
#pragma unroll
            for (int t = 0; t < TB; ++t) b[f][t] = l.d[slot & 1][t][col][kw * 64 + f * 16 + (lane & 15)];
        uint4 a[TA];
#pragma unroll
        for (int t = 0; t < TA; ++t) a[t] = l.a[(slot + 2) & 3][t][col][c];
#pragma unroll
        for (int tap = 0; tap < 9; ++tap) {
            uint4 ahead[TA];
            if (tap < 8) {
#pragma unroll
                for (int t = 0; t < TA; ++t) ahead[t] = l.a[(slot + 2 + (tap + 1) / 3) & 3][t][col + (tap + 1) % 3][c];
            }
            __builtin_amdgcn_sched_barrier(0);        // these reads before this tap's products
#pragma unroll
            for (int p = 0; p < TA + TB - 1; ++p) {
                // hi hi, then hi lo and lo hi
                const int ta = TB == 2 ? p == 2 : p, tb = TB == 2 && p == 1;
#pragma unroll
                for (int f = 0; f < 4; ++f) acc[tap][f] = mfma16x16x32<kPrec>(b[f][tb], a[ta], acc[tap][f]);
            }
#pragma unroll
            for (int t = 0; t < TA; ++t) a[t] = ahead[t];
        }
    }

    __device__ __forceinline__ void sync() {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        wg_barrier();
    }

    __device__ __forceinline__ void run() {
        // every slice has a row, and its first strip's share three steps at least: their
        // loads together
        enter();
        fill_norm(next.oct);
        Raws raw;
        Step now = next;
        {
            Raws r0, r1;
            fetch(r0);
            const Step s0 = next;
            advance();
            fetch(r1);
            const Step s1 = next;
            advance();
            fetch(raw);
            now = next;
            sync();
            store(0, s0, r0);
            store(1, s1, r1);
        }
        store(2, now, raw);
        bool more = advance();
        Step ready = next;
        if (more) {
            if (next.oct != now.oct) fill_norm(next.oct);
            fetch(raw);
        }
        sync();
#pragma unroll
        for (int tap = 0; tap < 9; ++tap)
#pragma unroll
            for (int f = 0; f < 4; ++f) acc[tap][f] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        // half of the waves, one of each SIMD's two, convert before they multiply, so
        // that one has the matrix cores while the other has the vector units
        const bool early = wave >= kWaves / 2;
        for (int slot = 2;; ++slot) {
            const Step after = ready;
            bool fetched = false;
            auto refill = [&]() {
                if (!more) return;
                store(slot + 1, after, raw);
                fetched = advance();
                if (fetched) fetch(raw);
            };
            if (early) refill();
            if (now.active) multiply(slot);
            if (!early) refill();
            if (fetched && next.oct != after.oct) fill_norm(next.oct);
            if (!more) break;
            now = after;
            ready = next;
            more = fetched;
            sync();
        }
    }

    // acc to part: channel lane % 16 of the wave's, filters 4 (lane / 16) + i of each 16.
    __device__ __forceinline__ void finish(int slice) {
        const int wc = wave % WC, wk = wave / WC, kw = KS > 1 ? 0 : wk;
        if constexpr (KS > 1) {
            // the columns' halves joined through LDS, in order, three taps at a time
            static_assert(KS == 2 && sizeof(Lds) >= WC * 12 * 64 * sizeof(f32x4), "two halves, through Lds");
            f32x4(*red)[12][64] = (f32x4(*)[12][64])&l;
#pragma unroll
            for (int r = 0; r < 3; ++r) {
                sync();
                if (wk == 1)
#pragma unroll
                    for (int i = 0; i < 12; ++i) red[wc][i][lane] = acc[r * 3 + i / 4][i % 4];
                sync();
                if (wk == 0)
#pragma unroll
                    for (int i = 0; i < 12; ++i) acc[r * 3 + i / 4][i % 4] += red[wc][i][lane];
            }
            if (wk) return;
        }
        if constexpr (!kAsIs) {
            const int in = exponent_of(in_exps[wc * 16 + (lane & 15)]);
#pragma unroll
            for (int f = 0; f < 4; ++f)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int exponent = in + exponent_of(dy_exps[kw * 64 + f * 16 + (lane >> 4) * 4 + i]);
#pragma unroll
                    for (int tap = 0; tap < 9; ++tap) acc[tap][f][i] = ldexpf(acc[tap][f][i], -exponent);
                }
        }
        const int c = c0 + wc * 16 + (lane & 15), k = k0 + kw * 64 + (lane >> 4) * 4;
        if (c >= g.s.C) return;
        const size_t plane = (size_t)g.s.C * g.s.K;
        float* p = g.part + ((size_t)slice * 9 * g.s.C + c) * g.s.K + k;
        if (g.s.K % 4 == 0) {
#pragma unroll
            for (int tap = 0; tap < 9; ++tap, p += plane)
#pragma unroll
                for (int f = 0; f < 4; ++f)
                    if (k + f * 16 < g.s.K) *(f32x4*)(p + f * 16) = acc[tap][f];
        } else {
#pragma unroll
            for (int tap = 0; tap < 9; ++tap, p += plane)
#pragma unroll
                for (int f = 0; f < 4; ++f)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (k + f * 16 + i < g.s.K) p[f * 16 + i] = acc[tap][f][i];
        }
    }
};

// The exponents of the largest of `rows` values of each channel, value(row, channel) as
// magnitude bits: row `block` of `blocks`, a thread a channel.
template <typename F>
__device__ __forceinline__ void most_by_channel(int64_t rows, int C, int block, int blocks, uint32_t* lds, uint8_t* out,
                                                F value) {
    constexpr int threads = kMostThreads;
    const int t = threadIdx.x, wide = C < threads ? C : threads, per = threads / wide, row = t / wide;
    for (int c0 = 0; c0 < C; c0 += threads) {
        const int c = c0 + t % wide;
        uint32_t m = 0;
        if (c < C && row < per)
            for (int64_t i = (int64_t)block * per + row; i < rows; i += (int64_t)blocks * per) {
                const uint32_t v = value(i, c);
                m = v > m ? v : m;
            }
        lds[t] = 0;
        __syncthreads();
        if (c < C && row < per) atomicMax(lds + (c - c0), m);
        __syncthreads();
        if (c0 + t < C) out[c0 + t] = (uint8_t)(lds[t] >> 23);
        __syncthreads();
    }
}

// The exponents of a channel-last tensor's largest magnitudes, n values of C channels:
// row `block` of `blocks`.  16 bytes a load of whichever C: a run of C / gcd(C, V) vectors
// is whole pixels, so a thread that moves on by whole runs keeps its V channels.  (One
// value a load, each thread a channel, for tensors off 16-byte addresses and for more runs'
// vectors than threads.)  205 MB in 33 us, 6.2 TB/s.
template <typename T>
__device__ __forceinline__ void most_of(const T* p, int64_t n, int C, int block, int blocks, uint32_t* lds, uint8_t* out) {
    constexpr int V = 16 / sizeof(T), threads = kMostThreads;
    const int g = C % V == 0 ? V : C % 4 == 0 ? 4 : C % 2 == 0 ? 2 : 1;      // gcd(C, V): V is 4 or 8
    const int t = threadIdx.x, run = C / g;
    if (((uintptr_t)p & 15) || run > threads) {
        most_by_channel(n / C, C, block, blocks, lds, out, [&](int64_t i, int c) { return larger(0, (float)p[i * C + c]); });
        return;
    }
    const int per = threads / run, col = t % run, row = t / run;
    for (int c = t; c < C; c += threads) lds[c] = 0;
    __syncthreads();
    uint32_t m[V] = {};
    const int64_t all = n / V, step = (int64_t)blocks * per * run;
    if (row < per) {
        int64_t i = ((int64_t)block * per + row) * run + col;
        auto take = [&](const Held<T, V>& h) {
#pragma unroll
            for (int j = 0; j < V; ++j) m[j] = larger(m[j], h.value(j));
        };
        for (; i + 3 * step < all; i += 4 * step) {
            Held<T, V> h[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) h[u].load(p + (i + u * step) * V);
#pragma unroll
            for (int u = 0; u < 4; ++u) take(h[u]);
        }
        for (; i < all; i += step) {
            Held<T, V> h;
            h.load(p + i * V);
            take(h);
        }
#pragma unroll
        for (int j = 0, c = col * V % C; j < V; ++j, c = c + 1 < C ? c + 1 : 0) atomicMax(lds + c, m[j]);
    }
    if (block == 0 && t < n - all * V) atomicMax(lds + (all * V + t) % C, larger(0, (float)p[all * V + t]));
    __syncthreads();
    for (int c = t; c < C; c += threads) out[c] = (uint8_t)(lds[c] >> 23);
}

// The largest magnitude that a channel may have, a row for one block in nx: a raw
// tensor's own, the norm's |gamma| 2 sqrt(D H W) + |beta| (|n| is at most sqrt(D H W) for
// its own statistics; twice that for their roundings), a checkpoint's |centre| + 127 step,
// or through the norm |gamma| (|centre - mean| + 127 step) rstd + |beta|; dy's own of the
// other blocks.
template <typename T>
__global__ __launch_bounds__(kMostThreads) void k_wgrad_most(Args g) {
    __shared__ uint32_t lds[kMostThreads * 16 / sizeof(T)];
    const int b = blockIdx.x, C = g.s.C;
    uint8_t* out = g.most + (size_t)b * most_row(C);
    const float top = 0x1.fffffep127f;        // a finite bound past this is this
    if (b >= g.nx) {
        out = g.most + (size_t)g.nx * most_row(C) + (size_t)(b - g.nx) * most_row(g.s.K);
        most_of((const T*)g.a.dy, (int64_t)g.s.N * g.s.Ho * g.s.Wo * g.s.K, g.s.K, b - g.nx, g.nd, lds, out);
    } else if (g.s.x8) {
        most_by_channel(g.s.N, C, b, g.nx, lds, out, [&](int64_t n, int c) {
            const float* r = g.a.rows + ((size_t)n * C + c) * 2;
            float v = fabsf(r[0]) + kCodes * r[1];
            if (g.s.norm) {
                const float* st = g.a.stats + ((size_t)n * g.s.G + c / g.s.D) * 2;
                v = (fabsf(r[0] - st[0]) + kCodes * r[1]) * st[1] * fabsf(g.a.gamma ? g.a.gamma[c] : 1.0f) +
                    fabsf(g.a.beta ? g.a.beta[c] : 0.0f);
            }
            return larger(0, v > top ? top : v);
        });
    } else if (g.s.norm) {
        const float bound = 2.0f * sqrtf((float)g.s.D * (float)g.s.H * (float)g.s.W);
        for (int c = threadIdx.x; c < C; c += kMostThreads) {
            const float v = fabsf(g.a.gamma ? g.a.gamma[c] : 1.0f) * bound + fabsf(g.a.beta ? g.a.beta[c] : 0.0f);
            out[c] = (uint8_t)(larger(0, v > top ? top : v) >> 23);
        }
    } else {
        most_of((const T*)g.a.x, (int64_t)g.s.N * g.s.H * g.s.W * C, C, b, g.nx, lds, out);
    }
}

// A workgroup a tile of channels and filters and a slice of the rows; tiles of the
// same slice run on one XCD, so that they share its rows in L2.  144 accumulators a lane
// hold the nine taps of 16 channels by 64 filters: a step reads 18 words of the input and
// 8 of dy from LDS for 108 products, so the matrix cores bound it (N = 64, 256 -> 256 at
// 56x56 in calls in a row, less the other launches: fp32 495 to 533 us, 1.34 to 1.43
// PFLOP/s of fp16 products; formed from the checkpoint with SiLU 527 to 573, the matrix
// cores 59% busy; bf16, one product of each, 277 to 282, 0.84, bound by the loads of two
// bytes a lane; a kernel trace shows 10 to 23% more).  Small layers are a chain of steps
// of 1.3 us.
template <typename T, bool X8, bool NORM, int WC, int KW, int KS>
__global__ __launch_bounds__(WC* KW* KS * 64, WC* KW* KS / 4) void k_wgrad(Args g) {
    typedef Wgrad<T, X8, NORM, WC, KW, KS> W;
    __shared__ typename W::Lds lds;
    __shared__ uint32_t exps[W::CT + W::KT];
    const int tiles = g.w.ctiles * g.w.ktiles, per = (g.w.slices * tiles + 7) / 8;
    const int item = blockIdx.x % 8 * per + blockIdx.x / 8;
    if (item >= g.w.slices * tiles) return;
    const int slice = item / tiles, tile = item % tiles;
    const int c0 = tile % g.w.ctiles * W::CT, k0 = tile / g.w.ctiles * W::KT;
    if constexpr (!W::kAsIs) {
        // the rows' largest, all loads before the first wait; unscaled: what exponent_of takes to 0
        constexpr int ccols = W::CT / 4, kcols = W::KT / 4;
        const int t = threadIdx.x;
        Most4 in, dy;
        in.load(g.most, g.nx, g.s.C, c0 + t % ccols * 4, t / ccols, W::kThreads / ccols);
        dy.load(g.most + (size_t)g.nx * most_row(g.s.C), g.nd, g.s.K, k0 + t % kcols * 4, t / kcols, W::kThreads / kcols);
        if (t < W::CT + W::KT) exps[t] = (t < W::CT ? g.nx : g.nd) ? 0 : 14 + 127;
        __syncthreads();
        in.join(exps + t % ccols * 4);
        dy.join(exps + W::CT + t % kcols * 4);
        __syncthreads();
    }
    W w(g, lds, c0, k0, g.w.rows * slice / g.w.slices, g.w.rows * (slice + 1) / g.w.slices, exps, exps + W::CT);
    w.run();
    w.finish(slice);
}

// dg [K][C][3][3] = the slices' sum, in order: 8 channels x 32 filters x one row of
// taps a workgroup, through LDS so that reads run along the filters.
__global__ __launch_bounds__(256) void k_wgrad_sum(const float* __restrict__ part, float* __restrict__ dg, int C, int K,
                                                   int slices) {
    __shared__ float out[32][25];
    const int r = blockIdx.x % 3, tile = blockIdx.x / 3, kb = (K + 31) / 32;
    const int c0 = tile / kb * 8, k0 = tile % kb * 32, k = threadIdx.x & 31, c = threadIdx.x >> 5;
    if (c0 + c < C && k0 + k < K) {
        const size_t plane = (size_t)C * K;
        const float* p = part + r * 3 * plane + (size_t)(c0 + c) * K + k0 + k;
        float v[3] = {};
        auto add = [&](auto count) {          // slices at a time, so that their loads are in flight together
            float u[count.value][3];
#pragma unroll
            for (int i = 0; i < count.value; ++i)
#pragma unroll
                for (int t = 0; t < 3; ++t) u[i][t] = p[(i * 9 + t) * plane];
#pragma unroll
            for (int i = 0; i < count.value; ++i)
#pragma unroll
                for (int t = 0; t < 3; ++t) v[t] += u[i][t];
            p += count.value * 9 * plane;
        };
        int sl = 0;
        for (; sl + 8 <= slices; sl += 8) add(std::integral_constant<int, 8>());
        for (; sl < slices; ++sl) add(std::integral_constant<int, 1>());
#pragma unroll
        for (int t = 0; t < 3; ++t) out[k][c * 3 + t] = v[t];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 32 * 24; i += 256) {
        const int kk = i / 24, j = i % 24, cc = c0 + j / 3;
        if (k0 + kk < K && cc < C) dg[((size_t)(k0 + kk) * C + cc) * 9 + r * 3 + j % 3] = out[kk][j];
    }
}

// Three forms of a workgroup: 64 channels by 128 filters in strips of 4 columns, 64 by
// 64 in strips of 8 whose halves go to different waves, and 32 by 64 of the same.
struct Form {
    int ct, kt, cols;
};
constexpr Form kForms[3] = {{64, 128, 4}, {64, 64, 8}, {32, 64, 8}};

Walk walk_of(const WgradShape& s, int form, int slices) {
    const Form f = kForms[form];
    Walk w;
    w.form = form;
    w.lb = s.N % 8 == 0 ? 0 : s.N % 4 == 0 ? 1 : s.N % 2 == 0 ? 2 : 3;
    const int bands = 1 << w.lb;
    w.hb = (s.Ho + bands - 1) / bands;
    w.strips = (s.Wo + f.cols - 1) / f.cols;
    w.rows = ((int64_t)s.N << w.lb) / 8 * w.strips * w.hb;
    w.ctiles = (s.C + f.ct - 1) / f.ct;
    w.ktiles = (s.K + f.kt - 1) / f.kt;
    w.dstrips = make_fastdiv(w.strips);
    w.dhb = make_fastdiv(w.hb);
    w.slices = slices;
    return w;
}

// Workgroups of k_wgrad_sum.
int64_t sum_blocks(const WgradShape& s) { return (int64_t)((s.K + 31) / 32) * ((s.C + 7) / 8) * 3; }

// Products on the matrix cores that one product of the operands takes.
int products_of(const WgradShape& s) { return s.io == Io::F32 ? 3 : s.norm || s.x8 ? 2 : 1; }

// A step's time in us: the products, and forming the input, which the second and third
// form do for half as many filters (third: half the products, but no second wave on a
// SIMD to run them meanwhile).
double step_of(const WgradShape& s, int form) {
    const double products = 0.95 + 0.45 * products_of(s), formed = s.norm || s.x8 ? (form == 0 ? 0.45 : 0.9) : 0.0;
    return products * (form == 0 ? 1.0 : form == 1 ? 1.04 : 0.87) + formed;
}

// The form and number of slices of the least estimated time: 11 us for two launches,
// the first loads and the last stores; a step for every row of a slice and two for
// every strip that it enters; the slices' parts, 72 bytes a filter and channel, written
// and read at 8 TB/s.  (The launch for the scale is the same for all.)  Against every
// form at 4 to 224 slices its choice was within 6% of the best (us, with one scale a
// tensor; the channels' own add 1 to 2 to all): N = 8, 128 -> 128 at
// 28x28 31.4 (third form, 28 slices; first form 35.7 at best); N = 1, 256 -> 256 at 56x56
// 37.4 (second, 13; 36.1 at 16); N = 32, 512 -> 512 at 14x14 97.5 (second, 4; 97.3);
// N = 32, 256 -> 256 at 28x28 in bf16 59.3 (59.5).
Walk walk_of(const WgradShape& s) {
    Walk best = {};
    double least = 0.0;
    for (int form = 0; form < 3; ++form) {
        Walk w = walk_of(s, form, 1);
        const int64_t tiles = (int64_t)w.ctiles * w.ktiles, most = tiles >= 256 ? 1 : 256 / tiles;
        const double step = step_of(s, form), rounds = (double)((tiles + 255) / 256);
        auto take = [&](int64_t slices) {
            if (slices < 1 || slices > most || slices > w.rows) return;
            const double rows = (double)((w.rows + slices - 1) / slices);
            const double parts = (double)slices * s.C * s.K * 72.0 / 8e6;
            const double t = 11.0 + rounds * step * (rows + 2.0 * (1.0 + (rows - 1.0) / w.hb)) + parts;
            if (best.slices && t >= least) return;
            least = t;
            w.slices = (int)slices;
            best = w;
        };
        take(most < w.rows ? most : w.rows);
        for (int64_t r = 1; r <= 64 && r <= w.rows; r += r < 8 ? 1 : r / 4) take((w.rows + r - 1) / r);
    }
    return best;
}

// Rows of exponents, of the input and of dy: none where both tensors are multiplied as
// they are, and fp16's own dy is not scaled.
struct Scales {
    int nx, nd;
};
Scales scales_of(const WgradShape& s) {
    auto blocks = [](int64_t n) { return (int)(n > (int64_t)kMost * 8192 ? kMost : (n + 8191) / 8192); };
    Scales m = {0, 0};
    if (s.x8) m.nx = blocks((int64_t)s.N * s.C * 8);      // a value a thread
    else if (s.norm) m.nx = 1;
    else if (s.io == Io::F32) m.nx = blocks((int64_t)s.N * s.H * s.W * s.C);
    if (s.io == Io::F32 || (s.io == Io::BF16 && m.nx)) m.nd = blocks((int64_t)s.N * s.Ho * s.Wo * s.K);
    return m;
}

}  // namespace

bool wgrad_fits(const WgradShape& s) {
    // 32-bit offsets into an image, also of the rows above and below it, and counts of
    // images, rows and workgroups in 32 bits
    const int64_t high = (int64_t)s.H + 2 * (int64_t)s.pad + 16, top = (int64_t)1 << 29, count = (int64_t)1 << 27;
    if (high >= top || s.W >= top / high || s.C >= top / high / s.W || s.Wo >= top / high || s.K >= top / high / s.Wo)
        return false;
    const Walk w = walk_of(s, 2, 1);
    // a launch has fewer than 2^32 threads
    return s.N < count && w.rows < count && (int64_t)w.ctiles * w.ktiles * 512 < (int64_t)1 << 31 &&
           sum_blocks(s) * 256 < (int64_t)1 << 32;
}

size_t wgrad_workspace(const WgradShape& s) {
    const Scales m = scales_of(s);
    return (size_t)walk_of(s).slices * 9 * s.C * s.K * sizeof(float) + (size_t)m.nx * most_row(s.C) +
           (size_t)m.nd * most_row(s.K);
}

hipError_t launch_wgrad(const WgradArgs& a, const WgradShape& s, void* ws, hipStream_t st) {
    Args g{a, s, walk_of(s), (float*)ws, nullptr, 0, 0};
    g.most = (uint8_t*)(g.part + (size_t)g.w.slices * 9 * s.C * s.K);
    const Scales m = scales_of(s);
    g.nx = m.nx;
    g.nd = m.nd;
    if (g.nx + g.nd) {
        if (s.io == Io::F32) k_wgrad_most<float><<<g.nx + g.nd, kMostThreads, 0, st>>>(g);
        else if (s.io == Io::F16) k_wgrad_most<_Float16><<<g.nx + g.nd, kMostThreads, 0, st>>>(g);
        else k_wgrad_most<__bf16><<<g.nx + g.nd, kMostThreads, 0, st>>>(g);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const unsigned grid = ((unsigned)g.w.slices * g.w.ctiles * g.w.ktiles + 7) / 8 * 8;
    auto go = [&](auto t, auto x8, auto norm) {
        typedef decltype(t) T;
        if (g.w.form == 0) k_wgrad<T, x8.value, norm.value, 4, 2, 1><<<grid, 512, 0, st>>>(g);
        else if (g.w.form == 1) k_wgrad<T, x8.value, norm.value, 4, 1, 2><<<grid, 512, 0, st>>>(g);
        else k_wgrad<T, x8.value, norm.value, 2, 1, 2><<<grid, 256, 0, st>>>(g);
    };
    auto with = [&](auto t) {
        if (s.x8 && s.norm) go(t, std::true_type(), std::true_type());
        else if (s.x8) go(t, std::true_type(), std::false_type());
        else if (s.norm) go(t, std::false_type(), std::true_type());
        else go(t, std::false_type(), std::false_type());
    };
    if (s.io == Io::F32) with(float());
    else if (s.io == Io::F16) with(_Float16());
    else with(__bf16());
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    k_wgrad_sum<<<(unsigned)sum_blocks(s), 256, 0, st>>>((const float*)ws, a.dg, s.C, s.K, g.w.slices);
    return hipGetLastError();
}

}  // namespace wino
