// Attention: plans, and the launches by element type.
#include "wino_attn_device.h"
#include "wino_checks.h"

namespace wino {

namespace {

// A launch has fewer than 2^32 threads, 256 a workgroup.
constexpr int64_t kMostItems = ((int64_t)1 << 24) - 1;
constexpr int64_t kCus = 256;

// Parts of `length` (steps of `step`, two at least a part), as many as fill the card once: a
// few workgroups past that run when the others are done, with the card to themselves (560
// in place of 480, 2 images of 1200 tokens to 900 keys, 4 heads of 64, backward: 53.4 us and 50.1).
int splits_of(int64_t fill, int64_t groups, int64_t length, int step) {
    const int64_t want = fill / groups, most = length / (2 * (int64_t)step);
    const int64_t s = want < most ? want : most;
    return s < 1 ? 1 : s > 64 ? 64 : (int)s;
}

bool all16(const AttnShape& s, std::initializer_list<const void*> ps) {
    const int z = io_size(s.io);
    if (s.D * z % 16 || (int64_t)s.ldq * z % 16 || (int64_t)s.ldk * z % 16 || (int64_t)s.ldv * z % 16) return false;
    for (const void* p : ps)
        if (!aligned16(p)) return false;
    return true;
}

hipError_t run(const AttnK& g, const AttnPlan& p, bool backward, hipStream_t st) {
    if (g.s.io == Io::F32) return attn_f32(g, p, backward, st);
    return g.s.io == Io::F16 ? attn_f16(g, p, backward, st) : attn_bf16(g, p, backward, st);
}

}  // namespace

AttnPlan attn_plan(const AttnShape& s, bool backward) {
    AttnPlan p{};
    const int64_t pairs = (int64_t)s.N * s.Hk;
    p.few = !backward && s.rows <= 32;
    const int per = p.few ? 32 : 128;
    p.rows.tiles = (s.rows + per - 1) / per;
    // workgroups a CU, by the kernels' registers (of 512 a wave has 256 where two share a SIMD):
    // 4 of 1500 tokens to 900 keys, heads of 128, bf16, backward 165 us with twice as many as fit, 92
    const bool one = s.io == Io::F32 ? backward || s.D > 48 : backward && s.D > 64;
    const int64_t fill = kCus * (p.few ? 4 : one ? 1 : 2);
    p.rows.splits = splits_of(fill, pairs * p.rows.tiles, s.Lk, 64);
    const int64_t all = pairs * s.rows;
    p.keys.tiles = (s.Lk + kOwnKeys - 1) / kOwnKeys;
    p.keys.splits = splits_of(fill, pairs * p.keys.tiles, s.rows, 64);
    // pairs are rounded up to eight; a row of a tile past 2^31 would pass 32 bits
    const int64_t eights = (pairs + 7) / 8 * 8;
    p.fits = eights * p.rows.tiles * p.rows.splits <= kMostItems && eights * p.keys.tiles * p.keys.splits <= kMostItems &&
             s.rows <= INT32_MAX - 128;
    if (!p.fits) return p;
    const bool parts = p.rows.splits > 1;
    size_t part = parts ? (size_t)p.rows.splits * all * s.D * (backward ? 8 : 4) : 0;
    if (backward) {
        p.delta = round_up((size_t)all * 4, 16) * (s.io == Io::F32 ? 3 : 2);   // delta, offset, share
        p.stat = parts ? round_up((size_t)p.rows.splits * all * 8, 16) : 0;
        const size_t keys = p.keys.splits > 1 ? (size_t)p.keys.splits * pairs * s.Lk * s.D * 8 : 0;
        part = part > keys ? part : keys;
    } else if (parts) {
        p.stat = round_up((size_t)p.rows.splits * all * 8, 16);
    }
    p.part = round_up(part, 16);
    p.need = p.delta + p.part + p.stat;
    return p;
}

hipError_t launch_attn(const AttnArgs& a, const AttnShape& s, const AttnPlan& p, void* ws, hipStream_t st) {
    AttnK g{};
    g.s = s;
    g.a = a;
    g.vec = all16(s, {a.q, a.k, a.v, a.y});
    g.rep = make_fastdiv((uint32_t)s.rep);
    g.heads = make_fastdiv((uint32_t)s.Hk);
    g.part = (float*)ws;
    g.stat = (float*)((char*)ws + p.part);
    return run(g, p, false, st);
}

hipError_t launch_attn_backward(const AttnBwd& b, const AttnShape& s, const AttnPlan& p, void* ws, hipStream_t st) {
    AttnK g{};
    g.s = s;
    g.b = b;
    g.vec = all16(s, {b.dy, b.q, b.k, b.v, b.y, b.dq, b.dk, b.dv});
    g.rep = make_fastdiv((uint32_t)s.rep);
    g.heads = make_fastdiv((uint32_t)s.Hk);
    g.delta = (float*)ws;
    const size_t each = round_up((size_t)s.N * s.Hk * s.rows * 4, 16);
    g.offset = (float*)((char*)ws + each);
    g.share = (float*)((char*)ws + 2 * each);
    g.part = (float*)((char*)ws + p.delta);
    g.stat = (float*)((char*)ws + p.delta + p.part);
    return run(g, p, true, st);
}

}  // namespace wino
