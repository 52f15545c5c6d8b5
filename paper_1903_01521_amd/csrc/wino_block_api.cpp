// C-ABI of the attention half of a block: norm and rotation of queries and keys, cross
// attention, the gated layer.  Every check runs before the first HIP call.
#include <math.h>

#include "../../include/wino.h"
#include "wino_attn.h"
#include "wino_checks.h"
#include "wino_gated.h"
#include "wino_qknorm.h"

using namespace wino;

namespace {

constexpr int kMostD = 128;
constexpr float kLog2e = 1.44269504088896340736f;

int io_of(unsigned flags, unsigned more, Io* io) {
    const unsigned t = flags & WINO_IO_MASK;
    if (flags & ~(WINO_IO_MASK | more) || t == WINO_IO_MASK) return WINO_ERR_UNSUPPORTED;
    *io = t == 0 ? Io::F32 : t == WINO_IO_F16 ? Io::F16 : Io::BF16;
    return WINO_OK;
}

// A buffer of a call: rows of `width` bytes, `pitch` apart.  Outputs overlap nothing else.
struct Buf {
    const void* p;
    int64_t rows;
    size_t width, pitch;
    bool out;
    size_t span() const { return (size_t)(rows - 1) * pitch + width; }
};
Buf whole(const void* p, size_t bytes, bool out) { return {p, 1, bytes, bytes, out}; }

bool meet(const Buf& a, const Buf& b) {
    if (!overlap(a.p, a.span(), b.p, b.span())) return false;
    if (a.pitch != b.pitch || a.rows == 1 || b.rows == 1) return true;
    // rows of one pitch: disjoint if b's lie in the gaps of a's
    const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
    const size_t d = y >= x ? (y - x) % a.pitch : (a.pitch - (x - y) % a.pitch) % a.pitch;
    return d < a.width || d + b.width > a.pitch;
}
template <int n>
bool disjoint(const Buf (&b)[n]) {
    for (int i = 0; i < n; ++i)
        for (int j = 0; j < i; ++j)
            if (b[i].p && b[j].p && (b[i].out || b[j].out) && meet(b[i], b[j])) return false;
    return true;
}

int space(const void* ws, size_t bytes, size_t need) {
    return need && (!ws || bytes < need) ? WINO_ERR_WORKSPACE : !aligned16(ws) ? WINO_ERR_INVALID_ARG : WINO_OK;
}

// [N][L][heads][D] of tokens ld apart is in range.
bool tokens_ok(int N, int L, int heads, int D, int ld) {
    int64_t w, e;
    if (N <= 0 || L <= 0 || heads <= 0 || D <= 0 || !mul_ok(heads, D, &w) || ld < w) return false;
    return mul_ok((int64_t)N * L, ld, &e);
}
Buf tokens(const void* p, int N, int L, int heads, int D, int ld, Io io, bool out) {
    const size_t z = io_size(io);
    return {p, (int64_t)N * L, (size_t)heads * D * z, (size_t)ld * z, out};
}
Buf dense(const void* p, int N, int L, int heads, int D, Io io, bool out) {
    return whole(p, (size_t)N * L * heads * D * io_size(io), out);
}

// ---- norm of queries and keys

struct QkCall {
    QkShape s;
    QkSide t[2];
};

int make_qk(QkCall* c, const void* q, const void* k, const float* gq, const float* gk, const float* rot, const int* qpos,
            const int* kpos, int N, int Lq, int Lk, int Hq, int Hk, int D, int R, int T, int ldq, int ldk, float eps,
            unsigned flags) {
    if (!q || !(eps >= 0.0f) || !tokens_ok(N, Lq, Hq, D, ldq) || (k && !tokens_ok(N, Lk, Hk, D, ldk)))
        return WINO_ERR_INVALID_ARG;
    int64_t e;
    if (R < 0 || R > D || R % 2) return WINO_ERR_INVALID_ARG;
    if (R && (!rot || T <= 0 || !mul_ok(T, R, &e) || (!qpos && Lq > T) || (k && !kpos && Lk > T)))
        return WINO_ERR_INVALID_ARG;
    if (D > kMostD) return WINO_ERR_UNSUPPORTED;
    c->s = QkShape{N, D, R, R ? T : 0, (flags & WINO_FLAG_PAIRS) != 0, eps, R ? rot : nullptr, Io::F32};
    c->t[0] = QkSide{q, nullptr, gq, R ? qpos : nullptr, nullptr, nullptr, nullptr, Lq, Hq, ldq};
    c->t[1] = k ? QkSide{k, nullptr, gk, R ? kpos : nullptr, nullptr, nullptr, nullptr, Lk, Hk, ldk} : QkSide{};
    return io_of(flags, WINO_FLAG_PAIRS, &c->s.io);
}

size_t table_bytes(const QkShape& s) { return (size_t)s.T * s.R * sizeof(float); }

// ---- attention

int make_attn(AttnShape* s, int N, int Lq, int Lk, int Hq, int Hk, int D, int ldq, int ldk, int ldv, float scale,
              unsigned flags) {
    if (!tokens_ok(N, Lq, Hq, D, ldq) || !tokens_ok(N, Lk, Hk, D, ldk) || !tokens_ok(N, Lk, Hk, D, ldv) || Hq % Hk ||
        !(scale > 0.0f) || isinf(scale * kLog2e))           // exponents of two take the product
        return WINO_ERR_INVALID_ARG;
    if (D > kMostD) return WINO_ERR_UNSUPPORTED;
    s->N = N; s->Lq = Lq; s->Lk = Lk; s->Hq = Hq; s->Hk = Hk; s->D = D;
    s->rep = Hq / Hk;
    s->rows = (int64_t)Lq * s->rep;
    s->ldq = ldq; s->ldk = ldk; s->ldv = ldv;
    s->scale = scale;
    return io_of(flags, 0, &s->io);
}

size_t attn_need(int N, int Lq, int Lk, int Hq, int Hk, int D, unsigned flags, bool backward) {
    AttnShape s;
    int64_t wq, wk;
    if (Hq <= 0 || Hk <= 0 || D <= 0 || !mul_ok(Hq, D, &wq) || !mul_ok(Hk, D, &wk) || wq > INT32_MAX || wk > INT32_MAX)
        return (size_t)-1;
    if (make_attn(&s, N, Lq, Lk, Hq, Hk, D, (int)wq, (int)wk, (int)wk, 1.0f, flags) != WINO_OK) return (size_t)-1;
    const AttnPlan p = attn_plan(s, backward);
    return p.fits ? p.need : (size_t)-1;
}

// ---- gated layer

int make_gated(GatedShape* s, int N, int C, int H, int W, int K, unsigned flags) {
    int64_t e;
    if (N <= 0 || C <= 0 || H <= 0 || W <= 0 || K <= 0 || !mul_ok(H, W, &e) || !mul_ok(e, N, &s->M) ||
        !mul_ok(s->M, C, &e) || !mul_ok(s->M, 2 * (int64_t)K, &e) || !mul_ok(2 * (int64_t)K, C, &e))
        return WINO_ERR_INVALID_ARG;
    s->C = C; s->K = K;
    const unsigned a = flags & (WINO_FLAG_RELU | WINO_FLAG_SILU);
    if (a == (WINO_FLAG_RELU | WINO_FLAG_SILU)) return WINO_ERR_UNSUPPORTED;
    s->act = a == 0 ? Act::None : a == WINO_FLAG_RELU ? Act::Relu : Act::Silu;
    return io_of(flags, WINO_FLAG_RELU | WINO_FLAG_SILU, &s->io);
}

size_t gated_need(int N, int C, int H, int W, int K, unsigned flags, bool backward) {
    GatedShape s;
    if (make_gated(&s, N, C, H, W, K, flags) != WINO_OK) return (size_t)-1;
    const GatedPlan p = gated_plan(s, backward);
    return p.fits ? p.need : (size_t)-1;
}

}  // namespace

extern "C" {

int wino_qk_norm_nhwc(const void* q, const void* k, const float* gq, const float* gk, const float* rot, const int* qpos,
                      const int* kpos, void* yq, void* yk, int N, int Lq, int Lk, int Hq, int Hk, int D, int R, int T,
                      int ldq, int ldk, float eps, unsigned flags, void* stream) {
    QkCall c;
    if (!yq || (k && !yk)) return WINO_ERR_INVALID_ARG;
    const int st = make_qk(&c, q, k, gq, gk, rot, qpos, kpos, N, Lq, Lk, Hq, Hk, D, R, T, ldq, ldk, eps, flags);
    if (st != WINO_OK) return st;
    c.t[0].y = yq;
    if (k) c.t[1].y = yk;
    const QkPlan p = qk_plan(c.s, c.t, false);
    if (!p.fits) return WINO_ERR_UNSUPPORTED;
    const Io io = c.s.io;
    const size_t g = (size_t)D * sizeof(float);
    const Buf bufs[] = {tokens(q, N, Lq, Hq, D, ldq, io, false), tokens(k, N, Lk, Hk, D, ldk, io, false),
                        whole(gq, g, false), whole(k ? gk : nullptr, g, false), whole(c.s.rot, table_bytes(c.s), false),
                        whole(c.t[0].pos, (size_t)N * Lq * 4, false), whole(c.t[1].pos, (size_t)N * Lk * 4, false),
                        dense(yq, N, Lq, Hq, D, io, true), dense(c.t[1].y, N, Lk, Hk, D, io, true)};
    if (!disjoint(bufs)) return WINO_ERR_INVALID_ARG;
    return hip_status(launch_qk_norm(c.s, c.t, p, (hipStream_t)stream));
}

size_t wino_qk_norm_backward_workspace_bytes(int N, int Lq, int Lk, int Hq, int Hk, int D, unsigned flags) {
    QkCall c;
    int64_t wq, wk;
    const int x = 0;                                 // any tensor: only sizes count
    const bool both = Lk > 0 || Hk > 0;
    if (Hq <= 0 || D <= 0 || !mul_ok(Hq, D, &wq) || wq > INT32_MAX) return (size_t)-1;
    if (both && (Hk <= 0 || !mul_ok(Hk, D, &wk) || wk > INT32_MAX)) return (size_t)-1;
    if (make_qk(&c, &x, both ? &x : nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, N, Lq, Lk, Hq, Hk, D, 0, 0,
                (int)wq, both ? (int)wk : 0, 0.0f, flags) != WINO_OK)
        return (size_t)-1;
    const QkPlan p = qk_plan(c.s, c.t, true);
    return p.fits ? p.need : (size_t)-1;
}

int wino_qk_norm_backward_nhwc(const void* dyq, const void* dyk, const void* q, const void* k, const float* gq,
                               const float* gk, const float* rot, const int* qpos, const int* kpos, void* dq, void* dk,
                               float* dgq, float* dgk, int N, int Lq, int Lk, int Hq, int Hk, int D, int R, int T,
                               int ldq, int ldk, float eps, unsigned flags, void* workspace, size_t workspace_bytes,
                               void* stream) {
    QkCall c;
    if (!dyq || !dq || (k && (!dyk || !dk))) return WINO_ERR_INVALID_ARG;
    const int st = make_qk(&c, q, k, gq, gk, rot, qpos, kpos, N, Lq, Lk, Hq, Hk, D, R, T, ldq, ldk, eps, flags);
    if (st != WINO_OK) return st;
    c.t[0].dy = dyq; c.t[0].dx = dq; c.t[0].dgamma = dgq;
    if (k) { c.t[1].dy = dyk; c.t[1].dx = dk; c.t[1].dgamma = dgk; }
    const QkPlan p = qk_plan(c.s, c.t, true);
    if (!p.fits) return WINO_ERR_UNSUPPORTED;
    const size_t need = dgq || c.t[1].dgamma ? p.need : 0;
    const int sp = space(workspace, workspace_bytes, need);
    if (sp != WINO_OK) return sp;
    const Io io = c.s.io;
    const size_t g = (size_t)D * sizeof(float);
    const Buf bufs[] = {dense(dyq, N, Lq, Hq, D, io, false), dense(c.t[1].dy, N, Lk, Hk, D, io, false),
                        tokens(q, N, Lq, Hq, D, ldq, io, false), tokens(k, N, Lk, Hk, D, ldk, io, false),
                        whole(gq, g, false), whole(k ? gk : nullptr, g, false), whole(c.s.rot, table_bytes(c.s), false),
                        whole(c.t[0].pos, (size_t)N * Lq * 4, false), whole(c.t[1].pos, (size_t)N * Lk * 4, false),
                        tokens(dq, N, Lq, Hq, D, ldq, io, true), tokens(c.t[1].dx, N, Lk, Hk, D, ldk, io, true),
                        whole(dgq, g, true), whole(c.t[1].dgamma, g, true), whole(need ? workspace : nullptr, need, true)};
    if (!disjoint(bufs)) return WINO_ERR_INVALID_ARG;
    return hip_status(launch_qk_norm_backward(c.s, c.t, p, workspace, (hipStream_t)stream));
}

size_t wino_cross_attention_workspace_bytes(int N, int Lq, int Lk, int Hq, int Hk, int D, unsigned flags) {
    return attn_need(N, Lq, Lk, Hq, Hk, D, flags, false);
}

int wino_cross_attention_nhwc(const void* q, const void* k, const void* v, const int* klen, const unsigned char* mask,
                              void* y, float* lse, int N, int Lq, int Lk, int Hq, int Hk, int D, int ldq, int ldk,
                              int ldv, float scale, unsigned flags, void* workspace, size_t workspace_bytes,
                              void* stream) {
    if (!q || !k || !v || !y) return WINO_ERR_INVALID_ARG;
    AttnShape s;
    const int st = make_attn(&s, N, Lq, Lk, Hq, Hk, D, ldq, ldk, ldv, scale, flags);
    if (st != WINO_OK) return st;
    const AttnPlan p = attn_plan(s, false);
    if (!p.fits) return WINO_ERR_UNSUPPORTED;
    const int sp = space(workspace, workspace_bytes, p.need);
    if (sp != WINO_OK) return sp;
    const Buf bufs[] = {tokens(q, N, Lq, Hq, D, ldq, s.io, false), tokens(k, N, Lk, Hk, D, ldk, s.io, false),
                        tokens(v, N, Lk, Hk, D, ldv, s.io, false), whole(klen, (size_t)N * 4, false),
                        whole(mask, (size_t)N * Lk, false), dense(y, N, Lq, Hq, D, s.io, true),
                        whole(lse, (size_t)N * Hq * Lq * 4, true), whole(p.need ? workspace : nullptr, p.need, true)};
    if (!disjoint(bufs)) return WINO_ERR_INVALID_ARG;
    const AttnArgs a{q, k, v, klen, mask, y, lse};
    return hip_status(launch_attn(a, s, p, workspace, (hipStream_t)stream));
}

size_t wino_cross_attention_backward_workspace_bytes(int N, int Lq, int Lk, int Hq, int Hk, int D, unsigned flags) {
    return attn_need(N, Lq, Lk, Hq, Hk, D, flags, true);
}

int wino_cross_attention_backward_nhwc(const void* dy, const void* q, const void* k, const void* v, const void* y,
                                       const float* lse, const int* klen, const unsigned char* mask, void* dq, void* dk,
                                       void* dv, int N, int Lq, int Lk, int Hq, int Hk, int D, int ldq, int ldk,
                                       int ldv, float scale, unsigned flags, void* workspace, size_t workspace_bytes,
                                       void* stream) {
    if (!dy || !q || !k || !v || !y || !lse || !dq || !dk || !dv) return WINO_ERR_INVALID_ARG;
    AttnShape s;
    const int st = make_attn(&s, N, Lq, Lk, Hq, Hk, D, ldq, ldk, ldv, scale, flags);
    if (st != WINO_OK) return st;
    const AttnPlan p = attn_plan(s, true);
    if (!p.fits) return WINO_ERR_UNSUPPORTED;
    const int sp = space(workspace, workspace_bytes, p.need);
    if (sp != WINO_OK) return sp;
    const Buf bufs[] = {dense(dy, N, Lq, Hq, D, s.io, false), tokens(q, N, Lq, Hq, D, ldq, s.io, false),
                        tokens(k, N, Lk, Hk, D, ldk, s.io, false), tokens(v, N, Lk, Hk, D, ldv, s.io, false),
                        dense(y, N, Lq, Hq, D, s.io, false), whole(lse, (size_t)N * Hq * Lq * 4, false),
                        whole(klen, (size_t)N * 4, false), whole(mask, (size_t)N * Lk, false),
                        tokens(dq, N, Lq, Hq, D, ldq, s.io, true), tokens(dk, N, Lk, Hk, D, ldk, s.io, true),
                        tokens(dv, N, Lk, Hk, D, ldv, s.io, true), whole(workspace, p.need, true)};
    if (!disjoint(bufs)) return WINO_ERR_INVALID_ARG;
    const AttnBwd b{dy, q, k, v, y, lse, klen, mask, dq, dk, dv};
    return hip_status(launch_attn_backward(b, s, p, workspace, (hipStream_t)stream));
}

int wino_gated_layer_plan(int N, int C, int H, int W, int K, unsigned flags, int backward, int results[3], int parts[3]) {
    if (!results || !parts) return WINO_ERR_INVALID_ARG;
    GatedShape s;
    const int st = make_gated(&s, N, C, H, W, K, flags);
    if (st != WINO_OK) return st;
    const GatedPlan p = gated_plan(s, backward != 0);
    if (!p.fits) return WINO_ERR_UNSUPPORTED;
    results[0] = !backward && gated_few(s) ? 0 : gated_results(p.first);
    results[1] = backward ? gated_results(p.dx) : 0;
    results[2] = backward ? gated_results(p.dw) : 0;
    parts[0] = 1;
    parts[1] = backward ? p.dx_splits : 0;
    parts[2] = backward ? p.dw_splits : 0;
    return WINO_OK;
}

size_t wino_gated_layer_workspace_bytes(int N, int C, int H, int W, int K, unsigned flags) {
    return gated_need(N, C, H, W, K, flags, false);
}

int wino_gated_layer_nhwc(const void* x, const void* w, const float* bias, void* y, int N, int C, int H, int W, int K,
                          unsigned flags, void* workspace, size_t workspace_bytes, void* stream) {
    if (!x || !w || !y) return WINO_ERR_INVALID_ARG;
    GatedShape s;
    const int st = make_gated(&s, N, C, H, W, K, flags);
    if (st != WINO_OK) return st;
    const GatedPlan p = gated_plan(s, false);
    if (!p.fits) return WINO_ERR_UNSUPPORTED;
    const int sp = space(workspace, workspace_bytes, p.need);
    if (sp != WINO_OK) return sp;
    const size_t z = io_size(s.io);
    const Buf bufs[] = {whole(x, s.M * C * z, false), whole(w, (size_t)2 * K * C * z, false),
                        whole(bias, (size_t)2 * K * 4, false), whole(y, s.M * K * z, true),
                        whole(p.need ? workspace : nullptr, p.need, true)};
    if (!disjoint(bufs)) return WINO_ERR_INVALID_ARG;
    const GatedArgs a{nullptr, x, w, bias, y, nullptr, nullptr, nullptr};
    return hip_status(launch_gated(a, s, p, (hipStream_t)stream));
}

size_t wino_gated_layer_backward_workspace_bytes(int N, int C, int H, int W, int K, unsigned flags) {
    return gated_need(N, C, H, W, K, flags, true);
}

int wino_gated_layer_backward_nhwc(const void* dy, const void* x, const void* w, const float* bias, void* dx, void* dw,
                                   float* dbias, int N, int C, int H, int W, int K, unsigned flags, void* workspace,
                                   size_t workspace_bytes, void* stream) {
    if (!dy || !x || !w || (!dx && !dw && !dbias)) return WINO_ERR_INVALID_ARG;
    GatedShape s;
    const int st = make_gated(&s, N, C, H, W, K, flags);
    if (st != WINO_OK) return st;
    const GatedPlan p = gated_plan(s, true);
    if (!p.fits) return WINO_ERR_UNSUPPORTED;
    const int sp = space(workspace, workspace_bytes, p.need);
    if (sp != WINO_OK) return sp;
    const size_t z = io_size(s.io);
    const Buf bufs[] = {whole(dy, s.M * K * z, false), whole(x, s.M * C * z, false),
                        whole(w, (size_t)2 * K * C * z, false), whole(bias, (size_t)2 * K * 4, false),
                        whole(dx, s.M * C * z, true), whole(dw, (size_t)2 * K * C * z, true),
                        whole(dbias, (size_t)2 * K * 4, true), whole(workspace, p.need, true)};
    if (!disjoint(bufs)) return WINO_ERR_INVALID_ARG;
    const GatedArgs a{dy, x, w, bias, nullptr, dx, dw, dbias};
    return hip_status(launch_gated_backward(a, s, p, workspace, (hipStream_t)stream));
}

}  // extern "C"
