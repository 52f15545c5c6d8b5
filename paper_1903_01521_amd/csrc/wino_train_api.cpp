// C-ABI of the training calls: group norm, its backward pass, the 8-bit
// checkpoint, the weight gradient.  Every check runs before the first HIP call.
#include "../../include/wino.h"
#include "wino_checks.h"
#include "wino_norm.h"
#include "wino_wgrad.h"

using namespace wino;

namespace {

// Channel numbers are 32-bit, and a workgroup's columns run up to 1024 channels on.
constexpr int kMaxChannels = 1 << 30;

// The element type and activation of the flags, the others being `more`.
int flags_of(unsigned flags, unsigned more, Io* io, Act* act) {
    if (flags & ~(WINO_FLAG_RELU | WINO_FLAG_SILU | WINO_IO_MASK | more)) return WINO_ERR_UNSUPPORTED;
    const unsigned t = flags & WINO_IO_MASK, a = flags & (WINO_FLAG_RELU | WINO_FLAG_SILU);
    if (t == WINO_IO_MASK || a == (WINO_FLAG_RELU | WINO_FLAG_SILU)) return WINO_ERR_UNSUPPORTED;
    *io = t == 0 ? Io::F32 : t == WINO_IO_F16 ? Io::F16 : Io::BF16;
    *act = a == 0 ? Act::None : a == WINO_FLAG_RELU ? Act::Relu : Act::Silu;
    return WINO_OK;
}

int make_shape(int N, int C, int H, int W, int G, unsigned flags, unsigned more, NormShape* s) {
    if (N <= 0 || C <= 0 || H <= 0 || W <= 0 || G <= 0 || C % G) return WINO_ERR_INVALID_ARG;
    int64_t e;
    if (!mul_ok(H, W, &s->P) || !mul_ok(s->P, C, &e) || !mul_ok(e, N, &e)) return WINO_ERR_INVALID_ARG;
    if (C > kMaxChannels) return WINO_ERR_UNSUPPORTED;
    s->N = N; s->C = C; s->G = G; s->D = C / G;
    return flags_of(flags, more, &s->io, &s->act);
}

size_t tensor_bytes(const NormShape& s) { return (size_t)s.N * s.P * s.C * io_size(s.io); }

// A buffer of a call; outputs must overlap nothing else.
struct Buf {
    const void* p;
    size_t bytes;
    bool out;
};
template <int n>
bool disjoint(const Buf (&b)[n]) {
    for (int i = 0; i < n; ++i)
        for (int j = 0; j < i; ++j)
            if (b[i].p && b[j].p && (b[i].out || b[j].out) && overlap(b[i].p, b[i].bytes, b[j].p, b[j].bytes))
                return false;
    return true;
}

// The larger of what aligned and unaligned tensors need.
size_t norm_need(const NormShape& s, bool backward) {
    const NormPlan a = norm_plan(s, backward, true), b = norm_plan(s, backward, false);
    return !a.fits || !b.fits ? (size_t)-1 : a.need > b.need ? a.need : b.need;
}

int space(const void* ws, size_t bytes, size_t need) {
    return need && (!ws || bytes < need) ? WINO_ERR_WORKSPACE : !aligned16(ws) ? WINO_ERR_INVALID_ARG : WINO_OK;
}

float* rows_of(const void* q, const NormShape& s) { return (float*)((char*)q + act8_rows_at(s)); }

int make_wgrad(int N, int C, int H, int W, int K, int pad, unsigned flags, WgradShape* s) {
    if (N <= 0 || C <= 0 || H <= 0 || W <= 0 || K <= 0 || pad < 0) return WINO_ERR_INVALID_ARG;
    const int64_t Ho = (int64_t)H + 2 * (int64_t)pad - 2, Wo = (int64_t)W + 2 * (int64_t)pad - 2;
    if (Ho < 1 || Wo < 1 || Ho > INT32_MAX / 2 || Wo > INT32_MAX / 2) return WINO_ERR_INVALID_ARG;
    int64_t a, b, c;
    if (!mul_ok((int64_t)N * C, (int64_t)H * W, &a) || !mul_ok((int64_t)N * K, Ho * Wo, &b) ||
        !mul_ok((int64_t)C * K, 9 * 64, &c) || !mul_ok((int64_t)N * Ho, Wo, &c) || c > INT32_MAX)
        return WINO_ERR_INVALID_ARG;
    s->N = N; s->C = C; s->H = H; s->W = W; s->K = K; s->pad = pad; s->Ho = (int)Ho; s->Wo = (int)Wo;
    s->norm = false;
    s->x8 = (flags & WINO_FLAG_ACT8) != 0;
    s->G = s->D = 1;
    const int st = flags_of(flags, WINO_FLAG_ACT8, &s->io, &s->act);
    return st != WINO_OK ? st : wgrad_fits(*s) ? WINO_OK : WINO_ERR_UNSUPPORTED;
}

}  // namespace

extern "C" {

size_t wino_act8_bytes(int N, int C, int H, int W) {
    NormShape s;
    return make_shape(N, C, H, W, 1, 0, 0, &s) == WINO_OK ? act8_size(s) : 0;
}

size_t wino_act8_workspace_bytes(int N, int C, int H, int W, unsigned flags) {
    NormShape s;
    if (flags & ~WINO_IO_MASK || make_shape(N, C, H, W, C, flags, 0, &s) != WINO_OK) return (size_t)-1;
    return norm_need(s, false);
}

int wino_act8_pack_nhwc(const void* x, void* q, int N, int C, int H, int W, unsigned flags, void* workspace,
                        size_t workspace_bytes, void* stream) {
    if (!x || !q || ((uintptr_t)q & 15)) return WINO_ERR_INVALID_ARG;
    NormShape s;
    const int st = make_shape(N, C, H, W, C, flags, 0, &s);
    if (st != WINO_OK) return st;
    if (flags & ~WINO_IO_MASK) return WINO_ERR_UNSUPPORTED;
    const NormPlan p = norm_plan(s, false, aligned16(x));
    if (!p.fits) return WINO_ERR_UNSUPPORTED;
    const int sp = space(workspace, workspace_bytes, p.need);
    if (sp != WINO_OK) return sp;
    const Buf bufs[] = {{x, tensor_bytes(s), false}, {q, act8_size(s), true}, {workspace, p.need, true}};
    if (!disjoint(bufs)) return WINO_ERR_INVALID_ARG;
    const NormFwd a{x, nullptr, nullptr, nullptr, nullptr, (int8_t*)q, rows_of(q, s), 0.0f};
    return hip_status(launch_norm(a, s, p, workspace, (hipStream_t)stream));
}

int wino_act8_unpack_nhwc(const void* q, void* x, int N, int C, int H, int W, unsigned flags, void* stream) {
    if (!x || !q || ((uintptr_t)q & 15)) return WINO_ERR_INVALID_ARG;
    NormShape s;
    const int st = make_shape(N, C, H, W, C, flags, 0, &s);
    if (st != WINO_OK) return st;
    if (flags & ~WINO_IO_MASK) return WINO_ERR_UNSUPPORTED;
    const Buf bufs[] = {{x, tensor_bytes(s), true}, {q, act8_size(s), false}};
    if (!disjoint(bufs)) return WINO_ERR_INVALID_ARG;
    if (!norm_plan(s, false, aligned16(x)).fits) return WINO_ERR_UNSUPPORTED;
    const NormApply a{nullptr, (const int8_t*)q, rows_of(q, s), nullptr, nullptr, nullptr, x};
    return hip_status(launch_norm_apply(a, s, aligned16(x), (hipStream_t)stream));
}

size_t wino_group_norm_workspace_bytes(int N, int C, int H, int W, int G, unsigned flags) {
    NormShape s;
    return make_shape(N, C, H, W, G, flags, 0, &s) == WINO_OK ? norm_need(s, false) : (size_t)-1;
}

int wino_group_norm_nhwc(const void* x, const float* gamma, const float* beta, void* y, float* stats, void* q, int N,
                         int C, int H, int W, int G, float eps, unsigned flags, void* workspace,
                         size_t workspace_bytes, void* stream) {
    if (!x || !y || ((uintptr_t)q & 15) || !(eps >= 0.0f)) return WINO_ERR_INVALID_ARG;
    NormShape s;
    const int st = make_shape(N, C, H, W, G, flags, 0, &s);
    if (st != WINO_OK) return st;
    const NormPlan p = norm_plan(s, false, aligned16(x) && aligned16(y));
    if (!p.fits) return WINO_ERR_UNSUPPORTED;
    const int sp = space(workspace, workspace_bytes, p.need);
    if (sp != WINO_OK) return sp;
    const size_t row = (size_t)C * sizeof(float);
    const Buf bufs[] = {{x, tensor_bytes(s), false}, {gamma, row, false}, {beta, row, false}, {y, tensor_bytes(s), true},
                        {stats, (size_t)N * G * 2 * sizeof(float), true}, {q, act8_size(s), true},
                        {workspace, p.need, true}};
    if (!disjoint(bufs)) return WINO_ERR_INVALID_ARG;
    const NormFwd a{x, gamma, beta, y, stats, (int8_t*)q, q ? rows_of(q, s) : nullptr, eps};
    return hip_status(launch_norm(a, s, p, workspace, (hipStream_t)stream));
}

int wino_group_norm_apply_nhwc(const void* x, const float* stats, const float* gamma, const float* beta, void* y, int N,
                               int C, int H, int W, int G, unsigned flags, void* stream) {
    const bool x8 = (flags & WINO_FLAG_ACT8) != 0;
    if (!x || !stats || !y || (x8 && ((uintptr_t)x & 15))) return WINO_ERR_INVALID_ARG;
    NormShape s;
    const int st = make_shape(N, C, H, W, G, flags, WINO_FLAG_ACT8, &s);
    if (st != WINO_OK) return st;
    const size_t row = (size_t)C * sizeof(float);
    const Buf bufs[] = {{x, x8 ? act8_size(s) : tensor_bytes(s), false}, {gamma, row, false}, {beta, row, false},
                        {stats, (size_t)N * G * 2 * sizeof(float), false}, {y, tensor_bytes(s), true}};
    if (!disjoint(bufs)) return WINO_ERR_INVALID_ARG;
    if (!norm_plan(s, false, aligned16(x) && aligned16(y)).fits) return WINO_ERR_UNSUPPORTED;
    const NormApply a{x8 ? nullptr : x, x8 ? (const int8_t*)x : nullptr, x8 ? rows_of(x, s) : nullptr, stats, gamma,
                      beta, y};
    return hip_status(launch_norm_apply(a, s, aligned16(x) && aligned16(y), (hipStream_t)stream));
}

size_t wino_group_norm_backward_workspace_bytes(int N, int C, int H, int W, int G, unsigned flags) {
    NormShape s;
    return make_shape(N, C, H, W, G, flags, WINO_FLAG_ACT8, &s) == WINO_OK ? norm_need(s, true) : (size_t)-1;
}

int wino_group_norm_backward_nhwc(const void* dy, const void* x, const float* stats, const float* gamma,
                                  const float* beta, void* dx, float* dgamma, float* dbeta, int N, int C, int H, int W,
                                  int G, unsigned flags, void* workspace, size_t workspace_bytes, void* stream) {
    const bool x8 = (flags & WINO_FLAG_ACT8) != 0;
    if (!dy || !x || !stats || !dx || (x8 && ((uintptr_t)x & 15))) return WINO_ERR_INVALID_ARG;
    NormShape s;
    const int st = make_shape(N, C, H, W, G, flags, WINO_FLAG_ACT8, &s);
    if (st != WINO_OK) return st;
    const NormPlan p = norm_plan(s, true, aligned16(x) && aligned16(dy) && aligned16(dx));
    if (!p.fits) return WINO_ERR_UNSUPPORTED;
    const int sp = space(workspace, workspace_bytes, p.need);
    if (sp != WINO_OK) return sp;
    const size_t row = (size_t)C * sizeof(float), all = tensor_bytes(s);
    const Buf bufs[] = {{dy, all, false}, {x, x8 ? act8_size(s) : all, false},
                        {stats, (size_t)N * G * 2 * sizeof(float), false}, {gamma, row, false}, {beta, row, false},
                        {dx, all, true}, {dgamma, row, true}, {dbeta, row, true}, {workspace, p.need, true}};
    if (!disjoint(bufs)) return WINO_ERR_INVALID_ARG;
    const NormBwd a{dy, x8 ? nullptr : x, x8 ? (const int8_t*)x : nullptr, x8 ? rows_of(x, s) : nullptr, stats, gamma,
                    beta, dx, dgamma, dbeta};
    return hip_status(launch_norm_backward(a, s, p, workspace, (hipStream_t)stream));
}

size_t wino_conv2d_wgrad_workspace_bytes(int N, int C, int H, int W, int K, int pad, unsigned flags) {
    WgradShape s;
    if (make_wgrad(N, C, H, W, K, pad, flags, &s) != WINO_OK) return (size_t)-1;
    // the plan is another where the input is formed from the norm
    const size_t plain = wgrad_workspace(s);
    s.norm = true;
    const size_t formed = wgrad_workspace(s);
    return plain > formed ? plain : formed;
}

int wino_conv2d_wgrad_nhwc(const void* x, const void* dy, float* dg, const float* stats, const float* gamma,
                           const float* beta, int G, int N, int C, int H, int W, int K, int pad, unsigned flags,
                           void* workspace, size_t workspace_bytes, void* stream) {
    const bool x8 = (flags & WINO_FLAG_ACT8) != 0;
    if (!x || !dy || !dg || (x8 && ((uintptr_t)x & 15))) return WINO_ERR_INVALID_ARG;
    WgradShape s;
    int st = make_wgrad(N, C, H, W, K, pad, flags, &s);
    if (st != WINO_OK) return st;
    NormShape t;
    st = make_shape(N, C, H, W, stats ? G : 1, flags, WINO_FLAG_ACT8, &t);
    if (st != WINO_OK) return st;
    // without statistics the layer's input is x itself
    if (!stats && s.act != Act::None) return WINO_ERR_UNSUPPORTED;
    s.norm = stats != nullptr;
    s.G = t.G;
    s.D = t.D;
    const size_t need = wgrad_workspace(s);
    const int sp = space(workspace, workspace_bytes, need);
    if (sp != WINO_OK) return sp;
    const size_t row = (size_t)C * sizeof(float);
    const Buf bufs[] = {{x, x8 ? act8_size(t) : tensor_bytes(t), false},
                        {dy, (size_t)N * K * s.Ho * s.Wo * io_size(s.io), false},
                        {stats, (size_t)N * t.G * 2 * sizeof(float), false}, {gamma, row, false}, {beta, row, false},
                        {dg, (size_t)K * C * 9 * sizeof(float), true}, {workspace, need, true}};
    if (!disjoint(bufs)) return WINO_ERR_INVALID_ARG;
    const WgradArgs a{x8 ? nullptr : x, dy, x8 ? (const int8_t*)x : nullptr, x8 ? rows_of(x, t) : nullptr, stats, gamma,
                      beta, dg};
    return hip_status(launch_wgrad(a, s, workspace, (hipStream_t)stream));
}

}  // extern "C"
