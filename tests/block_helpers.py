"""Calls of the attention half's entry points on numpy inputs, and error bounds derived
from 64-bit values."""
import numpy as np
import torch

from oracle import block as O
from paper_1903_01521_amd import binding as B
from train_helpers import ACT, DEV, DTYPE, HALF_ULP, IO, U32, dev, host, space

# Roundings that a sum of n products counts for, of the absolute products: one each, some
# more, and for fp32 the terms of the operands' split that are dropped, 2^-20.
def sums(n, dtype):
    return (n + 16 + (16 if dtype == "f32" else 0)) * U32


TINY = {"f32": 2.0 ** -126, "f16": 2.0 ** -25, "bf16": 2.0 ** -126}     # half a step at the range's lower end


def within(got, want, tol, what=""):
    """Every element within its bound."""
    got = host(got) if isinstance(got, torch.Tensor) else got
    assert got.shape == want.shape, (what, got.shape, want.shape)
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    bad = ~same & ~(np.abs(got - want) <= tol)
    assert not bad.any(), (f"{what}: {bad.sum()} of {bad.size} past the bound, the worst by "
                           f"{np.nanmax(np.where(same, 0, np.abs(got - want)) / np.maximum(tol, 1e-300)):.3g} at "
                           f"{np.unravel_index(np.argmax(bad), bad.shape)}")


def stored(want, tol, dtype):
    """A bound before the result is rounded to dtype, and after."""
    return tol * (1 + HALF_ULP[dtype]) + HALF_ULP[dtype] * np.abs(want) + TINY[dtype]


def view(a, dtype, ld=None, offset=0, fill=float("nan")):
    """[N][L][heads][D] on the device with tokens ld apart; returns the view and its buffer."""
    N, L, H, D = a.shape
    ld = ld or H * D
    buf = torch.full((N * L * ld + offset + 64,), fill, dtype=DTYPE[dtype], device=DEV)
    v = buf[offset:].as_strided((N, L, H, D), (L * ld, ld, D, 1))
    v.copy_(torch.from_numpy(np.ascontiguousarray(a, np.float32)))
    return v, buf


def untouched(buf, v, fill):
    """Nothing of buf outside the view was written: fill is a number."""
    seen = torch.ones_like(buf, dtype=torch.bool)
    seen.as_strided(v.shape, v.stride(), v.storage_offset()).fill_(False)
    torch.cuda.synchronize()
    return bool((buf[seen] == fill).all())


# ---------------------------------------------------------------- norm and rotation

def table(T, R, rng):
    a = rng.uniform(-3.2, 3.2, (T, R // 2))
    return np.stack((np.cos(a), np.sin(a)), -1).astype(np.float32)


def angles(rot, pos, N, L):
    """cos, sin [N][L][1][R/2] in 64 bits."""
    rows = np.broadcast_to(rot[:L][None], (N, L) + rot.shape[1:]) if pos is None else rot[pos]
    return rows[:, :, None, :, 0].astype(np.float64), rows[:, :, None, :, 1].astype(np.float64)


def ints(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a, np.int32)).to(DEV)


# A sum of D squares over lanes, division, root, reciprocal, products and a rotation's two
# terms: D + 16 roundings bound all of them relative to |za| + |zb|.
def norm_tol(x, gamma, cos, sin, eps, pairs):
    D = x.shape[-1]
    z = np.abs(x / np.sqrt((x * x).mean(-1, keepdims=True) + eps))
    z = z if gamma is None else z * np.abs(gamma)
    return (D + 16) * U32 * O.turn(z, np.abs(cos), -np.abs(sin), pairs).clip(0) + (D + 16) * U32 * O.turn(
        z, np.abs(cos), np.abs(sin), pairs).clip(0) + (D + 16) * U32 * z


# ---------------------------------------------------------------- attention

def attend(q, k, v, scale, dtype="f32", klen=None, mask=None, lse=True, ld=(None, None, None), offset=0):
    """(y, lse) device tensors."""
    N, Lq, Hq, D = q.shape
    Lk, Hk = k.shape[1:3]
    ld = [l or h * D for l, h in zip(ld, (Hq, Hk, Hk))]
    (qt, _), (kt, _), (vt, _) = (view(a, dtype, l, offset) for a, l in zip((q, k, v), ld))
    y = dev(np.full(q.shape, np.nan), dtype, offset)
    st = torch.full((N, Hq, Lq), float("nan"), device=DEV) if lse else None
    wsb = B.wino_cross_attention_workspace_bytes(N, Lq, Lk, Hq, Hk, D, IO[dtype])
    mt = None if mask is None else torch.from_numpy(np.ascontiguousarray(mask, np.uint8)).to(DEV)
    B.check(B.wino_cross_attention_nhwc(qt, kt, vt, ints(klen), mt, y, st, N, Lq, Lk, Hq, Hk, D, *ld, scale, IO[dtype],
                                        space(wsb), wsb), "attention")
    return y, st


def score_error(q, k, scale, D, dtype):
    """Bound of |S| errors [N][Hq][Lq][Lk] for heads [..][L][D]: a sum of D products, scaled."""
    return sums(D, dtype) * scale * (np.abs(q) @ np.abs(k).transpose(0, 1, 3, 2))


def attend_tol(q, k, v, scale, kept, p, y, lse, dtype):
    """Bounds of y and lse: scores' errors, the exponent's argument (|S| and the largest
    score, rounded some times each), P's rounding, and sums over Lk keys; fp16 loses
    values below 2^-25 of a row's largest share."""
    N, Lk, Hk, D = k.shape
    rep = q.shape[2] // Hk
    kk = np.repeat(O._drop(k, kept).transpose(0, 2, 1, 3), rep, 1)
    vv = np.repeat(O._drop(v, kept).transpose(0, 2, 1, 3), rep, 1)
    qq = q.transpose(0, 2, 1, 3)
    es = score_error(qq, kk, scale, D, dtype)
    s = scale * np.abs(qq @ kk.transpose(0, 1, 3, 2)) * kept[:, None, None]
    big = s.max(-1, keepdims=True)
    arg = es + 6 * U32 * (s + big) + 8 * U32                 # of a term's exponent
    worst = np.where(kept[:, None, None], arg, 0).max(-1, keepdims=True)
    rel = arg + worst + HALF_ULP[dtype] + sums(Lk + 16, dtype)
    ty = (p * rel) @ np.abs(vv) + 2 * TINY["f16"] * (dtype == "f16") * np.abs(vv).sum(2, keepdims=True)
    tl = worst[..., 0] + (Lk + 32) * U32 + 4 * U32 * np.abs(np.where(np.isinf(lse), 0, lse))
    return stored(y, ty.transpose(0, 2, 1, 3), dtype), tl


def attend_back(dy, q, k, v, y, lse, scale, dtype="f32", klen=None, mask=None, ld=(None, None, None), offset=0):
    """(dq, dk, dv) views, and their buffers filled with 7 elsewhere."""
    N, Lq, Hq, D = q.shape
    Lk, Hk = k.shape[1:3]
    ld = [l or h * D for l, h in zip(ld, (Hq, Hk, Hk))]
    (qt, _), (kt, _), (vt, _) = (view(a, dtype, l, offset) for a, l in zip((q, k, v), ld))
    outs = [view(np.full(a.shape, np.nan), dtype, l, offset, 7.0) for a, l in zip((q, k, v), ld)]
    wsb = B.wino_cross_attention_backward_workspace_bytes(N, Lq, Lk, Hq, Hk, D, IO[dtype])
    mt = None if mask is None else torch.from_numpy(np.ascontiguousarray(mask, np.uint8)).to(DEV)
    B.check(B.wino_cross_attention_backward_nhwc(
        dev(dy, dtype, offset), qt, kt, vt, dev(y, dtype, offset), dev(lse), ints(klen), mt, outs[0][0], outs[1][0],
        outs[2][0], N, Lq, Lk, Hq, Hk, D, *ld, scale, IO[dtype], space(wsb), wsb), "attention backward")
    return outs


def attend_back_tol(m, scale, kept, D, dtype, dq, dk, dv, lse):
    """Bounds of dq, dk, dv from attention_backward's intermediates: errors of S, dP and
    delta, dS's and P's rounding, and the sums.  dS is rounded while delta still has the
    rounding of y, h sum |dy y|, which is then taken off with P's: h of that again, twice.
    dS's roundings r_j enter dq as sum r_j k_j - (sum r_j) sum P k, so |r_j| <= h |dS_j| counts
    with |k_j| + sum P |k|."""
    a = {n: np.abs(m[n]) for n in ("q", "k", "v", "dy", "y")}
    finite = np.where(np.isinf(lse), 0, np.abs(lse))[..., None]
    ep = score_error(a["q"], a["k"], scale, D, dtype) + 6 * U32 * (np.abs(m["s"]) + finite) + 8 * U32
    edp = sums(D, dtype) * (a["dy"] @ a["v"].transpose(0, 1, 3, 2))
    Lq, Lk = m["p"].shape[-2:]
    h, dyy = HALF_ULP[dtype], (a["dy"] * a["y"]).sum(-1, keepdims=True)
    edelta = (D + 4) * U32 * dyy + (Lk + 16) * U32 * (m["p"] * (np.abs(m["dp"]) + np.abs(m["delta"]))).sum(
        -1, keepdims=True) + 3 * h * h * dyy + (m["p"] * (ep + edp)).sum(-1, keepdims=True) * h
    eds = m["p"] * (ep * (1 + ep) * np.abs(m["dp"] - m["delta"]) + edp + edelta) + (h + 8 * U32) * np.abs(m["ds"])
    epv = m["p"] * (ep * (1 + ep) + h + 4 * U32)
    if dtype == "f16":          # what falls below fp16's range, P held 2^12 up, dS near 2^14 of its column's largest
        epv = epv + 2.0 ** -36
        most = np.maximum(np.abs(m["ds"]).max(-1, keepdims=True), np.abs(m["ds"]).max(-2, keepdims=True))
        eds = eds + 2.0 ** -36 * most
    ads = np.abs(m["ds"])
    mean = m["p"] @ a["k"]
    tq = scale * (eds @ a["k"] + (h * ads).sum(-1, keepdims=True) * mean + sums(Lk, dtype) * (ads @ a["k"]))
    rows = sums(Lq * (m["q"].shape[1] // dk.shape[2]), dtype)
    t = lambda x: x.transpose(0, 1, 3, 2)  # noqa: E731
    tk = m["shared"](scale * (t(eds) @ a["q"] + rows * (t(ads) @ a["q"])))
    tv = m["shared"](t(epv) @ a["dy"] + rows * (t(m["p"]) @ a["dy"]))
    return (stored(dq, tq.transpose(0, 2, 1, 3), dtype), stored(dk, tk, dtype), stored(dv, tv, dtype))


# ---------------------------------------------------------------- gated layer

def gated(x, w, bias, dtype="f32", act="none", offset=0, y=None):
    """y of x [N][H][W][C], a device tensor."""
    N, H, W, C = x.shape
    K = w.shape[1]
    flags = IO[dtype] | ACT[act]
    y = dev(np.full((N, H, W, K), np.nan), dtype, offset)
    wsb = B.wino_gated_layer_workspace_bytes(N, C, H, W, K, flags)
    B.check(B.wino_gated_layer_nhwc(dev(x, dtype, offset), dev(w, dtype, offset), None if bias is None else dev(bias), y,
                                    N, C, H, W, K, flags, space(wsb), wsb), "gated")
    return y


def gated_back(dy, x, w, bias, dtype="f32", act="none", offset=0, want=(True, True, True)):
    N, H, W, C = x.shape
    K = w.shape[1]
    flags = IO[dtype] | ACT[act]
    outs = [dev(np.full(s, np.nan), d, offset) if on else None
            for s, d, on in zip((x.shape, w.shape, (2, K)), (dtype, dtype, "f32"), want)]
    wsb = B.wino_gated_layer_backward_workspace_bytes(N, C, H, W, K, flags)
    B.check(B.wino_gated_layer_backward_nhwc(dev(dy, dtype, offset), dev(x, dtype, offset), dev(w, dtype, offset),
                                             None if bias is None else dev(bias), *outs, N, C, H, W, K, flags,
                                             space(wsb), wsb), "gated backward")
    return outs


def layers_tol(x, w, bias, dtype):
    """Bound of zg's and zu's errors [2][M][K]: sums of C products and the bias."""
    a = np.stack([np.abs(x) @ np.abs(w[i]).T for i in (0, 1)])
    return sums(x.shape[-1], dtype) * (a if bias is None else a + np.abs(bias)[:, None])


# Sigmoid: its exponent is off by a few roundings of |z|, exp2, sum and reciprocal by some more.
def _sig_error(z):
    return (2 * np.abs(z) + 8) * U32


def gated_tol(x, w, bias, act, y, zg, zu, dtype):
    ez = layers_tol(x, w, bias, dtype)
    v, _ = O.act_slope(zg, act)
    top = 1.1 if act == "silu" else 1.0                          # of |act'|
    es = _sig_error(zg) if act == "silu" else 0.0
    tol = (top * ez[0] + np.abs(v) * es) * (np.abs(zu) + ez[1]) + np.abs(v) * ez[1] + 8 * U32 * np.abs(y)
    return stored(y, tol, dtype)


def gated_back_tol(dy, x, w, bias, act, dz, got_like, dtype):
    """Bounds of dx, dw, dbias.  act'' of SiLU is below 0.5; where zg is within its error
    of zero ReLU's slope may be either."""
    _, zg, zu = O.gated(x, w, bias, act)
    ez = layers_tol(x, w, bias, dtype)
    v, d = O.act_slope(zg, act)
    top, curve = (1.1, 0.5) if act == "silu" else (1.0, 0.0)
    es = _sig_error(zg) if act == "silu" else 0.0
    ed = curve * ez[0] + es * (1 + np.abs(zg)) * 2
    if act == "relu":
        ed = ed + (np.abs(zg) <= ez[0])
    e = np.stack((np.abs(dy) * (np.abs(zu) * ed + (np.abs(d) + ed) * ez[1]), np.abs(dy) * (top * ez[0] + np.abs(v) * es)))
    e = e + 8 * U32 * np.abs(dz)
    kept = e + HALF_ULP[dtype] * (np.abs(dz) + e) + TINY[dtype]      # as it goes through the workspace
    M, C, K = x.shape[0], x.shape[1], w.shape[1]
    a = np.abs(dz) + kept
    aw, ax = np.abs(w), np.abs(x)
    tx = sum(kept[i] @ aw[i] + sums(2 * K, dtype) * (a[i] @ aw[i]) for i in (0, 1))
    tw = np.stack([kept[i].T @ ax + sums(M, dtype) * (a[i].T @ ax) for i in (0, 1)])
    tb = e.sum(1) + (M + 16) * U32 * np.abs(dz).sum(1)
    dx, dw, _ = got_like
    return stored(dx, tx, dtype), stored(dw, tw, dtype), tb
