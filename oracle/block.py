"""Norm and rotation of queries and keys, cross attention and the gated layer in 64 bits,
from their formulas, with the sums of absolute values that bound fp32's rounding."""
import numpy as np


def silu(z):
    return z / (1.0 + np.exp(-z))


def act_slope(z, act):
    """act(z) and its derivative (ReLU: 0 at z <= 0)."""
    if act == "none":
        return z, np.ones_like(z)
    if act == "relu":
        return np.maximum(z, 0.0), (z > 0).astype(z.dtype)
    s = 1.0 / (1.0 + np.exp(-z))
    return z * s, s + z * s * (1.0 - s)


# ---------------------------------------------------------------- norm and rotation

def pair_index(R, pairs):
    """Channels a[i], b[i] that turn together."""
    i = np.arange(R // 2)
    return (2 * i, 2 * i + 1) if pairs else (i, i + R // 2)


def turn(z, cos, sin, pairs):
    """z [..., D] with its pairs turned by cos, sin [..., R/2]."""
    R = 2 * cos.shape[-1]
    a, b = pair_index(R, pairs)
    y = z.copy()
    y[..., a] = z[..., a] * cos - z[..., b] * sin
    y[..., b] = z[..., b] * cos + z[..., a] * sin
    return y


def head_norm(x, gamma, cos, sin, eps, pairs=False):
    """y of x [N][L][heads][D]; cos, sin [N][L][1][R/2]."""
    z = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return turn(z if gamma is None else z * gamma, cos, sin, pairs)


def head_norm_backward(dy, x, gamma, cos, sin, eps, pairs=False):
    """dx, dgamma and the sum of dgamma's absolute terms."""
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    n = x * r
    dz = turn(dy, cos, -sin, pairs)
    dn = dz if gamma is None else dz * gamma
    dx = r * (dn - n * (dn * n).mean(-1, keepdims=True))
    return dx, (dz * n).sum((0, 1, 2)), np.abs(dz * n).sum((0, 1, 2))


# ---------------------------------------------------------------- attention

def kept_keys(N, Lk, klen=None, mask=None):
    kept = np.ones((N, Lk), bool)
    if klen is not None:
        kept &= np.arange(Lk) < np.clip(np.asarray(klen), 0, Lk)[:, None]
    if mask is not None:
        kept &= np.asarray(mask) != 0
    return kept


def _heads(x, rep=1):
    """[N][L][H][D] to [N][H * rep][L][D], each head rep times."""
    return np.repeat(x.transpose(0, 2, 1, 3), rep, axis=1)


def _drop(x, kept):
    """Keys that are left out as zeros."""
    return np.where(kept[:, :, None, None], x, 0.0)


def attention(q, k, v, scale, kept):
    """y [N][Lq][Hq][D], lse [N][Hq][Lq], and P [N][Hq][Lq][Lk]."""
    rep = q.shape[2] // k.shape[2]
    k, v = _heads(_drop(k, kept), rep), _heads(_drop(v, kept), rep)
    s = np.where(kept[:, None, None], scale * (_heads(q) @ k.transpose(0, 1, 3, 2)), -np.inf)
    top = s.max(-1, keepdims=True)
    top = np.where(np.isinf(top), 0.0, top)
    e = np.exp(s - top)
    total = e.sum(-1, keepdims=True)
    with np.errstate(divide="ignore"):
        lse = (np.log(total) + top)[..., 0]
    p = e / np.where(total > 0, total, 1.0)
    return (p @ v).transpose(0, 2, 1, 3), lse, p


def attention_backward(dy, q, k, v, y, lse, scale, kept):
    """dq, dk, dv with the rows' log sums that the forward pass left, and the intermediates
    that bound rounding (y is one of them only)."""
    N, Lk, Hk, D = k.shape
    rep = q.shape[2] // Hk
    k, v = _heads(_drop(k, kept), rep), _heads(_drop(v, kept), rep)
    q, dy, y = _heads(q), _heads(dy), _heads(y)
    s = scale * (q @ k.transpose(0, 1, 3, 2))
    with np.errstate(invalid="ignore", over="ignore"):
        p = np.where(kept[:, None, None], np.exp(s - lse[..., None]), 0.0)
    dp = dy @ v.transpose(0, 1, 3, 2)
    delta = (p * dp).sum(-1, keepdims=True)
    ds = p * (dp - delta)

    def shared(g):
        return g.reshape(N, Hk, rep, Lk, D).sum(2).transpose(0, 2, 1, 3)
    dq = scale * (ds @ k)
    dk, dv = scale * (ds.transpose(0, 1, 3, 2) @ q), p.transpose(0, 1, 3, 2) @ dy
    more = {"s": s, "p": p, "dp": dp, "delta": delta, "ds": ds, "q": q, "k": k, "v": v, "dy": dy, "y": y,
            "shared": shared}
    return dq.transpose(0, 2, 1, 3), shared(dk), shared(dv), more


# ---------------------------------------------------------------- gated layer

def gated(x, w, bias, act):
    """y of tokens x [M][C], and zg, zu."""
    zg, zu = x @ w[0].T, x @ w[1].T
    if bias is not None:
        zg, zu = zg + bias[0], zu + bias[1]
    return act_slope(zg, act)[0] * zu, zg, zu


def gated_backward(dy, x, w, bias, act):
    """dx, dw, dbias, and dz [2][M][K]."""
    _, zg, zu = gated(x, w, bias, act)
    v, d = act_slope(zg, act)
    dz = np.stack((dy * zu * d, dy * v))
    return dz[0] @ w[0] + dz[1] @ w[1], np.stack((dz[0].T @ x, dz[1].T @ x)), dz.sum(1), dz
