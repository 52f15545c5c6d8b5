"""fp64 references of the training calls on channel-last tensors (test
infrastructure only): group norm with an activation and its gradients, the 8-bit
checkpoint, and the 3x3 layer's weight gradient, from their definitions.

Tensors are numpy arrays [N][H][W][C]; everything is float64 except the checkpoint,
whose codes are defined by 32-bit arithmetic.
"""
import numpy as np

FLAT = np.float32(2.0 ** -100)


def _per_group(x, G):
    N, H, W, C = x.shape
    return x.astype(np.float64).reshape(N, H * W, G, C // G)


def _channels(v, C):
    """[N][G] to [N][1][1][C]."""
    return np.repeat(v, C // v.shape[1], axis=1)[:, None, None, :]


def group_stats(x, G, eps):
    """(mean, rstd) [N][G]; the variance in two passes."""
    g = _per_group(x, G)
    mean = g.mean(axis=(1, 3))
    var = ((g - mean[:, None, :, None]) ** 2).mean(axis=(1, 3))
    return mean, 1.0 / np.sqrt(var + eps)


def act(z, kind):
    if kind == "relu":
        return np.maximum(z, 0.0)
    if kind == "silu":
        return z / (1.0 + np.exp(-z))
    return z


def act_grad(z, kind):
    if kind == "relu":
        return (z > 0).astype(np.float64)
    if kind == "silu":
        s = 1.0 / (1.0 + np.exp(-z))
        return s + z * s * (1.0 - s)
    return np.ones_like(z)


def normed(x, mean, rstd):
    C = x.shape[3]
    return (x.astype(np.float64) - _channels(mean, C)) * _channels(rstd, C)


def group_norm(x, gamma, beta, G, eps, kind):
    """(y, mean, rstd)"""
    mean, rstd = group_stats(x, G, eps)
    return act(normed(x, mean, rstd) * gamma + beta, kind), mean, rstd


def group_norm_backward(dy, x, mean, rstd, gamma, beta, kind):
    """(dx, dgamma, dbeta) of sum(y * dy), for the statistics given."""
    N, H, W, C = x.shape
    G = mean.shape[1]
    n = normed(x, mean, rstd)
    dz = dy.astype(np.float64) * act_grad(n * gamma + beta, kind)
    dn = dz * gamma
    m1 = _per_group(dn, G).mean(axis=(1, 3))
    m2 = _per_group(dn * n, G).mean(axis=(1, 3))
    dx = _channels(rstd, C) * (dn - _channels(m1, C) - n * _channels(m2, C))
    return dx, (dz * n).sum(axis=(0, 1, 2)), dz.sum(axis=(0, 1, 2))


def act8_pack(x):
    """(codes int8 [N][H][W][C], centre, step float32 [N][C]) of float32 x, in 32-bit steps."""
    x = x.astype(np.float32)
    lo, hi = x.min(axis=(1, 2)), x.max(axis=(1, 2))
    half = np.float32(0.5) * hi - np.float32(0.5) * lo
    centre = np.float32(0.5) * lo + np.float32(0.5) * hi
    flat = half < FLAT
    safe = np.where(flat, np.float32(1.0), half)
    inverse = np.where(flat, np.float32(0.0), np.float32(127.0) / safe)
    step = np.where(flat, np.float32(0.0), half / np.float32(127.0))
    q = np.rint((x - centre[:, None, None]) * inverse[:, None, None])
    return np.clip(q, -127, 127).astype(np.int8), centre.astype(np.float32), step.astype(np.float32)


def act8_unpack(codes, centre, step):
    """The values in 64 bits."""
    return centre[:, None, None].astype(np.float64) + step[:, None, None].astype(np.float64) * codes


def wgrad(a, dy, pad):
    """dg [K][C][3][3] of the layer with input a [N][H][W][C] and output gradient dy [N][Ho][Wo][K]."""
    N, Ho, Wo, K = dy.shape
    a = np.pad(a.astype(np.float64), ((0, 0), (pad, pad), (pad, pad), (0, 0)))
    C = a.shape[3]
    flat = dy.astype(np.float64).reshape(-1, K)
    dg = np.empty((K, C, 3, 3))
    for r in range(3):
        for s in range(3):
            dg[:, :, r, s] = flat.T @ a[:, r:r + Ho, s:s + Wo].reshape(-1, C)
    return dg
