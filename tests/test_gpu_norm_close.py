"""Group norm and its backward pass, element by element, against the fp64 oracle on the
call's own statistics, with means up to 1000 spreads away.

With the statistics given, no rounding is relative to |x| or |mean|, except a
checkpoint's value where it is formed as a number of its own (ReLU and none).  u = 2^-24:
  n = (x - mean) rstd          2u |n|
  z = n gamma + beta           3u |n gamma| + u |z|
  SiLU                         its slope is at most 1.1, that of its derivative 0.5;
                               a sigmoid is off by (2 |z| + 6) u of itself: u |z| for each of
                               the exponential's argument and its factor, a unit in the
                               last place for the exponential, the sum, the reciprocal
  sums                         SUM of the sums of absolute values
  dx                           four more roundings of each term
and a checkpoint's n, from folded constants (SiLU) u times |n|, |code step rstd| and
twice |(centre - mean) rstd|, else u rstd times |code step| and |x| and 2u |n|."""
import numpy as np
import pytest

import train_helpers as h
from oracle import train

pytestmark = pytest.mark.gpu

U, EPS = h.U32, 1e-5

# (N, H, W, C, G): in a workgroup's registers, odd channels, cut into chunks with one
# group and with groups of one channel, a group for a wide pixel
SHAPES = [(2, 14, 14, 32, 8), (2, 9, 11, 33, 11), (1, 150, 151, 8, 1), (2, 130, 129, 6, 6), (1, 40, 41, 520, 1)]


def _inputs(shape, dtype, shift, seed):
    N, H, W, C, G = shape
    rng = np.random.default_rng(seed)
    x = h.rounded(rng.standard_normal((N, H, W, C)) * np.exp(0.3 * rng.standard_normal(C)) + shift, dtype)
    gamma, beta = 1.0 + 0.2 * rng.standard_normal(C), 0.3 * rng.standard_normal(C)
    dy = h.rounded(rng.standard_normal((N, H, W, C)), dtype)
    return x, gamma.astype(np.float32).astype(np.float64), beta.astype(np.float32).astype(np.float64), dy


def _spread(v, C):
    return np.repeat(v, C // v.shape[1], axis=1)[:, None, None, :]


def _off_z(n, off_n, gamma, beta):
    return off_n * np.abs(gamma) + 3 * U * np.abs(n * gamma) + U * np.abs(n * gamma + beta)


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("dtype,shift", [("f32", 0.5), ("f32", 1000.0), ("bf16", 0.5), ("f16", 100.0)])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_forward(shape, dtype, shift, act):
    x, gamma, beta, _ = _inputs(shape, dtype, shift, 1)
    y, st, _ = h.group_norm(x, gamma, beta, shape[4], EPS, dtype, act)
    st = h.host(st)
    n = train.normed(x, st[..., 0], st[..., 1])
    z = n * gamma + beta
    ref = train.act(z, act)
    bound = (1.1 if act == "silu" else 1.0) * _off_z(n, 2 * U * np.abs(n), gamma, beta)
    if act == "silu":
        bound += np.abs(ref) * (2 * np.abs(z) + 8) * U
    off = np.abs(h.host(y) - ref)
    bound = bound * 1.01 + h.HALF_ULP[dtype] * (np.abs(ref) + bound) + 2.0 ** -25 * (dtype == "f16")
    assert (off <= bound).all(), float((off / bound).max())


def _check_backward(got, dy, x, off_n, st, gamma, beta, dtype, act):
    N, H, W, C = dy.shape
    G, count = st.shape[1], H * W * C // st.shape[1]
    mean, rstd = st[..., 0], st[..., 1]
    n = train.normed(x, mean, rstd)
    z = n * gamma + beta
    off_z = _off_z(n, off_n, gamma, beta)
    if act == "relu":
        assert (dy[np.abs(z) <= 2 * off_z] == 0).all()       # whose gradient may be either
    dz = dy * train.act_grad(z, act)
    off_dz = np.zeros_like(dz)
    if act == "silu":
        s = 1.0 / (1.0 + np.exp(-z))
        off_dz = np.abs(dy) * (0.5 * off_z + (1 + 2 * np.abs(z)) * (2 * np.abs(z) + 10) * U * s) + 2 * U * np.abs(dz)
    dn, rs = dz * gamma, _spread(rstd, C)
    rdx, rdgamma, rdbeta = train.group_norm_backward(dy, x, mean, rstd, gamma, beta, act)

    def group_mean(v):
        return _spread(v.reshape(N, H * W, G, C // G).sum(axis=(1, 3)) / count, C)
    m1, m2 = group_mean(dn), group_mean(dn * n)
    off_dn, off_dnn = off_dz * np.abs(gamma), off_dz * np.abs(n) + np.abs(dz) * off_n
    off_m1 = group_mean(off_dn + h.SUM * np.abs(dn))
    off_m2 = group_mean(off_dnn * np.abs(gamma) + h.SUM * np.abs(dn * n))
    terms = np.abs(dn) + np.abs(m1) + np.abs(n * m2)
    bound = rs * (off_dn + off_m1 + np.abs(n) * off_m2 + off_n * np.abs(m2) + 4 * U * terms) * 1.01
    dx, dgamma, dbeta = (h.host(v) for v in got)
    off = np.abs(dx - rdx)
    bound = bound + h.HALF_ULP[dtype] * (np.abs(rdx) + bound) + 2.0 ** -25 * (dtype == "f16")
    assert (off <= bound).all(), float((off / bound).max())
    assert (np.abs(dbeta - rdbeta) <= (off_dz + h.SUM * np.abs(dz)).sum(axis=(0, 1, 2))).all()
    assert (np.abs(dgamma - rdgamma) <= (off_dnn + h.SUM * np.abs(dz * n)).sum(axis=(0, 1, 2))).all()


def _stats(x, G):
    mean, rstd = train.group_stats(x, G, EPS)
    return np.stack((mean, rstd), -1).astype(np.float32).astype(np.float64)


def _for_relu(dy, n, off_n, gamma, beta, act):
    z = n * gamma + beta
    return np.where(np.abs(z) <= 2 * _off_z(n, off_n, gamma, beta), 0.0, dy) if act == "relu" else dy


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("dtype,shift", [("f32", 0.5), ("f32", 1000.0), ("bf16", 0.5), ("f16", 100.0)])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_backward(shape, dtype, shift, act):
    x, gamma, beta, dy = _inputs(shape, dtype, shift, 2)
    st = _stats(x, shape[4])
    n = train.normed(x, st[..., 0], st[..., 1])
    off_n = 2 * U * np.abs(n)
    dy = _for_relu(dy, n, off_n, gamma, beta, act)
    _check_backward(h.backward(dy, x, st, gamma, beta, dtype, act), dy, x, off_n, st, gamma, beta, dtype, act)


@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("dtype,shift", [("f32", 0.5), ("f32", 1000.0), ("bf16", 0.5), ("f16", 100.0)])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_backward_from_the_checkpoint(shape, dtype, shift, act, offset):
    x, gamma, beta, dy = _inputs(shape, dtype, shift, 3)
    C = shape[3]
    st = _stats(x, shape[4])
    codes, centre, step = train.act8_pack(x)
    v = train.act8_unpack(codes, centre, step)
    mean, rstd = _spread(st[..., 0], C), _spread(st[..., 1], C)
    n = train.normed(v, st[..., 0], st[..., 1])
    part, middle = np.abs(codes * step[:, None, None].astype(np.float64)), centre[:, None, None].astype(np.float64)
    if act == "silu":
        off_n = U * (np.abs(n) + rstd * (part + 2 * np.abs(middle - mean)))
    else:
        off_n = U * (2 * np.abs(n) + rstd * (part + np.abs(v)))
    off_n = off_n * 1.01
    dy = _for_relu(dy, n, off_n, gamma, beta, act)
    got = h.backward(dy, h.make_ckpt(codes, centre, step), st, gamma, beta, dtype, act, ckpt=True, offset=offset)
    _check_backward(got, dy, v, off_n, st, gamma, beta, dtype, act)
