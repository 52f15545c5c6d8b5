"""The weight gradient at operands of mixed magnitude: each channel of the input and each
filter of dy keeps its own precision, whatever the others hold.

Bound, from the arithmetic: an operand's two fp16 terms (bf16's one) are off by 2^-22 of it
and by 2^-39 of the largest value that its channel or filter may hold; a product of two by
as much from each and by 2^-22 for the term left out; sums by SUM; results by fp32's least
number, 2^-149.  Operands formed on load are off as off_a says.  The largest value of a
channel: of x or dy its own; of a checkpoint |centre| + 127 step; through the norm
|gamma| (|centre - mean| + 127 step) rstd + |beta| of a checkpoint, 2 |gamma| sqrt(D H W)
+ |beta| of x."""
import numpy as np
import pytest
import torch

import train_helpers as h
from oracle import train
from paper_1903_01521_amd import binding as B

pytestmark = pytest.mark.gpu

EPS, U = 1e-5, h.U32

# (N, H, W, C, K, pad): odd counts, whole 16 bytes, more channels than a workgroup's
# threads take at once
SHAPES = [(2, 9, 11, 35, 37, 1), (8, 7, 6, 40, 36, 1), (1, 13, 12, 64, 130, 0), (1, 4, 3, 1031, 33, 1),
          (1, 4, 3, 5, 1031, 1)]


def _call(x, dy, pad, dtype, dims, ckpt=False, stats=None, gamma=None, beta=None, act="none", offset=0):
    N, C, H, W, K = dims
    flags = h.IO[dtype] | h.ACT[act] | (B.WINO_FLAG_ACT8 if ckpt else 0)
    dg = torch.full((K, C, 3, 3), float("nan"), device=h.DEV)
    wsb = B.wino_conv2d_wgrad_workspace_bytes(N, C, H, W, K, pad, flags)
    ws = h.space(wsb)
    st, g, b = (None if v is None else h.dev(v) for v in (stats, gamma, beta))
    B.check(B.wino_conv2d_wgrad_nhwc(x if ckpt else h.dev(x, dtype, offset), h.dev(dy, dtype, offset), dg, st, g, b,
                                     0 if stats is None else stats.shape[1], N, C, H, W, K, pad, flags, ws, wsb))
    torch.cuda.synchronize()
    assert torch.isnan(ws[(wsb + 3) // 4:]).all()
    return h.host(dg)


def _check(dg, a, dy, pad, most_a, most_dy, off_a=None):
    size = train.wgrad(np.abs(a), np.abs(dy), pad)
    bound = (3 * 2.0 ** -22 + h.SUM) * size + 2.0 ** -149
    bound += 2.0 ** -39 * most_a[None, :, None, None] * train.wgrad(np.ones_like(a), np.abs(dy), pad)
    bound += 2.0 ** -39 * most_dy[:, None, None, None] * train.wgrad(np.abs(a), np.ones_like(dy), pad)
    if off_a is not None:
        bound += train.wgrad(off_a, np.abs(dy), pad)
    off = np.abs(dg - train.wgrad(a, dy, pad))
    assert (off <= 1.01 * bound).all(), float((off / bound).max())


def _most(v):
    return np.abs(v).max(axis=(0, 1, 2)).astype(np.float64)


def _powers(rng, count, least):
    """2^0 to 2^least in some order, both ends taken."""
    e = np.round(np.linspace(0, least, count))
    return 2.0 ** rng.permutation(e)


def _inputs(shape, dtype, least_x, least_dy, seed):
    N, H, W, C, K, pad = shape
    rng = np.random.default_rng(seed)
    sx, sd = _powers(rng, C, least_x), _powers(rng, K, least_dy)
    x = h.rounded(rng.standard_normal((N, H, W, C)) * sx, dtype)
    dy = h.rounded(rng.standard_normal((N, H + 2 * pad - 2, W + 2 * pad - 2, K)) * sd, dtype)
    return x, dy, sx, sd, rng


@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_channels_and_filters_of_different_magnitude(shape, offset):
    N, H, W, C, K, pad = shape
    x, dy, sx, sd, _ = _inputs(shape, "f32", -60, -60, 0)
    dg = _call(x, dy, pad, "f32", (N, C, H, W, K), offset=offset)
    _check(dg, x, dy, pad, _most(x), _most(dy))
    # at the same magnitude: rms errors of 2^-22 or so a product and, in 100 accumulations at
    # most of 2^-24 each, 2^-22 a sum (two terms of 8 bits: 4.5e-6)
    ref = train.wgrad(x, dy, pad)
    unit = (sx[None, :] * sd[:, None])[:, :, None, None]
    assert np.linalg.norm((dg - ref) / unit) <= 1e-6 * np.linalg.norm(ref / unit)


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_large_and_small(shape):
    # channels up to 2^60, filters down to 2^-90: results within fp32's range
    N, H, W, C, K, pad = shape
    x, dy, sx, sd, _ = _inputs(shape, "f32", 60, -90, 1)
    _check(_call(x, dy, pad, "f32", (N, C, H, W, K)), x, dy, pad, _most(x), _most(dy))


def test_values_of_one_channel_far_apart():
    # one value of dy a filter: dg is a row of products, of values from 1 to 2^-45 of the largest
    N, H, W, C, K = 1, 8, 9, 24, 72
    rng = np.random.default_rng(2)
    x = (2.0 ** rng.uniform(-45, 0, (N, H, W, C)) * rng.choice([-1, 1], (N, H, W, C))).astype(np.float32)
    dy = np.zeros((N, H, W, K), np.float32)
    for k in range(K):
        dy[0, k // W, k % W, k] = 1.0 + rng.random()
    dg = _call(x, dy, 1, "f32", (N, C, H, W, K))
    _check(dg, x, dy, 1, _most(x), _most(dy))
    ref = train.wgrad(x, dy, 1)
    off = np.abs(dg - ref)
    # no sums here: the products' own bound, 2^-39 of the channel's largest times the filter's value
    most = (_most(x)[None, :] * _most(dy)[:, None])[:, :, None, None]
    assert (off <= 1.01 * ((3 * 2.0 ** -22 + 2 * U) * np.abs(ref) + 2.0 ** -38 * most)).all()


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("dtype,least", [("f32", -50), ("bf16", -50), ("f16", -6)])
def test_from_the_checkpoint(shape, dtype, least):
    N, H, W, C, K, pad = shape
    x, dy, _, _, _ = _inputs(shape, dtype, least, least, 3)
    codes, centre, step = train.act8_pack(x)
    a = train.act8_unpack(codes, centre, step)
    most = (np.abs(centre) + 127.0 * step).max(axis=0).astype(np.float64)
    off_a = np.broadcast_to(4 * U * (np.abs(codes * step[:, None, None].astype(np.float64)) + np.abs(centre)[:, None, None]),
                            a.shape)
    dg = _call(h.make_ckpt(codes, centre, step), dy, pad, dtype, (N, C, H, W, K), ckpt=True)
    _check(dg, a, dy, pad, most, _most(dy), off_a)


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("ckpt", [False, True])
@pytest.mark.parametrize("dtype,least", [("f32", -50), ("bf16", -50), ("f16", -6)])
@pytest.mark.parametrize("shape,G", list(zip(SHAPES, [7, 8, 16, 1031, 1])), ids=str)
def test_through_the_norm(shape, G, dtype, least, ckpt, act):
    N, H, W, C, K, pad = shape
    x, dy, _, _, rng = _inputs(shape, dtype, 0, least, 4)
    gamma = (_powers(rng, C, -40) * (1 + 0.2 * rng.random(C))).astype(np.float32).astype(np.float64)
    gamma[C // 2] = 1000.0
    beta = (0.5 * rng.standard_normal(C) * gamma).astype(np.float32).astype(np.float64)
    st = np.stack(train.group_stats(x, G, EPS), -1).astype(np.float32).astype(np.float64)
    packed = train.act8_pack(x)
    v = train.act8_unpack(*packed) if ckpt else x
    n = train.normed(v, st[..., 0], st[..., 1])
    z = n * gamma + beta
    a = train.act(z, act)
    D = C // G
    mean, rstd = (np.repeat(st[..., i], D, axis=1) for i in range(2))       # [N][C]
    if ckpt:
        codes, centre, step = packed
        reach = (np.abs(centre - mean) + 127.0 * step) * rstd
        most = (np.abs(gamma) * reach + np.abs(beta)).max(axis=0)
        off_n = 6 * U * np.broadcast_to(reach[:, None, None], n.shape)
    else:
        most = 2 * np.abs(gamma) * np.sqrt(D * H * W) + np.abs(beta)
        off_n = 4 * U * np.abs(n)
    off_a = 1.1 * (off_n * np.abs(gamma) + 3 * U * (np.abs(n * gamma) + np.abs(beta)))
    if act == "silu":
        off_a = off_a + np.abs(a) * (2 * np.abs(z) + 8) * U
    dg = _call(h.make_ckpt(*packed) if ckpt else x, dy, pad, dtype, (N, C, H, W, K), ckpt, st, gamma, beta, act)
    _check(dg, a, dy, pad, most, _most(dy), off_a)


@pytest.mark.parametrize("ckpt", [False, True])
def test_a_bound_past_fp32s_range(ckpt):
    # gamma sqrt(D H W) overflows, the values do not
    N, H, W, C, K, G = 1, 10, 10, 8, 8, 2
    rng = np.random.default_rng(5)
    x = rng.standard_normal((N, H, W, C)).astype(np.float32)
    dy = (1e-3 * rng.standard_normal((N, H, W, K))).astype(np.float32)
    gamma = np.full(C, np.float32(3e37)).astype(np.float64)
    gamma[3] = 1.0
    st = np.stack(train.group_stats(x, G, EPS), -1).astype(np.float32).astype(np.float64)
    packed = train.act8_pack(x)
    a = train.normed(train.act8_unpack(*packed) if ckpt else x, st[..., 0], st[..., 1]) * gamma
    dg = _call(h.make_ckpt(*packed) if ckpt else x, dy, 1, "f32", (N, C, H, W, K), ckpt, st, gamma, np.zeros(C))
    most = np.where(gamma > 1, 3.4e38, 2 * np.sqrt(C // G * H * W))
    _check(dg, a, dy, 1, most, _most(dy), 1e-6 * np.abs(gamma) * np.ones_like(a))
