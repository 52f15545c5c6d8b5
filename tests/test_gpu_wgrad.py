"""The weight gradient of the channel-last 3x3 layer against the fp64 oracle.

Bound, fixed from the arithmetic: a product of operands held in two bf16 terms is off
by at most 2^-15 of itself (2^-17 from each operand's rounding, 2^-16 for the product
that is left out), the sums round by at most SUM, and an input formed from the norm by
SUM times 1 + kappa and the checkpoint's rounding: relative to sum |a| |dy|, and for the
last to sum |dy|."""
import numpy as np
import pytest
import torch

import train_helpers as h
from oracle import train
from paper_1903_01521_amd import binding as B

pytestmark = pytest.mark.gpu

EPS = 1e-5

# (N, H, W, C, K, pad): one pixel; no padding down to one output; channels and
# filters past a tile's edge, odd widths, fewer and more images than eight
SHAPES = [
    (1, 1, 1, 1, 1, 1), (1, 3, 3, 2, 3, 0), (2, 5, 4, 7, 5, 1), (3, 9, 11, 33, 17, 1), (1, 57, 57, 48, 48, 1),
    (8, 14, 14, 64, 64, 1), (9, 13, 7, 70, 65, 0), (2, 28, 28, 128, 130, 1), (1, 2, 40, 16, 16, 2), (17, 4, 3, 20, 36, 1),
    (1, 70, 9, 3, 64, 1), (4, 30, 31, 80, 40, 3),
]


def _inputs(shape, dtype, seed=0):
    N, H, W, C, K, pad = shape
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((N, H, W, C)) + 0.3 * rng.standard_normal(C)
    dy = rng.standard_normal((N, H + 2 * pad - 2, W + 2 * pad - 2, K))
    return h.rounded(x, dtype), h.rounded(dy, dtype)


def wgrad(x, dy, pad, dtype, C, H, W, ckpt=False, stats=None, gamma=None, beta=None, G=0, act="none", offset=0):
    N, Ho, Wo, K = dy.shape
    flags = h.IO[dtype] | h.ACT[act] | (B.WINO_FLAG_ACT8 if ckpt else 0)
    xt = x if ckpt else h.dev(x, dtype, offset)
    dg = torch.full((K, C, 3, 3), float("nan"), device=h.DEV)
    wsb = B.wino_conv2d_wgrad_workspace_bytes(N, C, H, W, K, pad, flags)
    ws = h.space(wsb)
    st, g, b = (None if v is None else h.dev(v) for v in (stats, gamma, beta))
    B.check(B.wino_conv2d_wgrad_nhwc(xt, h.dev(dy, dtype, offset), dg, st, g, b, G, N, C, H, W, K, pad, flags, ws, wsb))
    torch.cuda.synchronize()
    assert torch.isnan(ws[(wsb + 3) // 4:]).all()
    return dg


def _check(dg, a, dy, pad, extra=0.0):
    ref = train.wgrad(a, dy, pad)
    size = train.wgrad(np.abs(a), np.abs(dy), pad)
    bound = (2.0 ** -15 + h.SUM) * size + extra * train.wgrad(np.ones_like(a), np.abs(dy), pad)
    off = np.abs(h.host(dg) - ref)
    assert (off <= bound).all(), float((off - bound).max())


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_weight_gradient(shape, dtype):
    N, H, W, C, K, pad = shape
    x, dy = _inputs(shape, dtype)
    _check(wgrad(x, dy, pad, dtype, C, H, W), x, dy, pad)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_from_the_checkpoint(shape, dtype):
    N, H, W, C, K, pad = shape
    x, dy = _inputs(shape, dtype, 1)
    packed = train.act8_pack(x)
    _check(wgrad(h.make_ckpt(*packed), dy, pad, dtype, C, H, W, ckpt=True), train.act8_unpack(*packed), dy, pad,
           8 * h.U32 * np.abs(x).max())


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("ckpt", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape,G", [((2, 5, 4, 7, 5, 1), 7), ((3, 9, 11, 33, 17, 1), 3), ((8, 14, 14, 64, 64, 1), 16),
                                     ((1, 57, 57, 48, 48, 1), 16), ((9, 13, 7, 70, 65, 0), 1)])
def test_through_the_norm(shape, G, dtype, ckpt, act):
    N, H, W, C, K, pad = shape
    x, dy = _inputs(shape, dtype, 2)
    rng = np.random.default_rng(3)
    gamma = (1 + 0.2 * rng.standard_normal(C)).astype(np.float32).astype(np.float64)
    beta = (0.5 * rng.standard_normal(C)).astype(np.float32).astype(np.float64)
    mean, rstd = (v.astype(np.float32).astype(np.float64) for v in train.group_stats(x, G, EPS))
    packed = train.act8_pack(x)
    v = train.act8_unpack(*packed) if ckpt else x
    a = train.act(train.normed(v, mean, rstd) * gamma + beta, act)
    dg = wgrad(h.make_ckpt(*packed) if ckpt else x, dy, pad, dtype, C, H, W, ckpt, np.stack((mean, rstd), -1), gamma, beta,
               G, act)
    kappa = float((np.abs(x).max(axis=(1, 2)).max(axis=1)[:, None] * rstd).max())
    _check(dg, a, dy, pad, h.SUM * (1 + kappa) ** 2 * 1.2 * np.abs(gamma).max())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tensors_off_16_byte_addresses(dtype):
    shape = (2, 12, 13, 24, 40, 1)
    x, dy = _inputs(shape, dtype, 4)
    a = wgrad(x, dy, 1, dtype, 24, 12, 13, offset=1)
    assert torch.equal(a, wgrad(x, dy, 1, dtype, 24, 12, 13))


def test_gradient_is_that_of_the_layer():
    # sum(dg * g) = sum(conv(x, g) * dy), the layer being linear in g, through the
    # library's own forward call (normwise error 1e-5 of F(2x2,3x3))
    N, H, W, C, K = 2, 12, 10, 16, 24
    x, dy = _inputs((N, H, W, C, K, 1), "f32", 5)
    rng = np.random.default_rng(6)
    g = (rng.standard_normal((K, C, 3, 3)) / np.sqrt(9 * C)).astype(np.float32)
    U = torch.empty(B.wino_filter_bytes(C, K, 2) // 4, device=h.DEV)
    B.check(B.wino_filter_transform(h.dev(g), U, C, K, 2))
    y = torch.empty((N, H, W, K), device=h.DEV)
    wsb = B.wino_workspace_bytes_nhwc(N, C, H, W, K, 1, 2, 0)
    B.check(B.wino_conv2d_nhwc(h.dev(x), U, y, N, C, H, W, K, 1, 2, 0, h.space(wsb), wsb))
    y = h.host(y)
    dg = h.host(wgrad(x, dy, 1, "f32", C, H, W))
    size = np.sqrt((y ** 2).sum() * (dy.astype(np.float64) ** 2).sum())
    assert abs((dg * g).sum() - (y * dy).sum()) < 1e-4 * size


def test_values_that_are_not_finite_reach_their_channels_only():
    shape = (2, 9, 10, 40, 70, 1)
    N, H, W, C, K, pad = shape
    x, dy = _inputs(shape, "f32", 7)
    clean = h.host(wgrad(x, dy, pad, "f32", C, H, W))
    x[1, 4, 4, 5] = np.inf
    dy[0, 4, 5, 66] = np.nan
    dg = h.host(wgrad(x, dy, pad, "f32", C, H, W))
    assert not np.isfinite(dg[:, 5]).any() and not np.isfinite(dg[66]).any()
    keep = np.ones((K, C), bool)
    keep[:, 5] = keep[66] = False
    assert np.array_equal(dg[keep], clean[keep])


def test_small_and_large_values():
    shape = (1, 8, 8, 16, 16, 1)
    x, dy = _inputs(shape, "f32", 8)
    for scale in (1e-30, 1e30):
        dg = h.host(wgrad(x * np.float32(scale), dy, 1, "f32", 16, 8, 8)) / scale
        ref = train.wgrad(x, dy, 1)
        assert np.abs(dg - ref).max() <= 2.0 ** -14 * train.wgrad(np.abs(x), np.abs(dy), 1).max()


def test_repeats_on_a_stream_and_in_a_graph():
    shape = (3, 20, 21, 72, 40, 1)
    N, H, W, C, K, pad = shape
    x, dy = _inputs(shape, "f32", 9)
    first = wgrad(x, dy, pad, "f32", C, H, W)
    xt, dyt, dg = h.dev(x), h.dev(dy), torch.zeros((K, C, 3, 3), device=h.DEV)
    wsb = B.wino_conv2d_wgrad_workspace_bytes(N, C, H, W, K, pad, 0)
    ws = h.space(wsb)

    def step():
        B.check(B.wino_conv2d_wgrad_nhwc(xt, dyt, dg, None, None, None, 0, N, C, H, W, K, pad, 0, ws, wsb))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    assert torch.equal(first, dg)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        dg.zero_()
        ws.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(first, dg)


def test_tensors_past_4_gib():
    # 2.7e9 values a tensor; all but the last image zero, so that dg is that image's own.
    # Both calls sum in 32 bits in another order: SUM of the sums of absolute values.
    N, H, W, C, K = 41, 1024, 1024, 64, 64
    gen = torch.Generator(device=h.DEV)
    gen.manual_seed(0)
    x = torch.zeros((N, H, W, C), dtype=torch.bfloat16, device=h.DEV)
    dy = torch.zeros((N, H, W, K), dtype=torch.bfloat16, device=h.DEV)
    x[-1].copy_(torch.randn((H, W, C), generator=gen, device=h.DEV))
    dy[-1].copy_(torch.randn((H, W, K), generator=gen, device=h.DEV))

    def call(x, dy):
        n = x.shape[0]
        dg = torch.empty((K, C, 3, 3), device=h.DEV)
        wsb = B.wino_conv2d_wgrad_workspace_bytes(n, C, H, W, K, 1, B.WINO_IO_BF16)
        B.check(B.wino_conv2d_wgrad_nhwc(x, dy, dg, None, None, None, 0, n, C, H, W, K, 1, B.WINO_IO_BF16, h.space(wsb), wsb))
        return dg
    whole, last = call(x, dy), call(x[-1:], dy[-1:])
    size = call(x[-1:].abs(), dy[-1:].abs())
    assert bool(((whole - last).abs() <= h.SUM * size).all()) and float(last.abs().max()) > 0
