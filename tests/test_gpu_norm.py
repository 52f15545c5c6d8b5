"""Group norm with an activation and its backward pass against the fp64 oracle.

Bounds, fixed from the arithmetic before any run: the statistics and sums round at
most SUM relative to the sum of absolute values; x - mean rounds relative to |x| and
|mean|, so a normalised value is off by SUM times 1 + kappa, kappa the largest
|x| * rstd; the activation's slope is at most 1.1; results in 16 bits are rounded
once more."""
import numpy as np
import pytest
import torch

import train_helpers as h
from oracle import train
from paper_1903_01521_amd import binding as B

pytestmark = pytest.mark.gpu

EPS = 1e-5

# (N, H, W, C, G): one value; one pixel; one channel a group; odd channels and
# groups of three; a group for all; 16 bytes that straddle groups; the library's
# own sizes; images past a workgroup's registers (cut into chunks); more channels
# than a workgroup's columns, with a tail; groups past 1024 channels
SHAPES = [
    (1, 1, 1, 1, 1), (3, 1, 1, 8, 2), (2, 5, 3, 7, 7), (2, 9, 11, 33, 11), (2, 14, 14, 40, 1), (3, 13, 7, 20, 4),
    (2, 10, 9, 24, 8), (1, 57, 57, 48, 16), (8, 28, 28, 128, 32), (2, 56, 56, 64, 32), (1, 150, 151, 8, 1),
    (2, 130, 129, 20, 2), (1, 224, 224, 64, 32), (1, 131, 77, 33, 3), (1, 3, 5, 2100, 3), (2, 2, 2, 1500, 1),
    (1, 40, 41, 520, 1), (5, 1, 2, 4096, 1024),
]


def _inputs(shape, dtype, seed=0, shift=0.5):
    N, H, W, C, G = shape
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((N, H, W, C)) * np.exp(0.3 * rng.standard_normal(C)) + shift * rng.standard_normal(C)
    gamma, beta = 1.0 + 0.2 * rng.standard_normal(C), 0.3 * rng.standard_normal(C)
    dy = rng.standard_normal((N, H, W, C))
    return (h.rounded(x, dtype), gamma.astype(np.float32).astype(np.float64),
            beta.astype(np.float32).astype(np.float64), h.rounded(dy, dtype))


def _kappa(x, G, rstd):
    N, H, W, C = x.shape
    most = np.abs(x).reshape(N, H * W, G, C // G).max(axis=(1, 3))
    return float((most * rstd).max())


def _check_forward(y, st, x, gamma, beta, G, dtype, act, eps=EPS):
    ref, mean, rstd = train.group_norm(x, gamma, beta, G, eps, act)
    kappa = _kappa(x, G, rstd)
    most = np.abs(x).max()
    assert np.abs(h.host(st)[..., 0] - mean).max() <= h.SUM * most
    assert (np.abs(h.host(st)[..., 1] / rstd - 1) <= h.SUM * (1 + kappa)).all()
    bound = h.SUM * (1 + kappa) * (1.1 * np.abs(gamma).max() * (1 + kappa) + np.abs(beta).max())
    off = np.abs(h.host(y) - ref)
    assert (off <= bound + h.HALF_ULP[dtype] * np.abs(ref)).all(), off.max()


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_group_norm(shape, dtype, act):
    x, gamma, beta, _ = _inputs(shape, dtype)
    y, st, _ = h.group_norm(x, gamma, beta, shape[4], EPS, dtype, act)
    _check_forward(y, st, x, gamma, beta, shape[4], dtype, act)


def _check_backward(got, dy, x, mean, rstd, gamma, beta, dtype, act):
    dx, dgamma, dbeta = (h.host(v) for v in got)
    G = mean.shape[1]
    rdx, rdgamma, rdbeta = train.group_norm_backward(dy, x, mean, rstd, gamma, beta, act)
    kappa = _kappa(x, G, rstd)
    n = np.abs(train.normed(x, mean, rstd))
    err = h.SUM * (1 + kappa)
    sums = 1.2 * np.abs(dy)
    assert (np.abs(dbeta - rdbeta) <= err * sums.sum(axis=(0, 1, 2)) * 2).all()
    assert (np.abs(dgamma - rdgamma) <= err * (sums * (1 + n)).sum(axis=(0, 1, 2)) * 2).all()
    scale = rstd.max() * np.abs(gamma).max() * 1.2 * np.abs(dy).max() * (2 + n.max()) ** 2
    off = np.abs(dx - rdx)
    assert (off <= err * scale + h.HALF_ULP[dtype] * np.abs(rdx)).all(), off.max()


def _away_from_zero(dy, x, mean, rstd, gamma, beta):
    """dy without the values whose z is so near 0 that ReLU's gradient may be either."""
    z = train.normed(x, mean, rstd) * gamma + beta
    return np.where(np.abs(z) < 1e-3 * (1 + _kappa(x, mean.shape[1], rstd)), 0.0, dy)


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_group_norm_backward(shape, dtype, act):
    x, gamma, beta, dy = _inputs(shape, dtype, 1)
    mean, rstd = (v.astype(np.float32).astype(np.float64) for v in train.group_stats(x, shape[4], EPS))
    if act == "relu":
        dy = _away_from_zero(dy, x, mean, rstd, gamma, beta)
    got = h.backward(dy, x, np.stack((mean, rstd), -1), gamma, beta, dtype, act)
    _check_backward(got, dy, x, mean, rstd, gamma, beta, dtype, act)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_group_norm_backward_from_the_checkpoint(shape, dtype):
    N, H, W, C, G = shape
    x, gamma, beta, dy = _inputs(shape, dtype, 2)
    mean, rstd = (v.astype(np.float32).astype(np.float64) for v in train.group_stats(x, G, EPS))
    packed = train.act8_pack(x)
    got = h.backward(dy, h.make_ckpt(*packed), np.stack((mean, rstd), -1), gamma, beta, dtype, "silu", ckpt=True)
    _check_backward(got, dy, train.act8_unpack(*packed), mean, rstd, gamma, beta, dtype, "silu")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(2, 10, 9, 24, 8), (1, 150, 151, 8, 1), (2, 28, 28, 64, 8)], ids=str)
def test_tensors_off_16_byte_addresses(shape, dtype):
    x, gamma, beta, dy = _inputs(shape, dtype, 3)
    y, st, _ = h.group_norm(x, gamma, beta, shape[4], EPS, dtype, "silu", offset=1)
    _check_forward(y, st, x, gamma, beta, shape[4], dtype, "silu")
    mean, rstd = (v.astype(np.float32).astype(np.float64) for v in train.group_stats(x, shape[4], EPS))
    got = h.backward(dy, x, np.stack((mean, rstd), -1), gamma, beta, dtype, "silu", offset=1)
    _check_backward(got, dy, x, mean, rstd, gamma, beta, dtype, "silu")


@pytest.mark.parametrize("shape", [(2, 14, 14, 32, 8), (1, 150, 151, 8, 1)], ids=str)
def test_without_parameters_and_statistics(shape):
    x, _, _, dy = _inputs(shape, "f32", 4)
    C, G = shape[3], shape[4]
    one, zero = np.ones(C), np.zeros(C)
    y, _, _ = h.group_norm(x, None, None, G, EPS, stats=False)
    again, st, _ = h.group_norm(x, one, zero, G, EPS)
    assert torch.equal(y, again)
    stats = h.host(st)
    a = h.backward(dy, x, stats, None, None, act="silu")
    b = h.backward(dy, x, stats, one, zero, act="silu")
    assert all(torch.equal(u, v) for u, v in zip(a, b))


@pytest.mark.parametrize("shape", [(2, 14, 14, 32, 8), (1, 150, 151, 8, 1)], ids=str)
def test_variance_is_about_the_mean(shape):
    # mean 1000 times the spread: E[x^2] - mean^2 in 32 bits would lose the variance
    N, H, W, C, G = shape
    rng = np.random.default_rng(5)
    x = (1000.0 + rng.standard_normal((N, H, W, C))).astype(np.float32)
    y, st, _ = h.group_norm(x, np.ones(C), np.zeros(C), G, EPS)
    _, rstd = train.group_stats(x, G, EPS)
    # mean off by SUM * 1000 = 0.015 at worst, which adds its square to the variance
    assert np.abs(h.host(st)[..., 1] / rstd - 1).max() <= 3e-4


@pytest.mark.parametrize("shape", [(2, 14, 14, 32, 8), (2, 150, 151, 8, 2)], ids=str)
def test_constant_groups_and_one_value(shape):
    N, H, W, C, G = shape
    x, gamma, beta, _ = _inputs(shape, "f32", 6)
    x[0, :, :, :C // G] = 3.25                           # one group is constant: n = 0
    y, st, _ = h.group_norm(x, gamma, beta, G, EPS)
    assert np.array_equal(h.host(y)[0, :, :, :C // G], np.broadcast_to(beta[:C // G], (H, W, C // G)))
    assert h.host(st)[0, 0, 0] == 3.25
    one = np.full((1, 1, 1, 4), 7.0, np.float32)
    y, st, _ = h.group_norm(one, np.ones(4), np.full(4, 0.5), 4, EPS)
    assert (h.host(y) == 0.5).all()


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("shape", [(2, 14, 14, 32, 8), (2, 150, 151, 8, 2)], ids=str)
def test_a_value_that_is_not_finite_stays_in_its_group(shape, bad):
    N, H, W, C, G = shape
    D = C // G
    x, gamma, beta, dy = _inputs(shape, "f32", 7)
    clean, cst, _ = h.group_norm(x, gamma, beta, G, EPS, act="silu")
    x[1, 3, 2, D] = bad                                  # image 1, group 1
    y, st, _ = h.group_norm(x, gamma, beta, G, EPS, act="silu")
    y, clean = h.host(y), h.host(clean)
    assert not np.isfinite(y[1, :, :, D:2 * D]).any()
    y[1, :, :, D:2 * D] = clean[1, :, :, D:2 * D]
    assert np.array_equal(y, clean)
    dx, dgamma, _ = (h.host(v) for v in h.backward(dy, x, h.host(st), gamma, beta, act="silu"))
    ok, okgamma, _ = (h.host(v) for v in h.backward(dy, np.where(np.isfinite(x), x, 0), h.host(cst), gamma, beta,
                                                    act="silu"))
    assert not np.isfinite(dx[1, :, :, D:2 * D]).any()
    dx[1, :, :, D:2 * D] = ok[1, :, :, D:2 * D]
    assert np.array_equal(dx, ok)
    assert not np.isfinite(dgamma[D:2 * D]).any()
    keep = np.r_[0:D, 2 * D:C]
    assert np.array_equal(dgamma[keep], okgamma[keep])


def test_gradient_is_that_of_the_forward_pass():
    # differences of the forward pass itself, in a direction: the error is the
    # fp32 rounding of the two sums (their difference over 2 h) and h^2
    shape = (2, 6, 5, 8, 2)
    x, gamma, beta, dy = _inputs(shape, "f32", 8)
    rng = np.random.default_rng(9)
    v = rng.standard_normal(x.shape)
    step = 2.0 ** -7
    st = h.host(h.group_norm(x, gamma, beta, 2, EPS, act="silu")[1])
    dx = h.host(h.backward(dy, x, st, gamma, beta, act="silu")[0])
    moved = [h.host(h.group_norm((x + s * step * v).astype(np.float32), gamma, beta, 2, EPS, act="silu")[0])
             for s in (1, -1)]
    slope = ((moved[0] - moved[1]) * dy).sum() / (2 * step)
    size = np.sqrt((dx ** 2).sum() * (v ** 2).sum())
    assert abs(slope - (dx * v).sum()) < 1e-3 * size


@pytest.mark.parametrize("act", ["relu", "silu"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(2, 10, 9, 24, 8), (1, 150, 151, 8, 1), (2, 9, 11, 33, 11)], ids=str)
def test_apply_gives_the_forward_result_again(shape, dtype, act):
    N, H, W, C, G = shape
    x, gamma, beta, _ = _inputs(shape, dtype, 10)
    y, st, q = h.group_norm(x, gamma, beta, G, EPS, dtype, act, ckpt=True)
    again = h.like(y)
    flags = h.IO[dtype] | h.ACT[act]
    g, b = h.dev(gamma), h.dev(beta)
    B.check(B.wino_group_norm_apply_nhwc(h.dev(x, dtype), st, g, b, again, N, C, H, W, G, flags))
    assert torch.equal(y, again)
    # from the checkpoint: the oracle's values of it
    B.check(B.wino_group_norm_apply_nhwc(q, st, g, b, again, N, C, H, W, G, flags | B.WINO_FLAG_ACT8))
    v = train.act8_unpack(*h.split_ckpt(q, N, H, W, C))
    s = h.host(st)
    ref = train.act(train.normed(v, s[..., 0], s[..., 1]) * gamma + beta, act)
    kappa = _kappa(v, G, s[..., 1])
    bound = h.SUM * (1 + kappa) * (1.1 * np.abs(gamma).max() * (1 + kappa) + np.abs(beta).max())
    assert (np.abs(h.host(again) - ref) <= bound + h.HALF_ULP[dtype] * np.abs(ref)).all()


def test_calls_on_another_stream_and_in_a_graph():
    shapes = [(2, 14, 14, 32, 8), (1, 150, 151, 8, 1)]
    for shape in shapes:
        N, H, W, C, G = shape
        x, gamma, beta, dy = _inputs(shape, "f32", 11)
        flags = B.WINO_FLAG_SILU
        xt, dyt, g, b = h.dev(x), h.dev(dy), h.dev(gamma), h.dev(beta)
        y, dx, st = h.like(xt), h.like(xt), torch.zeros((N, G, 2), device=h.DEV)
        q = torch.zeros(B.wino_act8_bytes(N, C, H, W), dtype=torch.int8, device=h.DEV)
        dgamma, dbeta = h.like(g), h.like(b)
        n1 = B.wino_group_norm_workspace_bytes(N, C, H, W, G, flags)
        n2 = B.wino_group_norm_backward_workspace_bytes(N, C, H, W, G, flags | B.WINO_FLAG_ACT8)
        ws = h.space(max(n1, n2))

        def step():
            B.check(B.wino_group_norm_nhwc(xt, g, b, y, st, q, N, C, H, W, G, EPS, flags, ws, n1))
            B.check(B.wino_group_norm_backward_nhwc(dyt, q, st, g, b, dx, dgamma, dbeta, N, C, H, W, G,
                                                    flags | B.WINO_FLAG_ACT8, ws, n2))
        outs = (y, st, q, dx, dgamma, dbeta)
        step()
        torch.cuda.synchronize()
        first = [o.clone() for o in outs]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        for o in outs:
            o.zero_()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, o) for a, o in zip(first, outs))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for i in range(3):
            xt.copy_(h.dev(x * (1.0 + i)))
            for o in outs:
                o.zero_()
            ws.fill_(float("nan"))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            got = [o.clone() for o in outs]
            step()
            torch.cuda.synchronize()
            assert all(torch.equal(a, o) for a, o in zip(got, outs))


def test_workspace_is_not_written_past_its_size():
    for shape in [(1, 150, 151, 8, 1), (2, 14, 14, 32, 8)]:
        N, H, W, C, G = shape
        x, gamma, beta, dy = _inputs(shape, "f32", 12)
        xt, y, g, b = h.dev(x), h.like(h.dev(x)), h.dev(gamma), h.dev(beta)
        st = torch.zeros((N, G, 2), device=h.DEV)
        wsb = B.wino_group_norm_workspace_bytes(N, C, H, W, G, 0)
        ws = h.space(wsb)
        B.check(B.wino_group_norm_nhwc(xt, g, b, y, st, None, N, C, H, W, G, EPS, 0, ws, wsb))
        wsb2 = B.wino_group_norm_backward_workspace_bytes(N, C, H, W, G, 0)
        ws2 = h.space(wsb2)
        B.check(B.wino_group_norm_backward_nhwc(y, xt, st, g, b, h.like(y), None, None, N, C, H, W, G, 0, ws2, wsb2))
        torch.cuda.synchronize()
        assert torch.isnan(ws[wsb // 4:]).all() and torch.isnan(ws2[wsb2 // 4:]).all()


def test_offsets_past_32_bits():
    # 2^31 + 2^25 elements in bf16: the last image's values against torch in 32 bits
    N, H, W, C, G = 65, 512, 1024, 64, 8
    x = torch.empty((N, H, W, C), dtype=torch.bfloat16, device=h.DEV)
    gen = torch.Generator(device=h.DEV)
    gen.manual_seed(0)
    x[:-1].fill_(1.0)
    x[-1].copy_(torch.randn((H, W, C), generator=gen, device=h.DEV))
    y = torch.empty_like(x)
    st = torch.zeros((N, G, 2), device=h.DEV)
    q = torch.empty(B.wino_act8_bytes(N, C, H, W), dtype=torch.int8, device=h.DEV)
    wsb = B.wino_group_norm_workspace_bytes(N, C, H, W, G, B.WINO_IO_BF16)
    ws = h.space(wsb)
    B.check(B.wino_group_norm_nhwc(x, None, None, y, st, q, N, C, H, W, G, EPS, B.WINO_IO_BF16, ws, wsb))
    last = x[-1].double().view(H * W, G, C // G)
    mean, var = last.mean((0, 2)), last.var((0, 2), unbiased=False)
    ref = ((last - mean[:, None]) / torch.sqrt(var[:, None] + EPS)).view(H, W, C)
    assert float((y[-1].double() - ref).abs().max()) <= 2.0 ** -8 * float(ref.abs().max())
    assert float(y[0].abs().max()) == 0.0
    v = torch.empty_like(x)
    B.check(B.wino_act8_unpack_nhwc(q, v, N, C, H, W, B.WINO_IO_BF16))
    assert torch.equal(v[0], x[0])
    # the last image's codes and rows, as 32-bit arithmetic gives them
    X = N * H * W * C
    rows = q[X:].view(torch.float32).view(N, C, 2)[-1]
    f = x[-1].float()
    lo, hi = f.amin((0, 1)), f.amax((0, 1))
    half, most = 0.5 * hi - 0.5 * lo, torch.full_like(lo, 127.0)      # divided as tensors: rounded once
    assert torch.equal(rows[:, 0], 0.5 * lo + 0.5 * hi) and torch.equal(rows[:, 1], half / most)
    codes = torch.round((f - rows[:, 0]) * (most / half))
    assert torch.equal(q[X - H * W * C:X].view(H, W, C).float(), codes)
    assert torch.equal(v[-1], (codes * rows[:, 1] + rows[:, 0]).bfloat16())
