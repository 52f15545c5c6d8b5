"""The gated layer's gradients in fp16 where what goes through the workspace, dzg and dzu, would
pass fp16's range: both ends, one token that is not finite, and tokens of both ends."""
import numpy as np
import pytest
import torch

from block_helpers import B, DEV, O, dev, gated_back, gated_back_tol, host, space, within
from train_helpers import rounded

pytestmark = pytest.mark.gpu

# N, H, W, C, K: results that take tiles of each shape, whole words and not
SIZES = [(1, 8, 9, 64, 96, 0), (1, 7, 9, 33, 70, 0), (2, 40, 33, 48, 40, 1), (4, 56, 56, 64, 128, 0), (4, 64, 65, 40, 1000, 0),
         (4, 64, 65, 24, 1000, 1)]


def half(a):
    return rounded(a, "f16").astype(np.float64)


def check(dy, x, w, b, act="silu", offset=0, rows=None):
    """dx of the tokens `rows` (of all: and dw, dbias) within their bounds: dz is kept to a relative
    2^-11, and to half a step of fp16 where the largest is at 2^-2 at least: 2^-23 of it."""
    flat = [a.reshape(-1, a.shape[-1]) for a in (dy, x)]
    keep = slice(None) if rows is None else rows
    *want, dz = O.gated_backward(flat[0][keep], flat[1][keep], w, b, act)
    s = 2.0 ** -2 / np.abs(dz).max()
    tol = gated_back_tol(flat[0][keep] * s, flat[1][keep], w, b, act, dz * s, [a * s for a in want], "f16")
    got = gated_back(dy, x, w, b, "f16", act, offset=offset)
    for name, g, v, t in list(zip(("dx", "dw", "dbias"), got, want, tol))[:1 if rows is not None else 3]:
        g = host(g)
        g = g.reshape(-1, g.shape[-1])[keep] if name == "dx" else g.reshape(v.shape)
        # the result's own rounding at the range's lower end does not scale
        within(g, v, t / s + 2.0 ** -25, name)


def make(size, dy, x, w, b):
    N, H, W, C, K, offset = size
    rng = np.random.default_rng(93)
    r = lambda *s: np.abs(rng.standard_normal(s)) + 0.25  # noqa: E731, of one sign, so that sums do not cancel
    return (half(dy * r(N, H, W, K)), half(x * r(N, H, W, C)), half(w * r(2, K, C) / C),
            np.float32(b * r(2, K)) if b else None), offset


@pytest.mark.parametrize("size", SIZES)
def test_gradients_below_the_range(size):
    """dz of some 2^-28: sums over many tokens, or units, are far above it."""
    (dy, x, w, b), offset = make(size, 2.0 ** -14, 2.0 ** 3, 2.0 ** -14, 2.0 ** -14)
    check(dy, x, w, b, "silu", offset)
    check(dy, x, w, b, "none", offset)
    (dy, x, w, b), offset = make(size, 2.0 ** -14, 2.0 ** -18, size[3], 0)
    check(dy, x, w, b, "silu", offset)


@pytest.mark.parametrize("size", SIZES)
def test_gradients_above_the_range(size):
    """dz of some 2^17 and more: weights and inputs are small, and so are dx and dw."""
    (dy, x, w, b), offset = make(size, 2.0 ** 8, 2.0 ** -21, 2.0 ** -8, 2.0 ** 9)
    check(dy, x, w, b, "silu", offset)
    check(dy, x, w, b, "relu", offset)


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("junk", [np.nan, np.inf])
def test_one_token_that_is_not_finite(size, junk):
    """Its infinity is no part of the largest value: the other tokens keep their bits."""
    (dy, x, w, b), offset = make(size, 2.0 ** -14, 2.0 ** -18, size[3], 0)
    dy[0, 2, 5, 7] = junk
    rows = np.arange(dy.size // dy.shape[-1]) != 2 * dy.shape[2] + 5
    check(dy, x, w, b, "silu", offset, rows)


@pytest.mark.parametrize("size", SIZES)
def test_tokens_of_both_ends(size):
    """Half of the tokens past the range, the others within it and kept with their bits."""
    (dy, x, w, b), offset = make(size, 1.0, 2.0 ** -21, 2.0 ** -8, 2.0 ** 9)
    first = np.arange(dy.size // dy.shape[-1]).reshape(dy.shape[:-1]) < dy.size // dy.shape[-1] // 2
    check(half(np.where(first[..., None], 2.0 ** 8 * dy, 2.0 ** -2 * dy)), x, w, b, "silu", offset)
    check(half(np.where(first[..., None], 2.0 ** -2 * dy, 2.0 ** 8 * dy)), x, w, b, "relu", offset)


def test_zero_gradients():
    (dy, x, w, b), _ = make(SIZES[0], 1.0, 1.0, 1.0, 1.0)
    for g in gated_back(0 * dy, x, w, b, "f16", "silu"):
        assert (host(g) == 0).all()


def test_a_captured_call_finds_its_power_at_every_replay():
    """Gradients within the range, below it and above it, by one graph and one workspace."""
    N, H, W, C, K, _ = SIZES[3]
    rng = np.random.default_rng(94)
    x, w, dy = (dev(rng.standard_normal(s) * f, "f16") for s, f in (((N, H, W, C), 1.0), ((2, K, C), 0.01), ((N, H, W, K), 1.0)))
    dx, dw, db = torch.zeros_like(x), torch.zeros_like(w), torch.zeros((2, K), device=DEV)
    size = (N, C, H, W, K, B.WINO_IO_F16 | B.WINO_FLAG_SILU)
    need = B.wino_gated_layer_backward_workspace_bytes(*size)
    ws = space(need)

    def step():
        B.check(B.wino_gated_layer_backward_nhwc(dy, x, w, None, dx, dw, db, *size, ws, need))
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    first = dy.clone()
    for f in (1.0, 2.0 ** -14, 2.0 ** 12, 2.0 ** -10, 1.0):
        dy.copy_(first * f)
        for t in (ws, dx, dw, db):
            t.fill_(float("nan"))
        graph.replay()
        got = [t.clone() for t in (dx, dw, db)]
        for t in (ws, dx, dw, db):
            t.fill_(float("nan"))
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (dx, dw, db)))
        # of 2^12, dzu is some 2^12 * 0.04 and dw, over 12544 tokens, 2^12 * 0.04 * 112 = 18000 in the mean
        # square: four times as much, which some of its 16384 values reach, is past fp16 itself
        assert all(bool(torch.isfinite(t).all()) for t in ((dx, db) if f > 1 else (dx, dw, db)))
