"""The gated layer and its backward pass against 64 bits."""
import numpy as np
import pytest
import torch

from block_helpers import O, gated, gated_back, gated_back_tol, gated_tol, host, within
from train_helpers import U32, rounded

pytestmark = pytest.mark.gpu

# N, C, H, W, K: one token; tokens, units and channels at and beside the tiles' edges;
# widths that are no whole words
SIZES = [(1, 1, 1, 1, 1), (1, 512, 1, 1, 200), (1, 64, 1, 3, 64), (2, 16, 8, 8, 65), (1, 40, 5, 7, 24), (1, 129, 9, 15, 63),
         (3, 33, 6, 7, 130), (1, 72, 16, 17, 128), (2, 7, 13, 5, 5), (1, 256, 2, 8, 96), (1, 1000, 1, 17, 40)]


def make(N, C, H, W, K, dtype, seed, bias=True):
    rng = np.random.default_rng(seed)
    x, dy = rounded(rng.standard_normal((N, H, W, C)), dtype), rounded(rng.standard_normal((N, H, W, K)), dtype)
    w = rounded(rng.standard_normal((2, K, C)) / np.sqrt(C), dtype)
    return x, w, (0.5 * rng.standard_normal((2, K))).astype(np.float32) if bias else None, dy


def flat(a):
    return a.astype(np.float64).reshape(-1, a.shape[-1])


def check(x, w, b, dtype, act, **kw):
    w64 = w.astype(np.float64)
    y, zg, zu = O.gated(flat(x), w64, b, act)
    got = gated(x, w, b, dtype, act, **kw)
    within(host(got).reshape(y.shape), y, gated_tol(flat(x), w64, b, act, y, zg, zu, dtype), "y")


def check_back(dy, x, w, b, dtype, act, **kw):
    w64 = w.astype(np.float64)
    *want, dz = O.gated_backward(flat(dy), flat(x), w64, b, act)
    got = gated_back(dy, x, w, b, dtype, act, **kw)
    tol = gated_back_tol(flat(dy), flat(x), w64, b, act, dz, want, dtype)
    for name, g, v, t in zip(("dx", "dw", "dbias"), got, want, tol):
        if g is not None:
            within(host(g).reshape(v.shape), v, t, name)
    return got


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("size", SIZES)
def test_gated(size, dtype):
    for act, bias, offset in (("silu", True, 0), ("relu", False, 0), ("none", True, 1)):
        x, w, b, _ = make(*size, dtype, 41, bias)
        check(x, w, b, dtype, act, offset=offset)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("size", SIZES)
def test_gated_backward(size, dtype):
    for act, bias, offset in (("silu", True, 0), ("relu", False, 0), ("none", True, 1)):
        x, w, b, dy = make(*size, dtype, 42, bias)
        check_back(dy, x, w, b, dtype, act, offset=offset)


@pytest.mark.parametrize("tokens", list(range(1, 20)) + [31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 255, 257])
def test_every_few_tokens(tokens):
    for dtype in ("bf16", "f32"):
        x, w, b, _ = make(1, 96, 1, tokens, 72, dtype, 43)
        check(x, w, b, dtype, "silu")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_many_tokens_in_parts(dtype):
    """The weights' gradient summed over tokens in parts."""
    x, w, b, dy = make(2, 48, 40, 33, 36, dtype, 44)
    check_back(dy, x, w, b, dtype, "silu")


def test_what_is_not_wanted():
    x, w, b, dy = make(1, 32, 9, 9, 40, "bf16", 45)
    whole = gated_back(dy, x, w, b, "bf16", "silu")
    for want in ((True, False, False), (False, True, False), (False, False, True), (True, False, True)):
        got = gated_back(dy, x, w, b, "bf16", "silu", want=want)
        assert all(g is None or torch.equal(g, a) for g, a in zip(got, whole))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_values_that_are_not_finite(dtype):
    """A token's NaN stays in its results, a large gate neither overflows nor leaves a NaN."""
    x, w, b, dy = make(1, 64, 12, 12, 48, dtype, 46)
    clean, grads = host(gated(x, w, b, dtype, "silu")), [host(g) for g in gated_back(dy, x, w, b, dtype, "silu")]
    x2 = x.copy()
    x2[0, 3, 4, 5] = np.nan
    y = host(gated(x2, w, b, dtype, "silu"))
    assert np.isnan(y[0, 3, 4]).all()
    y[0, 3, 4] = clean[0, 3, 4]
    assert np.array_equal(y, clean)
    dx = host(gated_back(dy, x2, w, b, dtype, "silu")[0])
    assert np.isnan(dx[0, 3, 4]).all()
    dx[0, 3, 4] = grads[0][0, 3, 4]
    assert np.array_equal(dx, grads[0])
    big = b.copy()
    big[0, 7], big[0, 8] = 300.0, -300.0
    y = host(gated(x, w, big, dtype, "silu"))
    assert np.isfinite(y).all() and np.all(np.abs(y[..., 8]) <= 1e-30)
    assert all(np.isfinite(host(g)).all() for g in gated_back(dy, x, w, big, dtype, "silu"))


def test_same_results_every_time():
    x, w, b, dy = make(2, 64, 30, 30, 48, "bf16", 47)
    a, c = gated_back(dy, x, w, b, "bf16", "silu"), gated_back(dy, x, w, b, "bf16", "silu")
    assert all(torch.equal(p, q) for p, q in zip(a, c))


def test_long_sums_of_the_bias():
    """Gradients of one sign over many tokens."""
    N, H, W, C, K = 4, 200, 200, 8, 8
    x, w = np.ones((N, H, W, C), np.float32), np.full((2, K, C), 0.125, np.float32)
    dy = np.ones((N, H, W, K), np.float32)
    dx, dw, db = gated_back(dy, x, w, None, "f32", "none")
    M = N * H * W
    # 160000 terms: a lane's two, 32 lanes, two waves, 1250 tiles by 16 threads; dw: parts of 2500 tokens, joined
    within(db, np.full((2, K), float(M)), 256 * U32 * M)
    within(dw, np.full((2, K, C), float(M)), 4096 * U32 * M)
