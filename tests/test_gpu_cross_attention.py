"""Cross attention and its backward pass against 64 bits."""
import numpy as np
import pytest
import torch

from block_helpers import (B, DEV, IO, O, attend, attend_back, attend_back_tol, attend_tol, dev, host, ints, space,
                           untouched, within)
from train_helpers import rounded

pytestmark = pytest.mark.gpu


def make(N, Lq, Lk, Hq, Hk, D, dtype, seed, sharp=2.0):
    rng = np.random.default_rng(seed)
    q, k, v = (rounded(s * rng.standard_normal((N, L, H, D)), dtype).astype(np.float64)
               for s, L, H in ((sharp, Lq, Hq), (1.0, Lk, Hk), (1.0, Lk, Hk)))
    return q, k, v, rng


def check(q, k, v, dtype, klen=None, mask=None, scale=None, **kw):
    scale = float(np.float32(scale or q.shape[-1] ** -0.5))
    kept = O.kept_keys(k.shape[0], k.shape[1], klen, mask)
    y, lse, p = O.attention(q, k, v, scale, kept)
    got, st = attend(q, k, v, scale, dtype, klen, mask, **kw)
    ty, tl = attend_tol(q, k, v, scale, kept, p, y, lse, dtype)
    within(got, y, ty, "y")
    if st is not None:
        within(st, lse, tl, "lse")


def check_back(dy, q, k, v, dtype, klen=None, mask=None, scale=None, **kw):
    scale = float(np.float32(scale or q.shape[-1] ** -0.5))
    kept = O.kept_keys(k.shape[0], k.shape[1], klen, mask)
    y, lse, _ = O.attention(q, k, v, scale, kept)
    y, lse = rounded(y, dtype).astype(np.float64), lse.astype(np.float32).astype(np.float64)
    *want, more = O.attention_backward(dy, q, k, v, y, lse, scale, kept)
    outs = attend_back(dy, q, k, v, y, lse, scale, dtype, klen, mask, **kw)
    tol = attend_back_tol(more, scale, kept, q.shape[-1], dtype, *want, lse)
    for name, (g, buf), w, t in zip(("dq", "dk", "dv"), outs, want, tol):
        within(g, w, t, name)
        assert untouched(buf, g, 7.0), name


# one token and one key; rows and keys at and beside the tiles' edges; few rows of many
# heads; every width class and widths that are no whole words
SIZES = [(1, 1, 1, 1, 1, 8), (2, 1, 77, 4, 2, 64), (1, 33, 64, 1, 1, 32), (2, 31, 65, 3, 3, 40), (1, 128, 63, 2, 1, 64),
         (1, 129, 127, 1, 1, 128), (2, 4, 129, 8, 1, 80), (1, 16, 200, 6, 3, 20), (1, 65, 40, 2, 2, 1), (1, 40, 70, 1, 1, 100),
         (3, 7, 300, 2, 2, 17), (1, 64, 33, 5, 5, 96)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("size", SIZES)
def test_attention(size, dtype):
    N, Lq, Lk, Hq, Hk, D = size
    q, k, v, rng = make(*size, dtype, 21)
    check(q, k, v, dtype)
    klen = rng.integers(0, Lk + 1, N)
    mask = rng.integers(0, 2, (N, Lk))
    check(q, k, v, dtype, klen=klen, lse=False)
    check(q, k, v, dtype, mask=mask, ld=(Hq * D + 8, 2 * Hk * D, 2 * Hk * D))
    check(q, k, v, dtype, klen=klen, mask=mask, ld=(None, Hk * D + 3, Hk * D + 5), offset=1)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("size", SIZES)
def test_attention_backward(size, dtype):
    N, Lq, Lk, Hq, Hk, D = size
    q, k, v, rng = make(*size, dtype, 22)
    dy = rounded(rng.standard_normal(q.shape), dtype).astype(np.float64)
    check_back(dy, q, k, v, dtype)
    klen = rng.integers(0, Lk + 1, N)
    mask = rng.integers(0, 2, (N, Lk))
    check_back(dy, q, k, v, dtype, klen=klen, ld=(Hq * D + 8, 2 * Hk * D, 2 * Hk * D))
    check_back(dy, q, k, v, dtype, klen=klen, mask=mask, ld=(None, Hk * D + 3, Hk * D + 5), offset=1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(1, 1, 5000, 2, 1, 64), (1, 100, 3000, 1, 1, 40), (2, 2, 1111, 16, 1, 128)])
def test_long_keys_in_parts(size, dtype):
    """Few rows: the keys in parts, joined; ragged, so that parts are empty for some images."""
    N, Lq, Lk, Hq, Hk, D = size
    assert B.wino_cross_attention_workspace_bytes(*size, IO[dtype]) > 0
    q, k, v, rng = make(*size, dtype, 23)
    dy = rounded(rng.standard_normal(q.shape), dtype).astype(np.float64)
    for klen in (None, [Lk // 3] * N, [1] * N, [0] * N):
        check(q, k, v, dtype, klen=klen)
        check_back(dy, q, k, v, dtype, klen=klen)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
def test_long_rows_in_parts(dtype):
    """Few keys: the rows in parts for dk and dv."""
    size = (1, 3000, 20, 2, 1, 64)
    q, k, v, rng = make(*size, dtype, 24)
    dy = rounded(rng.standard_normal(q.shape), dtype).astype(np.float64)
    check(q, k, v, dtype)
    check_back(dy, q, k, v, dtype, mask=rng.integers(0, 2, (1, 20)))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("junk", [np.nan, np.inf, -np.inf])
def test_keys_left_out_are_not_read(dtype, junk):
    N, Lq, Lk, Hq, Hk, D = 3, 40, 150, 2, 2, 64
    q, k, v, rng = make(N, Lq, Lk, Hq, Hk, D, dtype, 25)
    dy = rounded(rng.standard_normal(q.shape), dtype).astype(np.float64)
    klen, mask = [100, 150, 7], rng.integers(0, 2, (N, Lk))
    mask[1] = 0                                             # an image without keys
    out = ~O.kept_keys(N, Lk, klen, mask)
    k[out], v[out] = junk, junk
    check(q, k, v, dtype, klen=klen, mask=mask)
    check(q[:, :3], k, v, dtype, klen=klen, mask=mask)      # few rows
    check_back(dy, q, k, v, dtype, klen=klen, mask=mask)


def test_lengths_outside_the_range():
    q, k, v, _ = make(4, 5, 30, 1, 1, 32, "f32", 26)
    check(q, k, v, "f32", klen=[-3, 31, 2**31 - 1, -2**31])


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_values_that_are_not_finite(dtype):
    """A query's NaN stays in its row, a value's infinity in its column (NaN in fp32, whose
    operands are split)."""
    N, Lq, Lk, H, D = 1, 70, 90, 2, 64
    q, k, v, _ = make(N, Lq, Lk, H, H, D, dtype, 27)
    want = attend(q, k, v, 0.125, dtype)[0].clone()
    q2, v2 = q.copy(), v.copy()
    q2[0, 3, 1, 5], v2[0, 88, 0, 9] = np.nan, np.inf
    got, lse = attend(q2, k, v2, 0.125, dtype)
    same = np.ones(q.shape, bool)
    same[0, 3, 1], same[0, :, 0, 9] = False, False
    g, w = host(got), host(want)
    assert np.array_equal(g[same], w[same]) and np.isnan(g[0, 3, 1]).all()
    assert (np.isnan if dtype == "f32" else np.isposinf)(g[0, :, 0, 9]).all()
    assert np.isnan(host(lse)[0, 1, 3]) and np.isfinite(host(lse)).sum() == lse.numel() - 1


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rising", [True, False])
def test_scores_of_hundreds(dtype, rising):
    """Maxima that move all the way, or are there at once: exponentials neither overflow nor vanish."""
    N, Lq, Lk, H, D = 1, 40, 260, 1, 32
    q, k, v, _ = make(N, Lq, Lk, H, H, D, dtype, 28)
    ramp = np.linspace(0.1, 30.0, Lk)
    k = rounded(np.abs(k) * (ramp if rising else ramp[::-1])[None, :, None, None], dtype).astype(np.float64)
    check(np.abs(q), k, v, dtype, scale=0.5)
    check(-np.abs(q), k, v, dtype, scale=0.5)


@pytest.mark.parametrize("Lq", [1, 40])
def test_half_precision_keeps_many_small_shares(Lq):
    """One key of score 0 and 16384 of some -11.8: shares of 2^-17, half of fp16's normal
    range away from the largest, that sum to an eighth of a row.  Each is off by its own
    rounding alone, and by 2^-32 of the largest."""
    Lk, D = 16385, 8
    q, k, v = np.zeros((1, Lq, 1, D)), np.zeros((1, Lk, 1, D)), np.zeros((1, Lk, 1, D))
    q[..., 0] = 1.0
    k[0, :, 0, 0] = -11.78125 - np.arange(Lk) % 7 / 128.0
    k[0, 77, 0, 0] = 0.0
    v[0, :, 0, 0], v[0, :, 0, 1] = 1.0, np.arange(Lk) % 5 - 2.0
    v[0, 77] = 0.0
    y, lse, p = O.attention(q, k, v, 1.0, np.ones((1, Lk), bool))
    got, st = attend(q, k, v, 1.0, "f16")
    # in 32 bits scores are exact here; an exponent of 17 and its sum with the largest, exp2 and
    # the sums over the keys: (17 * 4 + 8 + Lk) 2^-24; P's rounding, 2^-11; y's, 2^-11
    rel = (17 * 4 + 8 + Lk) * 2.0 ** -24 + 2.0 ** -11
    tol = (p @ np.abs(v.transpose(0, 2, 1, 3))).transpose(0, 2, 1, 3) * (2 * rel) + 2.0 ** -32 * np.abs(v).sum(1)[:, None]
    within(got, y, tol + 2.0 ** -11 * np.abs(y) + 2.0 ** -25, "y")
    within(st, lse, np.full(lse.shape, 2 * rel), "lse")


@pytest.mark.parametrize("scale", [2.0 ** -140, 1e-30, 3.0])
def test_scales(scale):
    q, k, v, _ = make(1, 9, 70, 2, 1, 16, "f32", 29, sharp=0.5)
    check(q, k, v, "f32", scale=scale)


@pytest.mark.parametrize("up", [2.0 ** -14, 2.0 ** 9])
def test_half_precision_gradients_keep_their_range(up):
    """dy so small that dS would fall below fp16's least value, or so large that it would
    pass the greatest; rows of both in one call."""
    N, Lq, Lk, H, D = 1, 96, 600, 1, 64
    q, k, v, rng = make(N, Lq, Lk, H, H, D, "f16", 30)
    dy = rounded(up * rng.standard_normal(q.shape) * np.exp2(-2.0 * (np.arange(Lq) % 5))[None, :, None, None], "f16")
    check_back(dy.astype(np.float64), q, k, rounded(8 * v, "f16").astype(np.float64), "f16")


def test_keys_and_values_of_one_projection():
    """k and v views of one tensor, dk and dv into one; nothing else of it is written."""
    N, Lq, Lk, Hq, Hk, D = 2, 50, 70, 4, 2, 64
    rng = np.random.default_rng(31)
    kv = rounded(rng.standard_normal((N, Lk, 3, Hk, D)), "bf16")
    q, dy = (rounded(rng.standard_normal((N, Lq, Hq, D)), "bf16") for _ in "ab")
    t, qt = dev(kv, "bf16"), dev(q, "bf16")
    y, lse = torch.empty_like(qt), torch.empty((N, Hq, Lq), device=DEV)
    ld, size = 3 * Hk * D, (N, Lq, Lk, Hq, Hk, D)
    f = B.WINO_IO_BF16
    wsb = B.wino_cross_attention_workspace_bytes(*size, f)
    B.check(B.wino_cross_attention_nhwc(qt, t[:, :, 0], t[:, :, 2], None, None, y, lse, *size, Hq * D, ld, ld, 0.125, f,
                                        space(wsb), wsb))
    g, dq = torch.full_like(t, 7.0), torch.empty_like(qt)
    wsb = B.wino_cross_attention_backward_workspace_bytes(*size, f)
    B.check(B.wino_cross_attention_backward_nhwc(dev(dy, "bf16"), qt, t[:, :, 0], t[:, :, 2], y, lse, None, None, dq,
                                                 g[:, :, 0], g[:, :, 2], *size, Hq * D, ld, ld, 0.125, f, space(wsb), wsb))
    kept = np.ones((N, Lk), bool)
    k, v, qd = kv[:, :, 0].astype(np.float64), kv[:, :, 2].astype(np.float64), q.astype(np.float64)
    wy, wl, p = O.attention(qd, k, v, 0.125, kept)
    ty, tl = attend_tol(qd, k, v, 0.125, kept, p, wy, wl, "bf16")
    within(y, wy, ty)
    *want, more = O.attention_backward(dy.astype(np.float64), qd, k, v, host(y), host(lse), 0.125, kept)
    for a, w, tol in zip((dq, g[:, :, 0], g[:, :, 2]), want,
                         attend_back_tol(more, 0.125, kept, D, "bf16", *want, host(lse))):
        within(a, w, tol)
    assert bool((g[:, :, 1] == 7).all())


def test_same_results_every_time():
    q, k, v, rng = make(2, 300, 500, 4, 2, 64, "bf16", 32)
    a, b = attend(q, k, v, 0.125, "bf16"), attend(q, k, v, 0.125, "bf16")
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    dy = rng.standard_normal(q.shape)
    g, h = (attend_back(dy, q, k, v, host(a[0]), host(a[1]), 0.125, "bf16") for _ in "ab")
    assert all(torch.equal(x[0], y[0]) for x, y in zip(g, h))


def test_offsets_past_32_bits():
    """Keys of one image past 2^31 elements, the last ones scored highest."""
    Lk, D, ld = 9, 16, 1 << 28
    buf = torch.zeros((Lk - 1) * ld + 64, dtype=torch.bfloat16, device=DEV)
    kt = buf.as_strided((1, Lk, 1, D), (Lk * ld, ld, D, 1))
    q, k, v, rng = make(1, 3, Lk, 1, 1, D, "bf16", 33)
    kt.copy_(torch.from_numpy(k.astype(np.float32)))
    vt, qt = dev(v, "bf16"), dev(q, "bf16")
    y, lse = torch.empty_like(qt), torch.empty((1, 1, 3), device=DEV)
    size = (1, 3, Lk, 1, 1, D)
    B.check(B.wino_cross_attention_nhwc(qt, kt, vt, None, None, y, lse, *size, D, ld, D, 0.25, B.WINO_IO_BF16))
    kept = np.ones((1, Lk), bool)
    wy, wl, p = O.attention(q, k, v, 0.25, kept)
    ty, tl = attend_tol(q, k, v, 0.25, kept, p, wy, wl, "bf16")
    within(y, wy, ty)
    within(lse, wl, tl)
    # and the gradients written there
    dy = rounded(rng.standard_normal(q.shape), "bf16")
    dq, dv = torch.empty_like(qt), torch.empty_like(vt)
    gbuf = torch.zeros((Lk - 1) * ld + 64, dtype=torch.bfloat16, device=DEV)
    gk = gbuf.as_strided((1, Lk, 1, D), (Lk * ld, ld, D, 1))
    wsb = B.wino_cross_attention_backward_workspace_bytes(*size, B.WINO_IO_BF16)
    B.check(B.wino_cross_attention_backward_nhwc(dev(dy, "bf16"), qt, kt, vt, y, lse, None, None, dq, gk, dv, *size, D,
                                                 ld, D, 0.25, B.WINO_IO_BF16, space(wsb), wsb))
    *want, more = O.attention_backward(dy.astype(np.float64), q, k, v, host(y), host(lse), 0.25, kept)
    for a, w, t in zip((dq, gk, dv), want, attend_back_tol(more, 0.25, kept, D, "bf16", *want, host(lse))):
        within(a, w, t)
