"""Norm and rotation of queries and keys, and its backward pass, against 64 bits."""
import numpy as np
import pytest
import torch

from block_helpers import (B, DEV, HALF_ULP, IO, U32, O, angles, dev, host, ints, norm_tol, space, stored, table, untouched,
                           view, within)
from train_helpers import rounded

pytestmark = pytest.mark.gpu
EPS = 1e-6

# N, Lq, Lk, Hq, Hk, D, R: one token; teams of 2 to 64 lanes; runs of heads that end
# inside four; widths of every vector size and of none; parts of a head turned
SIZES = [(1, 1, 1, 1, 1, 2, 2), (8, 1, 1, 8, 2, 64, 64), (2, 37, 11, 4, 2, 64, 32), (3, 50, 77, 5, 3, 40, 40),
         (2, 9, 130, 1, 1, 128, 128), (2, 33, 5, 3, 1, 96, 48), (1, 70, 3, 2, 2, 7, 4), (1, 13, 19, 9, 4, 1, 0),
         (2, 21, 8, 6, 5, 80, 16), (1, 300, 40, 4, 4, 33, 32), (1, 17, 6, 2, 1, 24, 24), (2, 5, 64, 3, 2, 128, 6)]


def make(size, dtype, seed, T):
    N, Lq, Lk, Hq, Hk, D, R = size
    rng = np.random.default_rng(seed)
    d = {x: rounded(rng.standard_normal((N, L, H, D)) * np.exp(0.5 * rng.standard_normal(D)), dtype)
         for x, L, H in (("q", Lq, Hq), ("k", Lk, Hk))}
    for x in "qk":
        d["g" + x] = (1 + 0.3 * rng.standard_normal(D)).astype(np.float32)
        d["dy" + x] = rounded(rng.standard_normal(d[x].shape), dtype)
        d[x + "pos"] = rng.integers(0, T, d[x].shape[:2]) if T else None
    d["rot"] = table(T or max(Lq, Lk), R, rng) if R else None
    return d


def call(d, size, dtype, pairs=False, gap=0, offset=0, back=False, only_q=False, want=(True, True)):
    N, Lq, Lk, Hq, Hk, D, R = size
    flags = IO[dtype] | (B.WINO_FLAG_PAIRS if pairs else 0)
    ldq, ldk = Hq * D + gap, Hk * D + gap
    (q, _), (k, _) = view(d["q"], dtype, ldq, offset), view(d["k"], dtype, ldk, offset)
    rot = None if d["rot"] is None else dev(d["rot"])
    T = 0 if rot is None else rot.shape[0]
    gq, gk = (None if d["g" + x] is None else dev(d["g" + x]) for x in "qk")
    given = (q, None if only_q else k, gq, gk, rot, ints(d["qpos"]), ints(d["kpos"]))
    shape = (N, Lq, Lk, Hq, Hk, D, R, T, ldq, ldk, EPS, flags)
    if not back:
        yq, yk = (dev(np.full(d[x].shape, np.nan), dtype, offset) for x in "qk")
        B.check(B.wino_qk_norm_nhwc(*given, yq, yk, *shape))
        return yq, yk
    dq, dk = (view(np.full(d[x].shape, np.nan), dtype, ld, offset, 7.0) for x, ld in (("q", ldq), ("k", ldk)))
    dgq, dgk = (torch.full((D,), float("nan"), device=DEV) if w else None for w in want)
    wsb = B.wino_qk_norm_backward_workspace_bytes(N, Lq, Lk, Hq, Hk, D, flags)
    ws = space(wsb)
    B.check(B.wino_qk_norm_backward_nhwc(dev(d["dyq"], dtype, offset), dev(d["dyk"], dtype, offset), *given, dq[0],
                                         dk[0], dgq, dgk, *shape, ws if any(want) else None, wsb if any(want) else 0))
    assert untouched(dq[1], dq[0], 7.0) and untouched(dk[1], dk[0], 7.0)
    assert bool(torch.isnan(ws[(wsb + 3) // 4:]).all())
    return dq[0], dk[0], dgq, dgk


def check_forward(d, size, dtype, got, pairs):
    for x, y, L in zip("qk", got, size[1:3]):
        v = d[x].astype(np.float64)
        c, s = (np.zeros((size[0], L, 1, 0)),) * 2 if d["rot"] is None else angles(d["rot"], d[x + "pos"], size[0], L)
        want = O.head_norm(v, d["g" + x], c, s, EPS, pairs)
        within(y, want, stored(want, norm_tol(v, d["g" + x], c, s, EPS, pairs), dtype), x)


def check_backward(d, size, dtype, got, pairs):
    N, D = size[0], size[5]
    for i, (x, L) in enumerate(zip("qk", size[1:3])):
        v, dy = d[x].astype(np.float64), d["dy" + x].astype(np.float64)
        c, s = (np.zeros((N, L, 1, 0)),) * 2 if d["rot"] is None else angles(d["rot"], d[x + "pos"], N, L)
        dx, dg, absolute = O.head_norm_backward(dy, v, d["g" + x], c, s, EPS, pairs)
        r = 1 / np.sqrt((v * v).mean(-1, keepdims=True) + EPS)
        n, g = np.abs(v * r), 1.0 if d["g" + x] is None else np.abs(d["g" + x])
        # |dz| as a sum of absolute terms; then the mean of D products and D + 16 roundings
        dz = np.abs(dy) + O.turn(np.abs(dy), np.abs(c), np.abs(s), pairs).clip(0) + O.turn(
            np.abs(dy), np.abs(c), -np.abs(s), pairs).clip(0) if d["rot"] is not None else np.abs(dy)
        e = (2 * D + 32) * U32
        within(got[i], dx, stored(dx, e * r * (dz * g + n * (dz * g * n).mean(-1, keepdims=True)), dtype), "d" + x)
        if got[2 + i] is not None:
            count = N * L * v.shape[2]
            within(got[2 + i], dg, (D + 32 + min(count, 512)) * U32 * (dz * n).sum((0, 1, 2)), "dg" + x)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("size", SIZES)
def test_norm(size, dtype):
    for pairs, T, gap, offset in ((False, 0, 0, 0), (True, 1000, 0, 0), (False, 50, 8, 0), (True, 0, 3, 1)):
        d = make(size, dtype, 11, T)
        check_forward(d, size, dtype, call(d, size, dtype, pairs, gap, offset), pairs)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("size", SIZES)
def test_norm_backward(size, dtype):
    for pairs, T, gap, offset in ((False, 0, 0, 0), (True, 1000, 8, 0), (False, 50, 3, 1)):
        d = make(size, dtype, 12, T)
        check_backward(d, size, dtype, call(d, size, dtype, pairs, gap, offset, back=True), pairs)


def test_without_gamma_and_keys():
    size = (2, 20, 20, 4, 4, 64, 64)
    d = make(size, "bf16", 13, 0)
    d["gq"] = d["gk"] = None
    check_forward(d, size, "bf16", call(d, size, "bf16"), False)
    check_backward(d, size, "bf16", call(d, size, "bf16", back=True), False)
    yq, yk = call(d, size, "bf16", only_q=True)
    both = call(d, size, "bf16")
    assert torch.equal(yq, both[0]) and bool(torch.isnan(yk).all())
    dq, dk, dgq, dgk = call(d, size, "bf16", back=True, only_q=True)
    whole = call(d, size, "bf16", back=True)
    assert torch.equal(dq, whole[0]) and torch.equal(dgq, whole[2]) and bool(torch.isnan(dgk).all())
    for want in ((False, True), (True, False), (False, False)):
        part = call(d, size, "bf16", back=True, want=want)
        assert all(p is None or torch.equal(p, w) for p, w in zip(part, whole))


@pytest.mark.parametrize("pairs", [False, True])
def test_position_outside_the_table(pairs):
    size = (1, 6, 6, 2, 2, 64, 32)
    d = make(size, "f32", 14, 40)
    good = [t.clone() for t in call(d, size, "f32", pairs)]
    d["qpos"][0, 2], d["qpos"][0, 4], d["kpos"][0, 0] = 40, -1, 2**31 - 1
    got = call(d, size, "f32", pairs)
    turned = np.concatenate(O.pair_index(32, pairs))
    for g, w, at in ((got[0], good[0], [2, 4]), (got[1], good[1], [0])):
        g, w = host(g), host(w)
        for t in range(6):
            inside = np.isin(np.arange(64), turned)
            assert np.array_equal(g[0, t][:, ~inside], w[0, t][:, ~inside])
            assert np.isnan(g[0, t][:, inside]).all() if t in at else np.array_equal(g[0, t], w[0, t])


def test_views_of_one_projection_and_in_one_gradient():
    """q and k from one tensor, their gradients into one."""
    N, L, H, D = 2, 45, 3, 40
    rng = np.random.default_rng(15)
    qkv = rounded(rng.standard_normal((N, L, 3 * H, D)), "bf16")
    t = dev(qkv, "bf16")
    g = torch.full_like(t, 7.0)
    dyq, dyk = (dev(rng.standard_normal((N, L, H, D)), "bf16") for _ in "qk")
    ld = 3 * H * D
    args = (t[:, :, :H], t[:, :, H:2 * H], None, None, None, None, None)
    size = (N, L, L, H, H, D, 0, 0, ld, ld, EPS, B.WINO_IO_BF16)
    yq, yk = torch.empty_like(dyq), torch.empty_like(dyk)
    B.check(B.wino_qk_norm_nhwc(*args, yq, yk, *size))
    B.check(B.wino_qk_norm_backward_nhwc(dyq, dyk, *args, g[:, :, :H], g[:, :, H:2 * H], None, None, *size))
    none = np.zeros((N, L, 1, 0))
    for y, dy, x, dx in ((yq, dyq, qkv[:, :, :H], g[:, :, :H]), (yk, dyk, qkv[:, :, H:2 * H], g[:, :, H:2 * H])):
        x = x.astype(np.float64)
        want = O.head_norm(x, None, none, none, EPS)
        within(y, want, stored(want, norm_tol(x, None, none, none, EPS, False), "bf16"))
        want = O.head_norm_backward(host(dy), x, None, none, none, EPS)[0]
        assert np.abs(host(dx) - want).max() <= 2 * HALF_ULP["bf16"] * np.abs(want).max()
    assert bool((g[:, :, 2 * H:] == 7).all())


def test_long_sums_of_gamma():
    """A million terms of one sign: parts a thread, then workgroups in turn."""
    N, L, H, D = 4, 40000, 8, 8
    x = np.ones((N, L, H, D), np.float32)
    t, dy = dev(x), dev(x)
    dx, dg = torch.empty_like(t), torch.empty(D, device=DEV)
    wsb = B.wino_qk_norm_backward_workspace_bytes(N, L, 0, H, 0, D, 0)
    B.check(B.wino_qk_norm_backward_nhwc(dy, None, t, None, None, None, None, None, None, dx, None, dg, None, N, L, 0, H,
                                         0, D, 0, 0, H * D, 0, 0.0, 0, space(wsb), wsb))
    # 1.28e6 terms: 40 a thread, 64 teams, 4 waves, 1024 workgroups by 64 threads: below 256 roundings
    within(dg, np.full(D, float(N * L * H)), 256 * U32 * N * L * H)
    assert np.abs(host(dx)).max() <= 32 * U32


def test_offsets_past_32_bits():
    """Tokens so far apart that elements pass 2^31."""
    N, L, H, D, ld = 1, 5, 1, 8, 1 << 29
    buf = torch.zeros(4 * ld + 64, dtype=torch.float16, device=DEV)
    x = buf.as_strided((N, L, H, D), (L * ld, ld, D, 1))
    rng = np.random.default_rng(16)
    v = rounded(rng.standard_normal((N, L, H, D)), "f16")
    x.copy_(torch.from_numpy(v))
    y = torch.empty((N, L, H, D), dtype=torch.float16, device=DEV)
    B.check(B.wino_qk_norm_nhwc(x, None, None, None, None, None, None, y, None, N, L, 0, H, 0, D, 0, 0, ld, 0, EPS,
                                B.WINO_IO_F16))
    none = np.zeros((N, L, 1, 0))
    want = O.head_norm(v.astype(np.float64), None, none, none, EPS)
    within(y, want, stored(want, norm_tol(v.astype(np.float64), None, none, none, EPS, False), "f16"))
