"""Seeded random training calls, element by element against the fp64 oracle with the bounds
of test_gpu_norm_close.py and test_gpu_wgrad_scale.py: odd sizes, groups of one channel up
to one for all, every type, activation and source, tensors on and off 16-byte addresses."""
import math
import random

import numpy as np
import pytest

import test_gpu_norm_close as close
import test_gpu_wgrad_scale as scale
import train_helpers as h
from oracle import train

pytestmark = pytest.mark.gpu

U, EPS = h.U32, 1e-5


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw(seed):
    rng = random.Random(seed)
    N, H, W, C, K = _log(rng, 1, 17), _log(rng, 1, 60), _log(rng, 1, 60), _log(rng, 1, 140), _log(rng, 1, 140)
    if rng.random() < 0.5:
        C, K = (C + 7) // 8 * 8, (K + 3) // 4 * 4
    while N * H * W * max(C, K) > 600000:
        H, W = (H + 1) // 2, (W + 1) // 2
    return {"shape": (N, H, W, C, rng.choice([g for g in range(1, C + 1) if C % g == 0])), "K": K,
            "act": rng.choice(["none", "relu", "silu"]), "dtype": rng.choice(["f32", "f16", "bf16"]),
            "shift": rng.choice([0.5, 30.0]), "offset": rng.choice([0, 0, 1]), "ckpt": rng.random() < 0.5,
            "norm": rng.random() < 0.6, "pad": rng.choice([0, 1, 1, 1, 2])}


@pytest.mark.parametrize("seed", range(48))
def test_norm(seed):
    d = _draw(seed)
    shape, dtype, act = d["shape"], d["dtype"], d["act"]
    x, gamma, beta, dy = close._inputs(shape, dtype, d["shift"], seed)
    C, G = shape[3], shape[4]
    y, st, q = h.group_norm(x, gamma, beta, G, EPS, dtype, act, ckpt=True, offset=d["offset"])
    packed = train.act8_pack(x)
    for mine, ref in zip(h.split_ckpt(q, *shape[:4]), packed):
        assert np.array_equal(mine, ref)
    st = h.host(st)
    n = train.normed(x, st[..., 0], st[..., 1])
    z = n * gamma + beta
    ref = train.act(z, act)
    bound = 1.1 * close._off_z(n, 2 * U * np.abs(n), gamma, beta)
    if act == "silu":
        bound += np.abs(ref) * (2 * np.abs(z) + 8) * U
    bound = bound * 1.01 + h.HALF_ULP[dtype] * (np.abs(ref) + bound) + 2.0 ** -25 * (dtype == "f16")
    assert (np.abs(h.host(y) - ref) <= bound).all()
    if d["ckpt"]:
        codes, centre, step = packed
        v = train.act8_unpack(*packed)
        mean, rstd = close._spread(st[..., 0], C), close._spread(st[..., 1], C)
        n = train.normed(v, st[..., 0], st[..., 1])
        part, middle = np.abs(codes * step[:, None, None].astype(np.float64)), centre[:, None, None].astype(np.float64)
        off_n = U * (np.abs(n) + rstd * (part + 2 * np.abs(middle - mean))) if act == "silu" else \
            U * (2 * np.abs(n) + rstd * (part + np.abs(v)))
        off_n = off_n * 1.01
    else:
        v, off_n = x, 2 * U * np.abs(n)
    dy = close._for_relu(dy, n, off_n, gamma, beta, act)
    got = h.backward(dy, q if d["ckpt"] else x, st, gamma, beta, dtype, act, d["ckpt"], d["offset"])
    close._check_backward(got, dy, v, off_n, st, gamma, beta, dtype, act)


@pytest.mark.parametrize("seed", range(100, 164))
def test_weight_gradient(seed):
    d = _draw(seed)
    (N, H, W, C, G), K, pad, dtype, ckpt = d["shape"], d["K"], d["pad"], d["dtype"], d["ckpt"]
    if min(H, W) + 2 * pad < 3:
        pad = 1
    x, dy, _, _, rng = scale._inputs((N, H, W, C, K, pad), dtype, 0, -6 if dtype == "f16" else -40, seed)
    packed = train.act8_pack(x)
    codes, centre, step = packed
    v = train.act8_unpack(*packed) if ckpt else x.astype(np.float64)
    source = h.make_ckpt(*packed) if ckpt else x
    if d["norm"]:
        gamma = (1 + 0.2 * rng.standard_normal(C)).astype(np.float32).astype(np.float64)
        beta = (0.5 * rng.standard_normal(C)).astype(np.float32).astype(np.float64)
        st = np.stack(train.group_stats(x, G, EPS), -1).astype(np.float32).astype(np.float64)
        n = train.normed(v, st[..., 0], st[..., 1])
        z = n * gamma + beta
        a = train.act(z, d["act"])
        mean, rstd = (np.repeat(st[..., i], C // G, axis=1) for i in range(2))
        if ckpt:
            reach = (np.abs(centre - mean) + 127.0 * step) * rstd
            most = (np.abs(gamma) * reach + np.abs(beta)).max(axis=0)
            off_n = 6 * U * np.broadcast_to(reach[:, None, None], n.shape)
        else:
            most = 2 * np.abs(gamma) * np.sqrt(C // G * H * W) + np.abs(beta)
            off_n = 4 * U * np.abs(n)
        off_a = 1.1 * (off_n * np.abs(gamma) + 3 * U * (np.abs(n * gamma) + np.abs(beta)))
        if d["act"] == "silu":
            off_a = off_a + np.abs(a) * (2 * np.abs(z) + 8) * U
        dg = scale._call(source, dy, pad, dtype, (N, C, H, W, K), ckpt, st, gamma, beta, d["act"], d["offset"])
    else:
        a, off_a = v, 4 * U * np.abs(v) if ckpt else None
        most = (np.abs(centre) + 127.0 * step).max(axis=0).astype(np.float64) if ckpt else scale._most(x)
        if ckpt:
            off_a = off_a + 4 * U * np.abs(centre)[:, None, None]
        dg = scale._call(source, dy, pad, dtype, (N, C, H, W, K), ckpt, offset=d["offset"])
    scale._check(dg, a, dy, pad, most, scale._most(dy), off_a)
