"""Cross attention where images times key heads are a multiple of eight, or 64 and more: workgroups
of a pair on one XCD, pairs rounded up to eight.  And queries, keys and values of one tensor."""
import random

import numpy as np
import pytest
import torch

from block_helpers import IO, B, O, attend_back_tol, attend_tol, dev, host, space, within
from test_gpu_cross_attention import check, check_back, make
from train_helpers import rounded

pytestmark = pytest.mark.gpu


def both(size, dtype, seed, **kw):
    N, Lq, Lk, Hq, Hk, D = size
    q, k, v, rng = make(*size, dtype, seed)
    dy = rounded(rng.standard_normal(q.shape), dtype).astype(np.float64)
    klen, mask = rng.integers(0, Lk + 1, N), rng.integers(0, 2, (N, Lk))
    for given in ({}, {"klen": klen}, {"klen": klen, "mask": mask}):
        check(q, k, v, dtype, **given, **kw)
        check_back(dy, q, k, v, dtype, **given, **kw)


# 8, 16 and 64 pairs: several tiles of rows and keys, shared heads, few rows
SIZES = [(8, 130, 150, 1, 1, 16), (2, 130, 200, 8, 4, 32), (4, 65, 300, 8, 4, 20), (16, 70, 129, 4, 4, 16), (4, 1, 200, 8, 2, 64),
         (8, 40, 70, 3, 3, 40), (1, 150, 90, 8, 8, 128)]
# in parts: rows' keys, keys' rows
PARTS = [(8, 2, 900, 4, 1, 64), (1, 100, 700, 8, 8, 16), (8, 700, 40, 1, 1, 32)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("size", SIZES)
def test_pairs_in_eights(size, dtype):
    assert size[0] * size[4] % 8 == 0
    both(size, dtype, 101)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("size", PARTS)
def test_pairs_in_eights_and_parts(size, dtype):
    N, Lq, Lk, Hq, Hk, D = size
    assert N * Hk % 8 == 0
    need = B.wino_cross_attention_backward_workspace_bytes(*size, IO[dtype])
    assert need > 3 * N * Hq * Lq * 4 + 48           # more than three numbers a row: parts
    both(size, dtype, 102)


@pytest.mark.parametrize("pairs", range(64, 73))
def test_pairs_rounded_up_to_eight(pairs):
    for size, dtype in (((pairs, 70, 90, 1, 1, 16), "bf16"), ((pairs, 3, 130, 2, 1, 24), "f16"), ((1, 66, 65, pairs, pairs, 8), "f32")):
        both(size, dtype, 103)


@pytest.mark.parametrize("seed", range(24))
def test_random_pairs(seed):
    """Pairs of either order, sizes over their logarithm."""
    rng = random.Random(3000 + seed)
    pairs = rng.choice([8, 16, 24, 40, 64, 67, 70, 80])
    Hk = rng.choice([h for h in range(1, pairs + 1) if pairs % h == 0])
    N, Hq, D = pairs // Hk, Hk * rng.choice([1, 1, 2, 3]), rng.choice([8, 16, 20, 33, 40, 64, 96, 128])
    Lq, Lk = int(2 ** rng.uniform(0, 8)), int(2 ** rng.uniform(0, 9))
    while N * Hq * Lq * Lk > 1200000:
        Lq, Lk = (Lq + 1) // 2, (Lk + 1) // 2
    both((N, Lq, Lk, Hq, Hk, D), rng.choice(["f32", "f16", "bf16"]), 3100 + seed, offset=rng.choice([0, 0, 1]),
         ld=rng.choice([(None,) * 3, (Hq * D + 8, 2 * Hk * D, 2 * Hk * D)]))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("N,L,Hq,Hk,D", [(2, 150, 4, 4, 32), (8, 67, 4, 2, 64), (1, 300, 3, 1, 40), (3, 1, 2, 2, 128), (2, 70, 2, 1, 9)])
def test_queries_keys_and_values_of_one_tensor(N, L, Hq, Hk, D, dtype):
    """The pixels' attention to themselves: q, k and v are views of one projection's tensor, dq, dk and
    dv of its gradient; nothing behind them is written."""
    H = Hq + 2 * Hk
    rng = np.random.default_rng(104)
    a, dy = rounded(rng.standard_normal((N, L, H + 1, D)), dtype), rounded(rng.standard_normal((N, L, Hq, D)), dtype)
    t, g = dev(a, dtype), dev(np.full(a.shape, 7.0), dtype)
    cut = (slice(0, Hq), slice(Hq, Hq + Hk), slice(Hq + Hk, H))
    views, grads = ([x[:, :, c] for c in cut] for x in (t, g))
    y, lse = torch.empty((N, L, Hq, D), dtype=t.dtype, device=t.device), torch.empty((N, Hq, L), device=t.device)
    size, ld, scale = (N, L, L, Hq, Hk, D), ((H + 1) * D,) * 3, 0.25
    need = B.wino_cross_attention_workspace_bytes(*size, IO[dtype])
    B.check(B.wino_cross_attention_nhwc(*views, None, None, y, lse, *size, *ld, scale, IO[dtype], space(need), need))
    need = B.wino_cross_attention_backward_workspace_bytes(*size, IO[dtype])
    B.check(B.wino_cross_attention_backward_nhwc(dev(dy, dtype), *views, y, lse, None, None, *grads, *size, *ld, scale,
                                                 IO[dtype], space(need), need))
    q, k, v = (a[:, :, c].astype(np.float64) for c in cut)
    kept = np.ones((N, L), bool)
    wy, wl, p = O.attention(q, k, v, scale, kept)
    ty, tl = attend_tol(q, k, v, scale, kept, p, wy, wl, dtype)
    within(y, wy, ty, "y")
    within(lse, wl, tl, "lse")
    *want, more = O.attention_backward(dy.astype(np.float64), q, k, v, host(y), host(lse), scale, kept)
    for name, x, w, tol in zip(("dq", "dk", "dv"), grads, want,
                               attend_back_tol(more, scale, kept, D, dtype, *want, host(lse))):
        within(x, w, tol, name)
    assert bool((g[:, :, H:] == 7).all())


@pytest.mark.parametrize("which", ["q", "kv"])
@pytest.mark.parametrize("ld", [1 << 22, (1 << 22) + 8])
def test_the_limit_of_tiles_straight_to_lds(ld, which):
    """Tokens 2^22 elements apart, and past it: rows of a tile reach over 2^29 bytes."""
    N, Lq, Lk, Hq, Hk, D = size = 1, 67, 70, 2, 1, 64
    q, k, v, rng = make(*size, "bf16", 105)
    dy = rounded(rng.standard_normal(q.shape), "bf16").astype(np.float64)
    lds = (ld if which == "q" else None, *(2 * (ld if which == "kv" else None,)))
    check(q, k, v, "bf16", mask=rng.integers(0, 2, (N, Lk)), ld=lds)
    check(q[:, :3], k, v, "bf16", ld=lds)
    check_back(dy, q, k, v, "bf16", klen=[66], ld=lds)
